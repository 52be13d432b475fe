"""Plain 64-bit forms of the paged cache's operators and of token log probabilities, for the tests (CPU torch)."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # a rounding's largest relative error


def norm_rope(x, gain, eps, pos, theta):
    """x [..., rows, heads, hd] float64; pos [rows]."""
    hd = x.shape[-1]
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    if theta is None:
        return x
    ang = pos.double()[:, None] * theta ** (-torch.arange(0, hd, 2).double() / hd)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def to_e4m3(x):
    """Values an e4m3 row stands for: codes of x 2^-e times 2^e, e the smallest exponent with max |x| <= 448 2^e."""
    a = x.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    m, e = torch.frexp(torch.where(bad | (a == 0), 448.0, a).double())
    e = e - 9 + (m > 0.875)
    y = (x * torch.pow(2.0, -e.double())).float().to(torch.float8_e4m3fn).double() * torch.pow(2.0, e.double())
    return torch.where(bad, float("nan"), y), e


def attention(q, k, v, start, scale):
    """q [R, hq, hd], k / v [n, hkv, hd] float64, row r sees positions <= start + r.  (out, tolerance) of a bf16 result whose
    weights are rounded to bf16 too: half a step of every weight and of the result, and the scores' fp32 sums."""
    R, hq, hd = q.shape
    n, hkv, _ = k.shape
    out, tol = torch.zeros(R, hq, hd, dtype=torch.float64), torch.zeros(R, hq, hd, dtype=torch.float64)
    for r in range(R):
        end = min(n, start + r + 1)
        for h in range(hq):
            kk, vv = k[:end, h * hkv // hq], v[:end, h * hkv // hq]
            s = kk @ q[r, h] * scale
            p = torch.softmax(s, 0)
            out[r, h] = p @ vv
            mag = p @ vv.abs()
            # a score's error: hd products summed and scaled in fp32; it moves a weight, and the sum, by as much
            ds = (hd + 8) * 2.0 ** -24 * ((kk.abs() @ q[r, h].abs()).max() * abs(scale)) + 2.0 ** -22
            tol[r, h] = (1 + 2.0 ** -6) * (HALF[torch.bfloat16] * (mag + out[r, h].abs()) + 4 * ds * mag) + 1e-30
    return out, tol


def logprobs(z, token, n):
    """(log probability, entropy, top tokens, their log probabilities, tolerance) of one row."""
    z = z.double()
    V = len(z)
    m = z.max()
    d = z - m
    p = torch.exp(d)
    S = p.sum()
    pn = p / S
    fin = p > 0
    ed = float((pn[fin] * d[fin].abs()).sum())
    H = float(torch.log(S) + ed)
    # S: an exponential's argument and value, and the additions a thread and the joins make
    tol = 2.0 ** -22 + 2.0 ** -23 * ed + 2.0 ** -24 * (40 + V / 2048)
    logp = d - torch.log(S)
    lp = float(logp[token]) if 0 <= token < V else float("nan")
    order = sorted(range(V), key=lambda i: (-float(z[i]), i))[:n] if V < 3000 else torch.sort(z, descending=True, stable=True)[1][:n].tolist()
    ids = [i for i in order if z[i] > -math.inf]
    top = [float(logp[i]) for i in ids]
    ids += [-1] * (n - len(ids))
    top += [-math.inf] * (n - len(top))
    return lp, H, ids, top, tol * (1 + ed)
