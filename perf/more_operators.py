"""Performance cases of the 8-bit products around the paged cache: rows turned into e4m3 codes with a scale for each block of
128 columns (as they are, after a residual's addition and an RMS norm, or after SwiGLU), matrices turned into codes with a scale
for each 128 x 128 block, and the matrix product of such rows and matrices.

A case is one pass through one operator, as a serving program calls it between the attention of a decode, verify or prefill
step.  run() computes the plain form with elementary torch operations in float32, or, where `own` is set, calls the framework's
operators.  Scales are float32, or powers of two in a byte (float8_e8m0fnu); those of rows lie block-major, [blocks][rows].
"""
import math

import torch

own = False
DEV = "cuda"
BLOCK, TOP, TINY = 128, 448.0, 2.0 ** -126
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the attention's output of a verified block before the output projection; a bf16 checkpoint's q/k/v matrix on loading
        dict(name="quantize_block", op="quantize", M=33, K=8192, dtype="bf16", scale="f32"),
        dict(name="quantize_matrix", op="matrix", M=10240, K=5120, dtype="bf16", scale="f32"),
        # between two products of a decode step, and of a prompt's chunk with the residual kept in float32 and bf16 rows beside the codes
        dict(name="rmsnorm_token", op="rmsnorm", M=1, K=3584, dtype="bf16", residual="bf16", y=False, scale="f32"),
        dict(name="rmsnorm_prompt", op="rmsnorm", M=4095, K=5120, dtype="bf16", residual="f32", y=True, scale="e8m0"),
        # between the gate/up and down products of a verified block, and of a prompt's chunk
        dict(name="swiglu_block", op="swiglu", M=33, K=25600, dtype="bf16", scale="f32"),
        dict(name="swiglu_prompt", op="swiglu", M=2047, K=18944, dtype="bf16", scale="e8m0"),
        # one token's q/k/v: the smallest call, a chain of latencies
        dict(name="matmul_token", op="matmul", M=1, N=4608, K=3584, out="bf16", scale="f32"),
        # a block of 32 drafts and its bonus position: the widest matrix of a layer, and the longest rows into a float32 residual
        dict(name="matmul_block", op="matmul", M=33, N=51200, K=5120, out="bf16", scale="f32"),
        dict(name="matmul_down", op="matmul", M=33, N=5120, K=25600, out="f32", scale="e8m0"),
        # eight blocks verified together
        dict(name="matmul_block8", op="matmul", M=264, N=10240, K=5120, out="bf16", scale="f32"),
        # prompts: few columns and long rows, and the widest matrix
        dict(name="matmul_chunk", op="matmul", M=511, N=3584, K=18944, out="bf16", scale="e8m0"),
        dict(name="matmul_prompt", op="matmul", M=4095, N=51200, K=5120, out="bf16", scale="f32"),
    ]


# widths and heights of the layers' matrices, [out][in]
SHAPES = [(4608, 3584), (3584, 3584), (37888, 3584), (3584, 18944), (10240, 5120), (5120, 8192), (51200, 5120), (5120, 25600),
          (512, 256), (256, 256), (1376, 256), (256, 688), (4096, 256)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["matmul", "matmul", "matmul", "rmsnorm", "swiglu", "quantize", "matrix"])
    scale = rng.choice(["f32", "e8m0"])
    if op == "matmul":
        N, K = rng.choice(SHAPES + [(_log_int(rng, 1, 51200), 16 * _log_int(rng, 1, 1600))] * 6)
        M = rng.choice([1, 9, 33, rng.randint(1, 65), _log_int(rng, 66, 4095), _log_int(rng, 1, 4095)])
        while N * K > 51200 * 5120:
            N = max(1, N // 2)
        return dict(op=op, M=M, N=N, K=K, out=rng.choice(["bf16", "bf16", "f32"]), scale=scale)
    K = rng.choice([256, 688, 3584, 5120, 8192, 18944, 25600, 16 * _log_int(rng, 1, 1600), 16 * _log_int(rng, 1, 1600)])
    M = rng.choice([1, 9, 33, rng.randint(1, 65), _log_int(rng, 1, 10240 if op == "matrix" else 4095)])
    while M * K > 10240 * 5120:
        M = max(1, M // 2)
    case = dict(op=op, M=M, K=K, dtype=rng.choice(["bf16", "bf16", "f32"]), scale=scale)
    if op == "rmsnorm":
        case |= dict(residual=rng.choice(["bf16", "f32", "none"]), y=rng.choice([True, False]))
    return case


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    M, K = case["M"], case["K"]
    es = 4 if case["scale"] == "f32" else 1
    size = lambda t: {"bf16": 2, "f32": 4, "none": 0}[t]  # noqa: E731
    if case["op"] == "matmul":
        N = case["N"]
        return {"bytes": (M + N) * K + (M + _blocks(N)) * _blocks(K) * es + M * N * size(case["out"]), "flops": 2 * M * N * K}
    if case["op"] == "matrix":
        return {"bytes": M * K * (size(case["dtype"]) + 1) + _blocks(M) * _blocks(K) * es, "flops": 3 * M * K}
    left = M * K + M * _blocks(K) * es
    if case["op"] == "quantize":
        return {"bytes": M * K * size(case["dtype"]) + left, "flops": 3 * M * K}
    if case["op"] == "swiglu":
        return {"bytes": 2 * M * K * size(case["dtype"]) + left, "flops": 8 * M * K}
    res = size(case["residual"])
    return {"bytes": M * K * (size(case["dtype"]) + 2 * res + (2 if case["y"] else 0)) + 4 * K + left, "flops": 8 * M * K}


# ---- inputs -----------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    M, K = case["M"], case["K"]

    def rows(m, k):  # activations: a few channels stand out, and rows differ in size
        loud = torch.where(torch.rand(k, generator=g, device=DEV) < 0.01, 20.0, 1.0)
        return normal(m, k) * loud * torch.exp(0.5 * normal(m, 1))

    st = {"case": case}
    if case["op"] == "matmul":
        N = case["N"]
        st["x"], st["xs"] = _quantise(rows(M, K), case["scale"])
        w = normal(N, K).mul_(0.02)
        w *= torch.exp(0.5 * normal(N, 1))
        st["w"], st["ws"] = _quantise_matrix(w, case["scale"])
        del w
        if own:
            from paper_2608_14787_amd import sdd
            st["matrix"] = sdd.E4M3Matrix(st["w"], st["ws"])
            st["room"] = st["matrix"].workspace(M)
    elif case["op"] == "matrix":
        st["x"] = (normal(M, K).mul_(0.02) * torch.exp(0.5 * normal(M, 1))).to(TYPES[case["dtype"]])
    elif case["op"] == "swiglu":
        st["x"] = torch.cat([2.0 * normal(M, K), rows(M, K)], dim=1).to(TYPES[case["dtype"]])
    else:
        st["x"] = rows(M, K).to(TYPES[case["dtype"]])
        if case["op"] == "rmsnorm":
            st["gain"] = 1 + 0.1 * normal(K)
            if case["residual"] != "none":
                st["res"] = (4.0 * rows(M, K)).to(TYPES[case["residual"]])
                st["res_out"] = torch.empty_like(st["res"])
    return st


# ---- one pass ---------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if own:
        return _own(case, state)
    return {"quantize": _rows, "matrix": _matrix, "rmsnorm": _rmsnorm, "swiglu": _swiglu, "matmul": _matmul}[case["op"]](case, state)


def _own(case, st):
    from paper_2608_14787_amd import sdd
    if case["op"] == "matmul":
        return st["matrix"].matmul(st["x"], st["xs"], dtype=TYPES[case["out"]], ws=st["room"])
    if case["op"] == "matrix":
        return sdd.e4m3_quantize_matrix(st["x"], scale=case["scale"])
    if case["op"] == "quantize":
        return sdd.e4m3_quantize(st["x"], scale=case["scale"])
    if case["op"] == "swiglu":
        return sdd.e4m3_swiglu(st["x"], scale=case["scale"])
    return sdd.e4m3_rmsnorm(st["x"], st["gain"], eps=EPS, residual=st.get("res"), residual_out=st.get("res_out"), y=case["y"],
                            scale=case["scale"])


def _tiles(x, high):
    """x [M, K] as blocks [M / high, high, K / 128, 128], zeros behind its ends."""
    M, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % BLOCK, 0, -M % high))
    return x.view(-1, high, _blocks(K), BLOCK)


def _encode(x, high, scale):
    """Codes float8_e4m3fn like x [M, K] (float32), and the scales [M / high, K / 128] of its blocks."""
    M, K = x.shape
    t = _tiles(x, high)
    a = t.abs().amax((1, 3))
    bad = ~torch.isfinite(a)
    if scale == "f32":
        s = torch.where(a > 0, (a / TOP).clamp(min=TINY), 1.0).masked_fill(bad, 1.0)
        held = s
    else:
        m, e = torch.frexp(a.masked_fill(bad, 1.0))
        e = torch.where(a > 0, e - 9 + (m > 0.875), 0).clamp(-126, 127).masked_fill(bad, 0)
        s = torch.exp2(e.float())
        held = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    y = (t / s[:, None, :, None]).clamp(-TOP, TOP).masked_fill(bad[:, None, :, None], math.nan)
    return y.flatten(0, 1).flatten(1, 2)[:M, :K].to(torch.float8_e4m3fn), held


def _quantise(x, scale):
    codes, s = _encode(x, 1, scale)
    return codes, (s.t().contiguous() if scale == "f32" else s.view(torch.uint8).t().contiguous().view(torch.float8_e8m0fnu))


def _quantise_matrix(x, scale):
    return _encode(x, BLOCK, scale)


def _rows(case, st):
    return _quantise(st["x"].float(), case["scale"])


def _matrix(case, st):
    return _quantise_matrix(st["x"].float(), case["scale"])


def _swiglu(case, st):
    gate, up = st["x"].float().chunk(2, dim=1)
    return _quantise(gate / (1 + torch.exp(-gate)) * up, case["scale"])


def _rmsnorm(case, st):
    r, res = st["x"].float(), None
    if "res" in st:
        r = r + st["res"].float()
        res = r.to(st["res"].dtype)
    y = r * torch.rsqrt((r * r).mean(1, keepdim=True) + EPS) * st["gain"]
    return (*_quantise(y, case["scale"]), res, y.to(torch.bfloat16) if case["y"] else None)


def _matmul(case, st):
    M, N, K = case["M"], case["N"], case["K"]
    x = st["x"].float() * st["xs"].float().t().repeat_interleave(BLOCK, 1)[:, :K]
    w = st["w"].float() * st["ws"].float().repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]
    return torch.matmul(x, w.t()).to(TYPES[case["out"]])


# ---- the same in 64 bits ------------------------------------------------------------------------------


def _exact_scales(y, high, scale):
    """Scales of 64-bit values by their definition; None for powers of two, where a maximum next to a border decides."""
    if scale != "f32":
        return None
    out = torch.ones(-(-y.shape[0] // high), _blocks(y.shape[1]), dtype=torch.float64, device=DEV)
    for j in range(out.shape[1]):
        part = y[:, BLOCK * j:BLOCK * (j + 1)].abs().max(dim=1).values
        if high > 1:
            part = torch.stack([p.max() for p in part.split(high)])
        out[:, j] = torch.where(part == 0, 1.0, torch.maximum(part / TOP, torch.full_like(part, TINY)))
    return out


def exact(case, seed):
    """Which way a value next to a rounding border goes is not part of the definition: no 64-bit value for codes."""
    outs = _exact(case, prepare(case, seed))
    return None if isinstance(outs, tuple) and all(t is None for t in outs) else outs


def _exact(case, st):
    if case["op"] == "matmul":
        of = torch.arange(case["K"], device=DEV) // BLOCK
        x = st["x"].double() * st["xs"].double()[of].T
        w = st["w"].double() * st["ws"].double()[torch.arange(case["N"], device=DEV) // BLOCK][:, of]
        return x @ w.T.contiguous()
    x = st["x"].double()
    if case["op"] == "matrix":
        return None, _exact_scales(x, BLOCK, case["scale"])
    if case["op"] == "quantize":
        s = _exact_scales(x, 1, case["scale"])
        return None, None if s is None else s.T.contiguous()
    if case["op"] == "swiglu":
        y = x[:, :case["K"]] * torch.sigmoid(x[:, :case["K"]]) * x[:, case["K"]:]
        s = _exact_scales(y, 1, case["scale"])
        return None, None if s is None else s.T.contiguous()
    r = x + st["res"].double() if "res" in st else x
    y = r / torch.sqrt(torch.linalg.vecdot(r, r).unsqueeze(1) / case["K"] + EPS) * st["gain"].double()
    s = _exact_scales(y, 1, case["scale"])
    return None, None if s is None else s.T.contiguous(), r if "res" in st else None, y if case["y"] else None
