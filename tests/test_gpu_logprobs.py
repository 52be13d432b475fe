"""GPU parity of sdd_token_logprobs with the plain form in 64 bits: values to the fp32 sums' rounding, tokens exactly."""
import math

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    assert sdd.device_ok(), "needs a gfx950 device"
    return sdd


def gen(seed):
    return torch.Generator().manual_seed(seed)


def check(S, z, tokens, n, ws=None):
    """z [B, R, V] on the CPU (any strides the binding takes)."""
    B, R, V = z.shape
    dev = torch.empty_strided(z.shape, z.stride(), dtype=z.dtype, device="cuda")
    dev.copy_(z)
    out = S.token_logprobs(dev, tokens.cuda(), n, ws=ws)
    lp, H = out[0].cpu(), out[1].cpu()
    for b in range(B):
        for r in range(R):
            wlp, wH, ids, top, tol = ref.logprobs(z[b, r], int(tokens[b, r]), n)
            ctx = (b, r, V, n)
            for got, want in [(float(lp[b, r]), wlp), (float(H[b, r]), wH)] + (
                    list(zip(out[3][b, r].tolist(), top)) if n else []):
                if math.isinf(want) or math.isnan(want):
                    assert got == want or (math.isnan(got) and math.isnan(want)), ctx
                else:
                    assert abs(got - want) <= tol + 2.0 ** -23 * abs(want), (ctx, got, want, tol)
            if n:
                assert out[2][b, r].tolist() == ids, ctx
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V, n", [(1, 0), (1, 1), (1, 5), (2, 1), (3, 32), (7, 7), (8, 4), (9, 32), (63, 1), (64, 32), (65, 20), (300, 32),
                                  (1000, 5), (2047, 32), (4097, 20), (20011, 32), (151936, 20), (152064, 0)])
def test_vocabularies(S, dtype, V, n):
    B, R = (2, 3) if V < 10000 else (1, 2)
    z = (4 * torch.randn(B, R, V, generator=gen(V + n))).to(dtype)
    tokens = torch.randint(0, V, (B, R), generator=gen(1)).int()
    check(S, z, tokens, n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 5, 32])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two", "steps", "zeros"])
def test_orders_and_ties(S, dtype, n, order):
    """Rows that pass every threshold, and rows of equal logits (the lowest indices win; -0 equals 0)."""
    V = 9001
    i = torch.arange(V, dtype=torch.float32)
    z = {"rising": i / 64, "falling": -i / 64, "equal": torch.full((V,), 2.5), "two": (i % 2), "steps": (i / 1000).floor(),
         "zeros": torch.where(i % 3 == 0, 0.0, -0.0)}[order].to(dtype).view(1, 1, V).repeat(1, 2, 1)
    check(S, z, torch.tensor([[0, V - 1]], dtype=torch.int32), n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 5003])
def test_masks(S, dtype, V):
    """-inf and the type's lowest value over most, all but one and all of a row; tokens inside and outside the mask."""
    low = torch.finfo(dtype).min
    z = torch.randn(8, 1, V, generator=gen(3))
    keep = torch.rand(V, generator=gen(4)) < 0.2
    keep[17] = True
    z[0, 0, ~keep] = -math.inf
    z[1, 0, :] = -math.inf
    z[1, 0, 17] = 3.0
    z[2, 0, ~keep] = low
    z[3, 0, :] = low
    z[4, 0, :] = low
    z[4, 0, 17] = 1.0
    z[5, 0, :20] = -math.inf
    z[6, 0, 20:] = -math.inf
    z[7, 0, :] *= 1e30
    z = z.to(dtype)
    for t in (17, int((~keep).nonzero()[0])):
        check(S, z, torch.full((8, 1), t, dtype=torch.int32), 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [33, 70001])
def test_rows_without_a_distribution(S, dtype, V):
    z = torch.randn(1, 6, V, generator=gen(5)).to(dtype)
    z[0, 0, V // 2] = math.nan
    z[0, 1, V - 1] = math.inf
    z[0, 2, :] = -math.inf
    z[0, 3, 0], z[0, 3, 1] = math.nan, math.inf
    z[0, 4, :] = math.nan
    lp, H, top, tlp = S.token_logprobs(z.cuda(), torch.zeros(1, 6, dtype=torch.int32, device="cuda"), 8)
    assert torch.isnan(lp[0, :5]).all() and torch.isnan(H[0, :5]).all() and (top[0, :5] == -1).all() and torch.isnan(tlp[0, :5]).all()
    check(S, z[:, 5:].contiguous(), torch.zeros(1, 1, dtype=torch.int32), 8)


def test_tokens_out_of_range_and_optional_outputs(S):
    z = torch.randn(1, 3, 500, generator=gen(6))
    tokens = torch.tensor([[-1, 500, 7]], dtype=torch.int32)
    full = check(S, z, tokens, 3)
    lp, H, top, tlp = S.token_logprobs(z.cuda(), None, 3)
    assert lp is None and torch.equal(H, full[1]) and torch.equal(top, full[2]) and torch.equal(tlp, full[3])
    lp, H = S.token_logprobs(z.cuda(), tokens.cuda())
    assert torch.equal(lp[0, 2], full[0][0, 2]) and torch.isnan(lp[0, :2]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V, off", [(1001, 1), (1000, 3), (517, 5), (64, 0)])
def test_strides_and_alignment(S, dtype, V, off):
    """Rows that begin anywhere, sequences further apart than their rows; what lies outside a row is NaN."""
    B, R = 3, 2
    buf = torch.full((off + B * (R * V + 13),), math.nan, dtype=dtype)
    z = torch.as_strided(buf, (B, R, V), (R * V + 13, V, 1), off)
    z.copy_(torch.randn(B, R, V, generator=gen(V)).to(dtype))
    dev = torch.as_strided(buf.cuda(), (B, R, V), (R * V + 13, V, 1), off)
    tokens = torch.full((B, R), V - 1, dtype=torch.int32)
    got = S.token_logprobs(dev, tokens.cuda(), 6)
    want = S.token_logprobs(z.contiguous().cuda(), tokens.cuda(), 6)
    assert torch.equal(got[2], want[2])
    check(S, z.contiguous(), tokens, 6)
    for i in (0, 1, 3):  # (vectors begin elsewhere in the row: the sums' order differs)
        assert (got[i] - want[i]).abs().max() <= 2.0 ** -19


def test_one_workspace_for_calls_of_any_shape(S):
    ws = S.logprobs_workspace(1100, 152064, 32)
    cases = [(1, 1, 152064, 32), (4, 33, 5000, 3), (1, 1100, 700, 0), (2, 2, 60000, 20), (1, 1, 152064, 5), (16, 64, 9000, 32)]
    for B, R, V, n in cases * 2:
        z = torch.randn(B, R, V, generator=gen(V))
        tok = torch.randint(0, V, (B, R), generator=gen(2)).int()
        got = S.token_logprobs(z.cuda(), tok.cuda(), n, ws=ws)
        want = S.token_logprobs(z.cuda(), tok.cuda(), n)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (B, R, V, n)
    check(S, torch.randn(1, 1, 152064, generator=gen(9)), torch.tensor([[3]], dtype=torch.int32), 32, ws=ws)


def test_verified_block_reports_what_it_committed(S):
    """With acceptance: the greedy token of every row is its best alternative, and its log probability the maximum's."""
    B, gamma, V = 3, 4, 6000
    p = torch.randn(B, gamma + 1, V, generator=gen(8)).cuda()
    draft = p[:, :gamma].argmax(-1).int()
    draft[1, 2] = 5
    L, nxt, _ = S.accept(draft, p, S.GREEDY)
    tok = torch.cat([draft, torch.zeros(B, 1, dtype=torch.int32, device="cuda")], 1)
    tok.scatter_(1, L.long().unsqueeze(1), nxt.unsqueeze(1))
    lp, _, top, tlp = S.token_logprobs(p, tok, 2)
    for b in range(B):
        n = int(L[b]) + 1
        assert torch.equal(top[b, :n, 0], tok[b, :n]) and torch.equal(lp[b, :n], tlp[b, :n, 0])
