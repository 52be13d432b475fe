"""Paged attention over values that are not finite, in sequences long enough that the cost shows: what one bad value may cost,
and that it reaches the rows that see it and no other."""
import math

import pytest
import torch

import paged_ref as ref
from test_gpu_paged import Cache, S, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu


def filled(S, dtype, hkv, hd, page, n, seed=1):  # noqa: F811
    """A cache of one sequence of n positions, its values made on the device; and what it stands for, on the CPU."""
    c = Cache(S, dtype, hkv, hd, page, [n])
    g = torch.Generator(device="cuda").manual_seed(seed)
    kv = torch.randn(1, n, 2 * hkv * hd, generator=g, device="cuda").to(torch.bfloat16)
    return c, kv


def put(c, kv):
    n = kv.shape[1]
    c.pool.append(torch.cat([torch.zeros_like(kv[:, :, :c.hkv * c.hd]), kv], 2), c.hkv, c.table, i32([0]))
    k, v = c.pool.read(c.table, i32([0]), n)
    return k[0].cpu().double(), v[0].cpu().double()


def microseconds(f, n=3):
    f()
    best = 1e30
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3)
    return best


LONG = [  # query heads, KV heads, head_dim, rows, positions before them: many query vectors, the sequence in one part
    (64, 8, 128, 1024, 3000), (16, 16, 64, 2048, 2500)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, R, at", LONG)
@pytest.mark.parametrize("side, where", [("v", "last"), ("v", "first"), ("k", "last"), ("v", "middle")])
def test_one_bad_value_costs_little(S, dtype, hq, hkv, hd, R, at, side, where):  # noqa: F811
    """The call with a NaN in one row of every KV head's K or V, seen by all rows or hidden from most, takes at most four times
    the call without (the rows that share products with it are at most those of one 32-vector tile)."""
    c, kv = filled(S, dtype, hkv, hd, 64, at + R)
    put(c, kv)
    q = randn(3, 1, R, hq, hd).to(torch.bfloat16).cuda()
    lens, out = i32([at]), torch.empty_like(q)
    ws = c.pool.attention_workspace(1, R, hq, at + R)
    call = lambda: c.pool.attention(q, c.table, lens, max_len=at + R, out=out, ws=ws)  # noqa: E731
    clean = microseconds(call)
    pos = {"last": at + R - 1, "first": 0, "middle": at + R // 2 + 1}[where]
    rows = kv[0, pos].view(2, hkv, hd)
    rows[0 if side == "k" else 1, :, 3] = math.nan
    put(c, kv)
    spoilt = microseconds(call)
    assert spoilt <= 4 * clean, (clean, spoilt)
    sees = torch.arange(at, at + R) >= pos
    o = out[0].cpu()
    assert torch.isfinite(o[~sees].float()).all()
    if sees.any():
        dims = slice(3, 4) if side == "v" and dtype == "bf16" else slice(None)
        assert torch.isnan(o[sees][..., dims]).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, R, at", LONG)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bad_value_on_the_diagonal_of_a_long_part(S, dtype, hq, hkv, hd, R, at, bad):  # noqa: F811
    c, kv = filled(S, dtype, hkv, hd, 64, at + R, seed=2)
    r0 = R // 2 + 5
    kv[0, at + r0].view(2, hkv, hd)[1, 2, 7] = bad
    k, v = put(c, kv)
    q = randn(4, 1, R, hq, hd).to(torch.bfloat16)
    got = c.pool.attention(q.cuda(), c.table, i32([at]))[0].cpu().double()
    grp = hq // hkv
    for r in (0, 1, r0 - 33, r0 - 2, r0 - 1, r0, r0 + 1, r0 + 40, R - 1):
        want, tol = ref.attention(q[0, r:r + 1].double(), k, v, at + r, hd ** -0.5)
        off, w, t = (got[r:r + 1] - want).abs()[0], want[0], tol[0]
        ok = torch.ones(hq, hd, dtype=torch.bool)
        if r >= r0:
            heads = slice(2 * grp, 3 * grp)
            dims = slice(None) if dtype == "e4m3" else slice(7, 8)
            ok[heads, dims] = False
            assert not torch.isfinite(got[r, heads, dims]).any(), r
        assert torch.isfinite(w[ok]).all() and (off <= t)[ok].all(), r


FEW = [(64, 8, 128, 33, 1000), (64, 8, 128, 60, 6000), (28, 4, 128, 200, 2200), (8, 8, 64, 17, 500), (28, 4, 128, 1, 700)]  # (as above)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, R, at", FEW)
@pytest.mark.parametrize("side, where", [("v", "last"), ("v", "first"), ("k", "last")])
def test_one_bad_value_costs_little_among_few_rows(S, dtype, hq, hkv, hd, R, at, side, where):  # noqa: F811
    """The same where the sequence's steps are shared out over waves and workgroups: two and a half times at most."""
    c, kv = filled(S, dtype, hkv, hd, 64, at + R)
    put(c, kv)
    q = randn(3, 1, R, hq, hd).to(torch.bfloat16).cuda()
    lens, out = i32([at]), torch.empty_like(q)
    ws = c.pool.attention_workspace(1, R, hq, at + R)
    call = lambda: c.pool.attention(q, c.table, lens, max_len=at + R, out=out, ws=ws)  # noqa: E731
    clean = microseconds(call, 10)
    kv[0, at + R - 1 if where == "last" else 0].view(2, hkv, hd)[0 if side == "k" else 1, :, 3] = math.nan
    put(c, kv)
    spoilt = microseconds(call, 10)
    assert spoilt <= 2.5 * clean, (clean, spoilt)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, R, at", FEW)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", [0, 0.5, 1])
def test_a_bad_value_among_few_rows(S, dtype, hq, hkv, hd, R, at, bad, where):  # noqa: F811
    c, kv = filled(S, dtype, hkv, hd, 32, at + R, seed=3)
    r0 = round(where * (R - 1))
    h0, d0 = hkv - 1, hd - 5
    kv[0, at + r0].view(2, hkv, hd)[1, h0, d0] = bad
    k, v = put(c, kv)
    q = randn(4, 1, R, hq, hd).to(torch.bfloat16)
    got = c.pool.attention(q.cuda(), c.table, i32([at]))[0].cpu().double()
    grp = hq // hkv
    for r in sorted({0, 1, r0 - 1, r0, r0 + 1, R - 1} & set(range(R))):
        want, tol = ref.attention(q[0, r:r + 1].double(), k, v, at + r, hd ** -0.5)
        off = (got[r:r + 1] - want).abs()[0]
        ok = torch.ones(hq, hd, dtype=torch.bool)
        if r >= r0:
            heads = slice(h0 * grp, (h0 + 1) * grp)
            dims = slice(None) if dtype == "e4m3" else slice(d0, d0 + 1)
            ok[heads, dims] = False
            if dtype == "e4m3" or math.isnan(bad):
                assert torch.isnan(got[r, heads, dims]).all(), r
            else:  # (its weight is positive)
                assert (got[r, heads, dims] == bad).all(), r
        assert (off <= tol[0])[ok].all(), r


@pytest.mark.parametrize("hq, hkv, B, R", [(16, 8, 1, 1), (16, 8, 1, 33), (16, 8, 1, 1400), (80, 40, 4, 20)])
def test_scores_past_the_range(S, hq, hkv, B, R):  # noqa: F811
    """A score that passes fp32's range is no weight of 0: the row's result is the softmax's (that position alone) or NaN."""
    hd, at = 64, 40
    c = Cache(S, "bf16", hkv, hd, 32, [at + R] * B)
    k, v = torch.zeros(B, at + R, hkv, hd, dtype=torch.float64), randn(2, 1, at + R, hkv, hd).repeat(B, 1, 1, 1)
    k[:, 7, :, 0] = 2e19
    k, v = c.put(k, v, [0] * B)
    q = torch.zeros(B, R, hq, hd, dtype=torch.bfloat16)
    q[..., 0] = 1.6e19  # 3.2e38, and more than fp32 holds once log2 e is in it
    got = c.pool.attention(q.cuda(), c.table, i32([at] * B), scale=1.0).cpu().double()
    want = v[0, 7].repeat_interleave(hq // hkv, 0).expand(B, R, hq, hd)
    assert (torch.isnan(got) | ((got - want).abs() <= 2.0 ** -8 * want.abs())).all()
