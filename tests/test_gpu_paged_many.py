"""Paged attention of calls with many query vectors (the kernel of 128 a workgroup), against plain 64-bit forms.

A call takes that kernel from B * n_kv_heads * ceil(R * n_q_heads / n_kv_heads / 128) = 160 on; each shape here is on that
side, which test_shapes_are_many states."""
import math

import pytest
import torch

import paged_ref as ref
from test_gpu_paged import Cache, S, check_attention, fill, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu

MANY = [  # query heads, KV heads, head_dim, page, rows, positions before them
    (64, 8, 128, 64, 33, [0, 1, 511, 512, 513, 1023, 1600]), (40, 40, 64, 32, 17, [0, 31, 700, 1500]),
    (28, 4, 128, 128, 65, [5, 63, 64, 0, 300, 447, 448, 449, 130, 1100]), (2, 2, 64, 1024, 130, [(37 * i) % 400 for i in range(40)]),
    (32, 32, 128, 32, 40, [96, 0, 2000, 33, 1])]


def vectors(hq, hkv, R, B):
    return B * hkv * -(-R * hq // hkv // 128)


def test_shapes_are_many():
    for hq, hkv, _, _, R, at in MANY:
        assert vectors(hq, hkv, R, len(at)) >= 160


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, page, R, at", MANY)
def test_attention(S, dtype, hq, hkv, hd, page, R, at):  # noqa: F811
    c, k, v = fill(S, dtype, hkv, hd, page, R, at)
    q = (2 * randn(9, len(at), R, hq, hd)).to(torch.bfloat16)
    check_attention(S, c, k, v, q, at)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_peaked_and_flat(S, dtype):  # noqa: F811
    """Scores far apart and rising along the sequence (the weights' reference has to move), equal scores, a negative scale."""
    hq, hkv, hd, R, at = 40, 40, 64, 17, [900, 3, 40, 200]
    c, k, v = fill(S, dtype, hkv, hd, 32, R, at, spread=6.0)
    q = (12 * randn(5, 4, R, hq, hd)).to(torch.bfloat16)
    for scale in (1.0, 0.0, -0.5):
        check_attention(S, c, k, v, q, at, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_a_prompt_that_is_not_cut(S, dtype):  # noqa: F811
    """One sequence, more page ids than a wave holds at once in its one chunk."""
    hq, hkv, hd, R, at = 16, 2, 64, 2560, 77
    assert vectors(hq, hkv, R, 1) >= 160
    c, k, v = fill(S, dtype, hkv, hd, 32, R, [at])
    q = randn(4, 1, R, hq, hd).to(torch.bfloat16)
    got = c.pool.attention(q.cuda(), c.table, i32([at]))[0].cpu().double()
    for r in (0, 1, 15, 16, 1499, 2047, 2559):
        want, tol = ref.attention(q[0, r:r + 1].double(), k[0], v[0], at + r, hd ** -0.5)
        assert ((got[r:r + 1] - want).abs() <= tol).all(), r


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("where", ["k", "v", "both"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("spoilt", [11, 0, 19])
def test_values_that_are_not_finite_stay_hidden(S, dtype, where, bad, spoilt):  # noqa: F811
    """A row whose K or V is not finite reaches the rows that see it and no other, neither of its sequence nor of another."""
    hq, hkv, hd, R, at = 80, 40, 64, 20, [43, 300, 12, 0]
    assert vectors(hq, hkv, R, 4) >= 160
    c = Cache(S, dtype, hkv, hd, 32, [a + R for a in at])
    k, v = randn(1, 4, max(at) + R, hkv, hd), randn(2, 4, max(at) + R, hkv, hd)
    if where != "v":
        k[1, at[1] + spoilt, 5, 3] = bad
    if where != "k":
        v[1, at[1] + spoilt, 5, 7] = bad
    wk, wv = [], []
    for b in range(4):
        one = [-1] * 4
        one[b] = 0
        kk, vv = c.put(k[:, :at[b] + R], v[:, :at[b] + R], one)
        wk.append(kk[b]), wv.append(vv[b])
    q = randn(3, 4, R, hq, hd).to(torch.bfloat16)
    got = c.pool.attention(q.cuda(), c.table, i32(at)).cpu().double()
    for b in range(4):
        want, tol = ref.attention(q[b].double(), wk[b], wv[b], at[b], hd ** -0.5)
        clean = torch.ones(R, hq, dtype=torch.bool)
        if b == 1:
            clean[spoilt:, 10:12] = False  # the heads of KV head 5 that see it
        assert torch.isfinite(got[b][clean]).all()
        assert ((got[b] - want).abs() <= tol)[clean].all()
    for r in range(spoilt, R):
        for h in (10, 11):
            if where != "v" and math.isinf(bad) and dtype == "bf16":
                continue  # a weight of 0 or of everything, by the query's sign: any finite or NaN result is the softmax's
            dims = slice(7, 8) if where == "v" and dtype == "bf16" else slice(None)
            assert not torch.isfinite(got[1, r, h, dims]).any(), (r, h)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_padded_long_and_broken_sequences(S, dtype):  # noqa: F811
    """Negative lengths, rows past the table or max_len, page ids out of range, among sequences that are in order."""
    hq, hkv, hd, R, B = 4, 2, 64, 33, 80
    assert vectors(hq, hkv, R, B) >= 160
    c = Cache(S, dtype, hkv, hd, 32, [160] * B)
    k, v = c.put(randn(1, B, 160, hkv, hd), randn(2, B, 160, hkv, hd), [0] * B)
    n_pages = c.pool.desc.n_pages
    at = [100] * B
    at[3], at[4], at[5] = -1, 128, -2 ** 31  # (128 + 33 positions in a table of 160)
    c.table[6, :], c.table[7, 1] = n_pages, 2 ** 31 - 1  # sequence 6 has no valid page, 7 not its second
    q = randn(3, B, R, hq, hd).to(torch.bfloat16)
    err, out = i32([0]), torch.full((B, R, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    c.pool.attention(q.cuda(), c.table, i32(at), out=out, err=err)
    assert err.item() == 5
    o = out.cpu().double()
    for b in range(B):
        if b in (3, 4, 5):
            assert (o[b] == 7).all()
        elif b == 6:
            assert (o[b] == 0).all()
        else:
            kk, vv, a = k[b], v[b], at[b]
            if b == 7:
                kk, vv, a = torch.cat([kk[:32], kk[64:]]), torch.cat([vv[:32], vv[64:]]), a - 32
            want, tol = ref.attention(q[b].double(), kk, vv, a, hd ** -0.5)
            assert ((o[b] - want).abs() <= tol).all(), b
    err.zero_()
    out.fill_(7.0)
    c.pool.attention(q.cuda(), c.table, i32(at), out=out, max_len=132, err=err)  # all are one position too long
    assert err.item() == 1 and (out == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_result_does_not_depend_on_the_others(S, dtype):  # noqa: F811
    """The same sequence among others of other lengths, in another place, under another max_len: the same bits."""
    hq, hkv, hd, R, at = 64, 8, 128, 33, [700, 3, 260, 0, 1900, 41, 513]
    c, k, v = fill(S, dtype, hkv, hd, 64, R, at)
    q = randn(4, 7, R, hq, hd).to(torch.bfloat16).cuda()
    both = c.pool.attention(q, c.table, i32(at))
    assert torch.equal(both, c.pool.attention(q, c.table, i32(at), max_len=1 << 15))
    turn = [4, 0, 6, 1, 2, 3, 5]
    other = c.pool.attention(q[turn].contiguous(), c.table[turn].contiguous(), i32([at[b] for b in turn]))
    for i, b in enumerate(turn):
        assert torch.equal(other[i], both[b]), b
    lens = [a if b in (2, 4) else -1 for b, a in enumerate(at)]
    some = c.pool.attention(q, c.table, i32(lens), out=torch.zeros_like(both))
    assert torch.equal(some[2], both[2]) and torch.equal(some[4], both[4]) and (some[0] == 0).all()


def test_captured_and_replayed(S):  # noqa: F811
    """One graph for all lengths up to max_len, its lengths on the device, the program's own work between the replays."""
    hq, hkv, hd, R, at = 64, 8, 128, 33, [0, 1, 511, 700, 513, 1023, 1600]
    c, k, v = fill(S, "bf16", hkv, hd, 64, R, at)
    q = randn(4, 7, R, hq, hd).to(torch.bfloat16).cuda()
    lens, out = i32(at), torch.zeros_like(q)
    ws = c.pool.attention_workspace(7, R, hq, 1633)
    c.pool.attention(q, c.table, lens, max_len=1633, ws=ws, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.pool.attention(q, c.table, lens, max_len=1633, ws=ws, out=out)
    for less in (0, 5, 0, 300):
        now = [max(a - less, 0) for a in at]
        lens.copy_(i32(now))
        out.zero_()
        g.replay()
        (q[0, 0].float() @ q[0, 0].float().T).sum()  # eager work of the program's own
        assert torch.equal(out, c.pool.attention(q, c.table, i32(now), max_len=1633)), less
        torch.cuda.synchronize()


def test_join_of_few_and_of_many_parts(S):  # noqa: F811
    """A decode step's parts are joined by one of two kernels, by what max_len allows: the same bits."""
    hq, hkv, hd, at = 8, 1, 128, [3000, 100, 700]
    c, k, v = fill(S, "bf16", hkv, hd, 64, 1, at)
    q = randn(4, 3, 1, hq, hd).to(torch.bfloat16).cuda()
    want = c.pool.attention(q, c.table, i32(at), max_len=3001)
    assert torch.equal(want, c.pool.attention(q, c.table, i32(at)))
    wide = torch.cat([c.table, torch.full((3, 1000), -1, dtype=torch.int32, device="cuda")], 1)
    assert torch.equal(want, c.pool.attention(q, wide, i32(at), max_len=60000))
    check_attention(S, c, k, v, q.cpu(), at)


def test_a_workspace_serves_smaller_calls(S):  # noqa: F811
    """The size for a call is enough for each with fewer sequences, rows or positions, whatever kernel that takes."""
    pool = S.PagePool(4, 8, 128, 64, "bf16")
    size = lambda B, R, n: pool.attention_workspace(B, R, 64, n).numel()
    for B, R, n in ((8, 65, 4096), (3, 97, 1000), (1, 1024, 2079), (64, 1, 4096)):
        most = size(B, R, n)
        for b in {1, 2, B // 2, B - 1, B} - {0}:
            for r in {1, 2, 16, 33, R // 2, R - 1, R} - {0}:
                for m in (1, 129, 257, 513, n // 2, n):
                    if b <= B and r <= R:
                        assert size(b, r, m) <= most, (B, R, n, b, r, m)


# ---- few rows, sequences that are cut --------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("R", [1, 33])
def test_peaks_in_different_parts(S, dtype, R):  # noqa: F811
    hq, hkv, hd, at = 8, 2, 64, [2500, 767, 768, 1600]
    c, k, v = fill(S, dtype, hkv, hd, 32, R, at, spread=8.0)
    q = (20 * randn(5, 4, R, hq, hd)).to(torch.bfloat16)
    for scale in (1.0, 0.0, -0.5):
        check_attention(S, c, k, v, q, at, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, R", [(16, 2, 1), (64, 8, 33)])
def test_lengths_around_the_cut(S, dtype, hq, hkv, R):  # noqa: F811
    at = [n - R for n in (255, 256, 257, 767, 768, 769, 1535, 1536, 1537, 2049)]
    for b in range(0, 10, 5):  # (five at a time: few workgroups)
        c, k, v = fill(S, dtype, hkv, 128, 64, R, at[b:b + 5])
        q = (2 * randn(9, 5, R, hq, 128)).to(torch.bfloat16)
        check_attention(S, c, k, v, q, at[b:b + 5])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("where", ["k", "v"])
def test_nan_in_one_part(S, dtype, where):  # noqa: F811
    """A NaN in a part that every row sees reaches all rows of its head, one on the diagonal those behind it."""
    hq, hkv, hd, R, at = 8, 2, 64, 3, 1500
    for spoilt, first in ((100, 0), (at + 1, 1)):
        c = Cache(S, dtype, hkv, hd, 32, [at + R])
        k, v = randn(1, 1, at + R, hkv, hd), randn(2, 1, at + R, hkv, hd)
        (k if where == "k" else v)[0, spoilt, 1, 5] = math.nan
        k, v = c.put(k, v, [0])
        q = randn(3, 1, R, hq, hd).to(torch.bfloat16)
        got = c.pool.attention(q.cuda(), c.table, i32([at]))[0].cpu().double()
        want, tol = ref.attention(q[0].double(), k[0], v[0], at, hd ** -0.5)
        clean = torch.ones(R, hq, dtype=torch.bool)
        clean[first:, 4:] = False
        assert ((got - want).abs() <= tol)[clean].all()
        dims = slice(5, 6) if where == "v" and dtype == "bf16" else slice(None)
        assert torch.isnan(got[first:, 4:, dims]).all()


# ---- streams and devices ---------------------------------------------------------------------------------


def test_tensors_made_on_another_stream_are_its_own(S):  # noqa: F811
    """Outputs and workspaces that calls on a busy stream make are not handed out again before that stream is done with them."""
    hq, hkv, hd, at = 8, 2, 128, [2000, 20]
    c, k, v = fill(S, "bf16", hkv, hd, 64, 1, at)
    q, lens = randn(4, 2, 1, hq, hd).to(torch.bfloat16).cuda(), i32(at)
    z, tok = randn(5, 2, 3, 5000).float().cuda(), i32([[1, 2, 3], [4, 5, 4999]])
    rows = randn(6, 2, 1, (hq + 2 * hkv) * hd).to(torch.bfloat16).cuda()
    want = (c.pool.attention(q, c.table, lens), *c.pool.read(c.table, i32([0, 0]), 20), *S.token_logprobs(z, tok, 5),
            S.rope_table(64, hd, 1e4))
    start, side, slow = i32([0, 0]), torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            slow = slow @ slow * 1e-3
    got = (c.pool.attention(q, c.table, lens, stream=side), *c.pool.read(c.table, start, 20, stream=side),
           *S.token_logprobs(z, tok, 5, stream=side), S.rope_table(64, hd, 1e4, stream=side))
    qo = c.pool.append(rows, hq, c.table, i32([-1, -1]), stream=side)
    junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1 << 12, 1 << 14, 1 << 16, 1 << 18, 1 << 20) for _ in range(4)]
    torch.cuda.synchronize()
    assert qo.shape == (2, 1, hq, hd) and len(junk) == 20
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_two_calls_at_once(S):  # noqa: F811
    """Calls on two streams over one pool, each with a workspace of its own."""
    hq, hkv, hd, R, at = 64, 8, 128, 33, [700, 3, 260, 0, 1900, 41, 513]
    c, k, v = fill(S, "bf16", hkv, hd, 64, R, at)
    q = randn(4, 7, R, hq, hd).to(torch.bfloat16).cuda()
    q1 = q[:, :1].contiguous()
    lens, many, one = i32(at), c.pool.attention(q, c.table, i32(at)), c.pool.attention(q1, c.table, i32(at))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [(c.pool.attention(q, c.table, lens, stream=a), c.pool.attention(q1, c.table, lens, stream=b)) for _ in range(8)]
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, many) and torch.equal(y, one)


def test_tensors_off_the_device_are_refused(S):  # noqa: F811
    c, k, v = fill(S, "bf16", 2, 64, 32, 1, [40])
    q = randn(4, 1, 1, 4, 64).to(torch.bfloat16)
    good, lens = q.cuda(), i32([40])
    for args in ((q, c.table, lens), (good, c.table.cpu(), lens), (good, c.table, lens.cpu())):
        with pytest.raises(ValueError, match="device"):
            c.pool.attention(*args)
    with pytest.raises(ValueError, match="device"):
        c.pool.attention(good, c.table, lens, out=torch.empty_like(q))
    with pytest.raises(ValueError, match="device"):
        c.pool.read(c.table.cpu(), i32([0]), 3)
    with pytest.raises(ValueError, match="device"):
        c.pool.append(torch.zeros(1, 1, 8 * 64, dtype=torch.bfloat16), 4, c.table, lens)
    with pytest.raises(ValueError, match="device"):
        S.token_logprobs(torch.zeros(1, 2, 8).cuda(), torch.zeros(1, 2, dtype=torch.int32))


# ---- long sequences of calls that both kernels take -------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, R, at", [(16, 2, 64, 200, [2359, 2360, 0, 2700]), (16, 2, 128, 65, [6078, 6079, 40]),
                                               (8, 1, 64, 64, [6080, 9000])])
def test_the_length_decides(S, dtype, hq, hkv, hd, R, at):  # noqa: F811
    """Sequences on both sides of the length from which the other kernel takes them, in one call: the values, and the bits of
    each alone and under another max_len."""
    assert vectors(hq, hkv, R, len(at)) < 160 and R * hq // hkv >= 512
    c, k, v = fill(S, dtype, hkv, hd, 64, R, at)
    q = randn(9, len(at), R, hq, hd).to(torch.bfloat16)
    got = check_attention(S, c, k, v, q, at)
    qd = q.cuda()
    for b, a in enumerate(at):
        for max_len in (a + R, 20000):
            table = torch.cat([c.table[b:b + 1], torch.full((1, 300), -1, dtype=torch.int32, device="cuda")], 1)
            one = c.pool.attention(qd[b:b + 1], table, i32([a]), max_len=max_len)
            assert torch.equal(one[0], got[b]), (b, max_len)
    # a padded one, and one without its first page, among them
    err, out = i32([0]), torch.full_like(qd, 7.0)
    c.table[-1, 0] = -1
    c.pool.attention(qd, c.table, i32([-1] + at[1:]), out=out, err=err)
    assert err.item() == 4 and (out[0] == 7).all() and torch.equal(out[1:-1], got[1:-1]) and not torch.equal(out[-1], got[-1])
