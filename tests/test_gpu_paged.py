"""GPU parity of the paged cache's operators (append, attention, read) with plain 64-bit forms.

Pools start as bytes of 0xff (NaN in bf16 and e4m3), so anything that leaks from a position that was not written shows."""
import math

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu

THETA = 1e6


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    assert sdd.device_ok(), "needs a gfx950 device"
    return sdd


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """A pool of NaN bytes, and sequences of given lengths whose pages are scattered over it."""

    def __init__(self, S, dtype, hkv, hd, page, room, spare=2):
        width = max(-(-n // page) for n in room)
        need = sum(-(-max(n, 0) // page) for n in room)
        self.S, self.dtype, self.hkv, self.hd, self.room = S, dtype, hkv, hd, room
        self.pool = S.PagePool(need + spare, hkv, hd, page, dtype)
        self.pool.buf.fill_(255)
        order = torch.randperm(need + spare, generator=torch.Generator().manual_seed(need + page)).tolist()
        rows = []
        for n in room:
            m = -(-max(n, 0) // page)
            rows.append(order[:m] + [-1] * (width - m))  # an id that must never be followed
            order = order[m:]
        self.table = i32(rows)

    def put(self, k, v, at, hq=None):
        """Rows k, v [B, R, hkv, hd] (bf16 values) as they are (no norm, no rotation); what the cache then stands for."""
        hq = self.hkv if hq is None else hq
        B, R = k.shape[:2]
        qkv = torch.cat([torch.zeros(B, R, hq * self.hd), k.flatten(2).float(), v.flatten(2).float()], 2)
        self.pool.append(qkv.to(torch.bfloat16).cuda(), hq, self.table, i32(at))
        if self.dtype == "bf16":
            return k.to(torch.bfloat16).double(), v.to(torch.bfloat16).double()
        return ref.to_e4m3(k.to(torch.bfloat16).double())[0], ref.to_e4m3(v.to(torch.bfloat16).double())[0]


# ---- append and read -----------------------------------------------------------------------------------

SHAPES = [  # query heads, KV heads, head_dim, page, rows, positions before them
    (64, 8, 128, 64, 1, [0, 63, 64, 1000]), (28, 4, 128, 32, 33, [0, 31, 500]), (4, 2, 64, 64, 9, [5, 0]),
    (3, 3, 64, 32, 7, [1, 25]), (8, 1, 128, 256, 300, [3]), (5, 5, 128, 128, 8, [0, 8, 16, 4]), (6, 2, 64, 1024, 17, [1019])]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("norm, rope", [(True, True), (False, False), (True, False), (False, True)])
@pytest.mark.parametrize("hq, hkv, hd, page, R, at", SHAPES)
def test_append_and_read(S, dtype, src, norm, rope, hq, hkv, hd, page, R, at):
    B = len(at)
    c = Cache(S, dtype, hkv, hd, page, [a + R for a in at])
    x = randn(hq + R, B, R, (hq + 2 * hkv) * hd) * torch.exp(randn(1, B, R, 1))
    x = x.to(torch.bfloat16 if src == "bf16" else torch.float32)
    gains = [(1 + 0.2 * randn(7 + i, hd)).float() for i in range(2)] if norm else [None, None]
    table = S.rope_table(max(at) + R, hd, THETA) if rope else None
    # rows at a stride of their own
    dev = torch.zeros(B, R, (hq + 2 * hkv) * hd + 64, dtype=x.dtype, device="cuda")[:, :, :(hq + 2 * hkv) * hd]
    dev.copy_(x)
    before = c.pool.buf.clone()
    err = i32([0])
    q = c.pool.append(dev, hq, c.table, i32(at), q_norm=None if gains[0] is None else gains[0].cuda(),
                      k_norm=None if gains[1] is None else gains[1].cuda(), rope=table, err=err)
    k, v = c.pool.read(c.table, i32(at), R, err=err)
    assert err.item() == 0
    heads = x.double().unflatten(2, (hq + 2 * hkv, hd))
    for b in range(B):
        pos = torch.arange(at[b], at[b] + R)
        th = THETA if rope else None
        # fp32 norm, table and rotation: a few roundings of values whose size is the pair's, not the element's
        want_q = ref.norm_rope(heads[b, :, :hq], gains[0], 1e-6, pos, th)
        want_k = ref.norm_rope(heads[b, :, hq:hq + hkv], gains[1], 1e-6, pos, th)
        for got, want, codes in ((q[b], want_q, False), (k[b], want_k, dtype == "e4m3")):
            pair = (want[..., :hd // 2] ** 2 + want[..., hd // 2:] ** 2).sqrt().repeat(1, 1, 2)
            fp32 = pair * 2.0 ** -24 * (hd / 16 + 16)
            if codes:
                _, e = ref.to_e4m3(want)
                # half a step of the code: 2^-4 of the value, or of the smallest normal code 2^-6; next to a border of the
                # row's exponent the code may be of the next one
                tol = (2.0 ** -4 * want.abs()).maximum(2.0 ** -10 * torch.pow(2.0, e.double() + 1)) * (1 + 2.0 ** -8) + fp32
            else:
                tol = ref.HALF[torch.bfloat16] * want.abs() * (1 + 2.0 ** -8) + fp32 + 1e-38
            off = (got.cpu().double() - want).abs()
            assert (off <= tol).all(), (b, (off / tol).max())
        want_v = heads[b, :, hq + hkv:]
        want_v = ref.to_e4m3(want_v)[0] if dtype == "e4m3" else want_v.to(torch.bfloat16).double()
        assert torch.equal(v[b].cpu().double(), want_v)
    # every byte that is not one of these rows' stays
    if max(at) > 0:
        n = min(a for a in at if a > 0)
        ks, vs = c.pool.read(c.table, i32([max(0, a - n) for a in at]), n)
        for b in range(B):
            if at[b] >= n:
                assert torch.isnan(ks[b].float()).all() and torch.isnan(vs[b].float()).all()
    changed = (c.pool.buf != before).sum().item()
    assert changed <= B * R * hkv * (2 * hd * (1 if dtype == "e4m3" else 2) + 2)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_rows_appended_one_by_one_equal_a_block(S, dtype):
    hq, hkv, hd, R = 8, 2, 128, 21
    x = randn(3, 2, R, (hq + 2 * hkv) * hd).to(torch.bfloat16).cuda()
    g = (1 + 0.1 * randn(4, hd)).float().cuda()
    rope = S.rope_table(200, hd, THETA)
    a, b = (Cache(S, dtype, hkv, hd, 32, [60, 90]) for _ in range(2))
    qa = a.pool.append(x, hq, a.table, i32([37, 5]), q_norm=g, k_norm=g, rope=rope)
    qb = [b.pool.append(x[:, r:r + 1], hq, b.table, i32([37 + r, 5 + r]), q_norm=g, k_norm=g, rope=rope) for r in range(R)]
    assert torch.equal(qa, torch.cat(qb, 1))
    assert torch.equal(a.pool.buf, b.pool.buf)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_rows_that_are_not_finite(S, dtype):
    """bf16 keeps them as they are; an 8-bit row that holds one reads as NaN; rows of zeros, of tiny and of huge values."""
    hkv, hd, R = 2, 64, 8
    k, v = randn(1, 1, R, hkv, hd).float(), randn(2, 1, R, hkv, hd).float()
    k[0, 1, 0, 5], k[0, 2, 1, 63], v[0, 3, 0, 0], v[0, 4, 1, 9] = math.inf, math.nan, -math.inf, math.nan
    k[0, 5], v[0, 5] = 0, 0
    k[0, 6] *= 1e-30
    v[0, 7] *= 1e35
    c = Cache(S, dtype, hkv, hd, 32, [40])
    wk, wv = c.put(k.double(), v.double(), [30])
    gk, gv = c.pool.read(c.table, i32([30]), R)
    for got, want in ((gk, wk), (gv, wv)):
        assert torch.equal(torch.nan_to_num(got.cpu().double(), nan=1e300, posinf=2e300, neginf=-2e300),
                           torch.nan_to_num(want, nan=1e300, posinf=2e300, neginf=-2e300))


def test_rotation_far_out(S):
    t = S.rope_table(1 << 20, 128, 1e4).cpu().double()
    for pos in (0, 1, 12345, 131071, (1 << 20) - 1):
        ang = pos * 1e4 ** (-torch.arange(0, 128, 2).double() / 128)
        # half a step of values up to 1, and the angle's own 64-bit rounding
        assert (t[pos] - torch.stack([ang.cos(), ang.sin()], 1)).abs().max() <= 2.0 ** -25 + pos * 2.0 ** -51


# ---- attention ----------------------------------------------------------------------------------------

ATTN = [  # query heads, KV heads, head_dim, page, rows, positions before them
    (8, 1, 128, 64, 1, [0]), (8, 1, 128, 64, 1, [1, 0, 31, 32, 33, 63, 64, 127, 128, 129]), (28, 4, 128, 32, 1, [511, 700]),
    (64, 8, 128, 128, 1, [255, 1300]), (4, 2, 64, 64, 9, [64, 0, 5]), (16, 2, 128, 64, 33, [0, 100, 260]),
    (7, 1, 128, 256, 33, [300]), (5, 5, 64, 32, 3, [40, 1]), (40, 1, 128, 32, 2, [77]), (3, 1, 64, 1024, 65, [1030]),
    (2, 1, 128, 32, 130, [0, 150]), (1, 1, 64, 32, 1, [9000])]


def check_attention(S, c, k, v, q, at, scale=None, out=None):
    hd = q.shape[3]
    got = c.pool.attention(q.cuda(), c.table, i32(at), scale=scale, out=out)
    for b in range(len(at)):
        want, tol = ref.attention(q[b].double(), k[b], v[b], at[b], hd ** -0.5 if scale is None else scale)
        off = (got[b].cpu().double() - want).abs()
        assert (off <= tol).all(), (b, (off / tol).max())
    return got


def fill(S, dtype, hkv, hd, page, R, at, seed=0, spread=1.0):
    c = Cache(S, dtype, hkv, hd, page, [a + R for a in at])
    k, v = [], []
    n = max(at) + R
    rk, rv = randn(seed + 1, len(at), n, hkv, hd) * spread, randn(seed + 2, len(at), n, hkv, hd)
    for b, a in enumerate(at):  # one sequence after the other (their lengths differ)
        one = [-1] * len(at)
        one[b] = 0
        m = a + R
        kk, vv = rk[:, :m], rv[:, :m]
        wk, wv = c.put(kk, vv, one)
        k.append(wk[b])
        v.append(wv[b])
    return c, k, v


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq, hkv, hd, page, R, at", ATTN)
def test_attention(S, dtype, hq, hkv, hd, page, R, at):
    c, k, v = fill(S, dtype, hkv, hd, page, R, at)
    q = (2 * randn(9, len(at), R, hq, hd)).to(torch.bfloat16)
    check_attention(S, c, k, v, q, at)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_peaked_and_flat(S, dtype):
    """Scores that leave one position all the weight, with the peak in a different chunk for each head; and equal scores."""
    hkv, hd, n = 2, 64, 700
    c, k, v = fill(S, dtype, hkv, hd, 32, 1, [n - 1], spread=8.0)
    q = (20 * randn(5, 1, 1, 4, hd)).to(torch.bfloat16)
    check_attention(S, c, k, v, q, [n - 1], scale=1.0)
    check_attention(S, c, k, v, q, [n - 1], scale=0.0)
    check_attention(S, c, k, v, q, [n - 1], scale=-0.5)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("where", ["k", "v", "both"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_stay_hidden(S, dtype, where, bad):
    """A row whose K or V is not finite reaches the rows that see it and no other, on the diagonal too."""
    hq, hkv, hd, R, at = 4, 2, 64, 20, 43
    c = Cache(S, dtype, hkv, hd, 32, [at + R])
    k, v = randn(1, 1, at + R, hkv, hd), randn(2, 1, at + R, hkv, hd)
    spoilt = at + 11
    if where != "v":
        k[0, spoilt, 0, 3] = bad
    if where != "k":
        v[0, spoilt, 0, 7] = bad
    k, v = c.put(k, v, [0])
    q = randn(3, 1, R, hq, hd).to(torch.bfloat16)
    got = c.pool.attention(q.cuda(), c.table, i32([at]))[0].cpu().double()
    want, tol = ref.attention(q[0].double(), k[0], v[0], at, hd ** -0.5)
    clean = torch.ones(R, hq, dtype=torch.bool)
    clean[11:, :2] = False  # the heads of KV head 0 that see it
    assert torch.isfinite(got[clean]).all()
    assert ((got - want).abs() <= tol)[clean].all()
    for r in range(11, R):
        for h in range(2):
            if where != "v" and math.isinf(bad) and dtype == "bf16":
                continue  # a weight of 0 or of everything, by the query's sign: any finite or NaN result is the softmax's
            dims = slice(7, 8) if where == "v" and dtype == "bf16" else slice(None)
            assert not torch.isfinite(got[r, h, dims]).any(), (r, h)
            if where == "v" and dtype == "bf16":
                rest = [d for d in range(hd) if d != 7]
                assert ((got[r, h] - want[r, h]).abs() <= tol[r, h])[rest].all()


def test_padded_long_and_broken_sequences(S):
    """Negative lengths, rows past the table or max_len, page ids out of range: left alone or masked, and reported."""
    hq, hkv, hd, page = 4, 2, 64, 32
    at = [40, -1, 63, 10, 33]
    c = Cache(S, "bf16", hkv, hd, page, [64] * 5)
    k, v = randn(1, 5, 64, hkv, hd), randn(2, 5, 64, hkv, hd)
    k, v = c.put(k, v, [0] * 5)
    n_pages = c.pool.desc.n_pages
    c.table[3, 0], c.table[4, 0] = n_pages, -5  # sequence 3 has no valid page, 4 only its second
    q = randn(3, 5, 2, hq, hd).to(torch.bfloat16)
    err, out = i32([0]), torch.full((5, 2, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    lens = i32(at)
    c.pool.attention(q.cuda(), c.table, lens, out=out, err=err)
    assert err.item() == 5
    o = out.cpu().double()
    want, tol = ref.attention(q[0].double(), k[0], v[0], 40, hd ** -0.5)
    assert ((o[0] - want).abs() <= tol).all()
    assert (o[1] == 7).all() and (o[2] == 7).all()  # padded, and 65 positions in a table of 64
    assert (o[3] == 0).all()
    want, tol = ref.attention(q[4].double(), k[4, 32:], v[4, 32:], 1, hd ** -0.5)
    assert ((o[4] - want).abs() <= tol).all()
    err.zero_()
    out.fill_(7.0)
    c.pool.attention(q.cuda(), c.table, lens, out=out, max_len=41, err=err)  # sequence 0 is one position too long now
    assert err.item() == 5 and (out[0] == 7).all()
    # append: nothing is written for any of them but sequence 0 and sequence 4's row in its second page
    before = c.pool.buf.clone()
    err.zero_()
    x = randn(5, 5, 2, (hq + 2 * hkv) * hd).to(torch.bfloat16).cuda()
    qo = torch.full((5, 2, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    c.pool.append(x, hq, c.table, i32([40, -1, 63, 10, 31]), q_out=qo, err=err)
    assert err.item() == 5
    assert (qo[1:3] == 7).all() and not (qo[0] == 7).all() and torch.equal(qo[3].flatten(1), x[3, :, :hq * hd])
    diff = (c.pool.buf != before).view(n_pages, -1).any(1).nonzero().flatten().tolist()
    assert sorted(diff) == sorted({c.table[0, 1].item(), c.table[4, 1].item()})
    # read
    err.zero_()
    kk, vv = (torch.full((5, 3, hkv, hd), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.pool.read(c.table, i32([3, -2, 62, 5, 31]), 3, out=(kk, vv), err=err)
    assert err.item() == 5 and (kk[1:3] == 7).all() and (kk[3] == 0).all() and (vv[3] == 0).all() and (kk[4, 0] == 0).all()
    assert torch.equal(kk[0].cpu().double(), k[0, 3:6]) and torch.equal(vv[4, 2].cpu().double(), v[4, 33])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("R", [1, 33])
def test_result_does_not_depend_on_the_batch(S, dtype, R):
    hq, hkv, hd, at = 16, 2, 128, [700, 3, 260, 0, 1000]
    c, k, v = fill(S, dtype, hkv, hd, 64, R, at)
    q = randn(4, 5, R, hq, hd).to(torch.bfloat16).cuda()
    both = c.pool.attention(q, c.table, i32(at))
    assert torch.equal(both, c.pool.attention(q, c.table, i32(at)))
    for b in range(5):
        one = c.pool.attention(q[b:b + 1], c.table[b:b + 1].contiguous(), i32(at[b:b + 1]), max_len=at[b] + R)
        assert torch.equal(one[0], both[b]), b


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_many_pages_in_one_chunk(S, dtype):
    """Rows so many that the sequence is not cut: more page ids than a wave holds at once."""
    hq, hkv, hd, R, at = 4, 2, 64, 2048, 1111
    c, k, v = fill(S, dtype, hkv, hd, 32, R, [at])
    q = randn(4, 1, R, hq, hd).to(torch.bfloat16)
    got = c.pool.attention(q.cuda(), c.table, i32([at]))[0].cpu().double()
    for r in (0, 1, 937, 2046, 2047):
        want, tol = ref.attention(q[0, r:r + 1].double(), k[0], v[0], at + r, hd ** -0.5)
        assert ((got[r:r + 1] - want).abs() <= tol).all(), r


@pytest.mark.parametrize("dtype, n_pages", [("bf16", 20000), ("e4m3", 40000)])
def test_pool_past_32_bits(S, dtype, n_pages):
    """Pages behind 4 GiB of others (5.2 GB pools)."""
    hq, hkv, hd, at, R = 16, 8, 128, 150, 5
    pool = S.PagePool(n_pages, hkv, hd, 64, dtype)
    assert pool.buf.numel() > 1 << 32
    c = Cache(S, dtype, hkv, hd, 64, [at + R])
    c.pool, c.table = pool, i32([[n_pages - 1, 0, n_pages - 7]])
    for p in c.table[0].tolist():
        pool.buf.view(n_pages, -1)[p].fill_(255)
    k, v = c.put(randn(1, 1, at + R, hkv, hd), randn(2, 1, at + R, hkv, hd), [0])
    q = randn(3, 1, R, hq, hd).to(torch.bfloat16)
    check_attention(S, c, k, v, q, [at])
    kk, vv = pool.read(c.table, i32([60]), 95)
    assert torch.equal(kk[0].cpu().double(), k[0, 60:155]) and torch.equal(vv[0].cpu().double(), v[0, 60:155])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_decode_loop_captured_and_replayed(S, dtype):
    """Append, attention and log probabilities as one captured graph, its lengths on the device: every replay is one token of
    each sequence, and equals the eager calls.  Two graphs share the workspaces; eager work runs between the replays."""
    hq, hkv, hd, V = 8, 2, 128, 1000
    at, steps = [126, 3, 250], 6
    a, b = (Cache(S, dtype, hkv, hd, 32, [n + steps for n in at]) for _ in range(2))
    room = max(at) + steps
    hist = randn(1, 3, max(at), hkv, hd), randn(2, 3, max(at), hkv, hd)
    for c in (a, b):
        for i, n in enumerate(at):
            c.put(hist[0][:, :n], hist[1][:, :n], [0 if j == i else -1 for j in range(3)])
    rope, g = S.rope_table(room, hd, THETA), torch.ones(hd, device="cuda")
    xs = randn(3, steps, 3, 1, (hq + 2 * hkv) * hd).to(torch.bfloat16).cuda()
    zs = randn(4, steps, 3, 1, V).float().cuda()
    tok = i32([[5], [999], [0]])
    ws, lws = a.pool.attention_workspace(3, 1, hq, room), S.logprobs_workspace(3, V, 4)

    def step(c, x, z, lens, stream=None):
        q = c.pool.append(x, hq, c.table, lens, q_norm=g, k_norm=g, rope=rope, stream=stream)
        o = c.pool.attention(q, c.table, lens, max_len=room, ws=ws, stream=stream)
        return (o, *S.token_logprobs(z, tok, 4, ws=lws, stream=stream))

    eager = []
    for i in range(steps):
        eager.append([t.clone() for t in step(b, xs[i], zs[i], i32([n + i for n in at]))])
    x, z, lens = xs[0].clone(), zs[0].clone(), i32([-1] * 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, x, z, lens)  # nothing is written: every sequence is padding
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs = step(a, x, z, lens)
        graphs.append((gr, outs))
    for i in range(steps):
        gr, outs = graphs[i % 2]
        x.copy_(xs[i])
        z.copy_(zs[i])
        lens.copy_(i32([n + i for n in at]))
        gr.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, eager[i]):
            assert torch.equal(got, want), i
        (xs[i].float() @ xs[i].float().transpose(1, 2)).sum()  # eager work of the program's own
    assert torch.equal(a.pool.buf, b.pool.buf)


def test_another_stream(S):
    hq, hkv, hd, at = 8, 2, 128, [300, 20]
    c, k, v = fill(S, "bf16", hkv, hd, 64, 1, at)
    q = randn(4, 2, 1, hq, hd).to(torch.bfloat16).cuda()
    want = c.pool.attention(q, c.table, i32(at))
    lens, ws, out = i32(at), c.pool.attention_workspace(2, 1, hq, 320), torch.empty_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.pool.attention(q, c.table, lens, max_len=320, ws=ws, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_shared_prefix_pages(S):
    """Two sequences over the same first pages, each with pages of its own behind them."""
    hq, hkv, hd, at = 4, 2, 64, 70
    c = Cache(S, "bf16", hkv, hd, 32, [96, 96])
    c.table[1, :2] = c.table[0, :2]
    pk, pv = randn(1, 2, 64, hkv, hd), randn(2, 2, 64, hkv, hd)
    pk[1], pv[1] = pk[0], pv[0]
    k0, v0 = c.put(pk, pv, [0, 0])
    k1, v1 = c.put(randn(3, 2, 7, hkv, hd), randn(4, 2, 7, hkv, hd), [64, 64])
    q = randn(5, 2, 1, hq, hd).to(torch.bfloat16)
    check_attention(S, c, torch.cat([k0, k1], 1), torch.cat([v0, v1], 1), q, [at, at])
