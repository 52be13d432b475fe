"""The matrix product in 8 bits against its 64-bit form."""
import pytest
import torch

import e4m3_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    return sdd


def gen(*seed):
    g = torch.Generator()
    g.manual_seed(sum(s * 7919 ** i for i, s in enumerate(seed)) & 0x7fffffff)
    return g


def check(S, M, N, K, scale, out, seed=0, wscale=None, where="cpu"):
    g = gen(M, N, K, seed)
    x, xs = (t.to(where) for t in R.random_codes(g, M, K, scale))
    w, ws = (t.to(where) for t in R.random_codes(g, N, K, wscale or scale, matrix=True))
    got = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).to(where)
    want, mag = R.matmul(x, xs, w, ws)
    tol = R.matmul_tol(want, mag, K, DT[out], R.group_max(x, xs, w, ws) if out == "bf16" and M > 16 else None)
    err = (got.double() - want).abs()
    assert got.shape == (M, N) and got.dtype == DT[out]
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 16), (1, 16, 128), (1, 300, 3584), (2, 17, 144), (9, 512, 256), (15, 15, 240), (16, 130, 1040), (17, 256, 688), (32, 33, 2064),
    (33, 512, 1296), (33, 1040, 256), (48, 100, 400), (49, 47, 128), (64, 257, 1152), (1, 20000, 64), (5, 16400, 272), (40, 33000, 64),
    (60, 20, 6000), (33, 600, 4240), (30, 9000, 272),
    (1, 5000, 8208), (4, 4200, 8464), (5, 300, 3584), (7, 33000, 272), (16, 600, 4240), (3, 33000, 400), (33, 32768, 144)])
def test_few_rows(S, M, N, K, scale, out):
    check(S, M, N, K, scale, out)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("M,N,K", [
    (65, 1, 16), (65, 128, 128), (66, 300, 1296), (100, 17, 2064), (127, 130, 144), (128, 256, 512), (129, 255, 640), (200, 513, 272),
    (257, 384, 1040), (264, 640, 1280), (511, 112, 2368), (600, 700, 64), (130, 20, 9008), (100, 33000, 144), (128, 33000, 400),
    (70, 32768, 272)])
def test_many_rows(S, M, N, K, scale, out):
    check(S, M, N, K, scale, out)


@pytest.mark.parametrize("scale,out", [("f32", "bf16"), ("e8m0", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("M,N,K", [(1500, 8200, 1168), (4100, 2100, 2064), (600, 33000, 144), (2048, 4096, 272), (511, 3600, 4752), (130, 33000, 48)])
def test_large(S, M, N, K, scale, out):
    """Sizes that take the large tiles (the reference in float64 on the GPU)."""
    check(S, M, N, K, scale, out, where="cuda")


@pytest.mark.parametrize("M", [5, 90])
@pytest.mark.parametrize("scale,wscale", [("f32", "e8m0"), ("e8m0", "f32")])
def test_two_kinds_of_scales(S, M, scale, wscale):
    check(S, M, 200, 400, scale, "bf16", wscale=wscale)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M", [3, 40, 70, 300])
def test_rows_of_out_lie_apart(S, M, out):
    """Stores of any alignment, and nothing between the rows or behind them."""
    g = gen(M, 1)
    x, xs = R.random_codes(g, M, 272, "f32")
    for N, stride, at in ((130, 133, 1), (130, 136, 0), (129, 129, 3), (64, 200, 4)):
        w, ws = R.random_codes(g, N, 272, "f32", matrix=True)
        flat = torch.full((M * stride + 64,), 7.5, dtype=DT[out], device="cuda")
        view = flat[at:at + M * stride].view(M, stride)[:, :N]
        m = S.E4M3Matrix(w.cuda(), ws.cuda())
        assert m.matmul(x.cuda(), xs.cuda(), out=view) is view
        assert torch.equal(view, m.matmul(x.cuda(), xs.cuda(), dtype=DT[out]))
        mask = torch.ones_like(flat, dtype=torch.bool)
        mask[at:at + M * stride].view(M, stride)[:, :N] = False
        assert (flat[mask] == 7.5).all()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M", [4, 33, 70, 140])
def test_what_a_value_that_is_no_number_reaches(S, M, out):
    """NaN codes or scales of a row reach that row, those of the matrix their columns (a scale: of its block), nothing else."""
    g = gen(M, 2)
    N, K = 260, 400
    x, xs = R.random_codes(g, M, K, "f32")
    w, ws = R.random_codes(g, N, K, "f32", matrix=True)
    want = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
    x.view(torch.uint8)[1, 5], x.view(torch.uint8)[3, 399] = 0x7f, 0xff
    xs[2, 2] = float("nan")
    w.view(torch.uint8)[7, 300], w.view(torch.uint8)[259, 0] = 0xff, 0x7f
    ws[1, 3] = float("nan")
    got = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[1:4] = True
    bad[:, 7], bad[:, 259], bad[:, 128:256] = True, True, True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M", [2, 40, 80, 200])
def test_zero_and_extreme_scales(S, M, out):
    g = gen(M, 3)
    x, xs = R.random_codes(g, M, 256, "f32")
    w, ws = R.random_codes(g, 40, 256, "f32", matrix=True)
    xs[:, 0] = 0
    xs[:, 1] = 2.0 ** -100
    got = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
    want, mag = R.matmul(x, xs, w, ws)
    tol = R.matmul_tol(want, mag, 256, DT[out], R.group_max(x, xs, w, ws) if out == "bf16" else None)
    assert (got[0] == 0).all() and ((got.double() - want).abs() <= tol).all()
    # powers of two on both sides: the smallest byte, large ones, and the byte that is no number
    w, ws = R.random_codes(g, 200, 256, "e8m0", matrix=True)
    b = torch.full((2, M), 127, dtype=torch.uint8)
    b[:, 0], b[0, 1] = 0, 255
    if M > 2:
        b[:, 2] = 200
    xs = b.view(torch.float8_e8m0fnu)
    got = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
    assert torch.isnan(got[1]).all()
    keep = torch.tensor([m for m in range(M) if m != 1])
    xk, sk = x.view(torch.uint8)[keep].view(torch.float8_e4m3fn), b[:, keep].contiguous().view(torch.float8_e8m0fnu)
    want, mag = R.matmul(xk, sk, w, ws)
    tol = R.matmul_tol(want, mag, 256, DT[out], R.group_max(xk, sk, w, ws) if out == "bf16" else None)
    # (2^-149: results among the smallest numbers)
    assert ((got[keep].double() - want).abs() <= tol + 2.0 ** -133).all()
    wb = ws.view(torch.uint8).clone()
    wb[1, 1] = 255
    got2 = S.E4M3Matrix(w.cuda(), wb.view(torch.float8_e8m0fnu).cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
    assert torch.isnan(got2[:, 128:]).all() and torch.equal(got2[keep][:, :128], got[keep][:, :128])


@pytest.mark.parametrize("M", [1, 33, 64, 65, 264])
def test_same_bits_again_and_in_a_graph(S, M):
    g = gen(M, 4)
    x, xs = R.random_codes(g, M, 1296, "f32")
    w, ws = R.random_codes(g, 700, 1296, "f32", matrix=True)
    m = S.E4M3Matrix(w.cuda(), ws.cuda())
    x, xs, room = x.cuda(), xs.cuda(), m.workspace(M)
    room.fill_(0xff)  # (what a workspace holds before a call does not matter)
    want = m.matmul(x, xs, ws=room).clone()
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.matmul(x, xs, out=out, ws=room)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(m.matmul(x, xs, ws=room), want)
    x2 = torch.roll(x.view(torch.uint8), 1, 0).view(torch.float8_e4m3fn)
    x.view(torch.uint8).copy_(x2.view(torch.uint8))
    graph.replay()
    assert torch.equal(out, m.matmul(x, xs))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("few,more", [(1, 4), (5, 16), (17, 32), (40, 48), (49, 64), (65, 128), (130, 256), (300, 384)])
def test_bits_do_not_depend_on_the_rows_beside(S, few, more, out):
    g = gen(few, more)
    x, xs = R.random_codes(g, more, 1296, "f32")
    w, ws = R.random_codes(g, 700, 1296, "f32", matrix=True)
    m = S.E4M3Matrix(w.cuda(), ws.cuda())
    want = m.matmul(x.cuda(), xs.cuda(), dtype=DT[out])
    got = m.matmul(x[more - few:].cuda(), xs[:, more - few:].contiguous().cuda(), dtype=DT[out])
    assert torch.equal(got, want[more - few:])


def test_workspace_serves_fewer_rows(S):
    g = gen(5)
    w, ws = R.random_codes(g, 500, 2064, "f32", matrix=True)
    m = S.E4M3Matrix(w.cuda(), ws.cuda())
    room = m.workspace(600)
    for M in (1, 4, 5, 16, 33, 64, 65, 100, 128, 129, 200, 256, 300, 511, 600):  # (cut into other parts)
        x, xs = (t.cuda() for t in R.random_codes(g, M, 2064, "f32"))
        assert torch.equal(m.matmul(x, xs, ws=room), m.matmul(x, xs))


def test_on_another_stream(S):
    g = gen(6)
    x, xs = (t.cuda() for t in R.random_codes(g, 130, 528, "f32"))
    w, ws = (t.cuda() for t in R.random_codes(g, 300, 528, "f32", matrix=True))
    want = S.E4M3Matrix(w, ws).matmul(x, xs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m = S.E4M3Matrix(w, ws, stream=side)
    got = m.matmul(x, xs, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_matrix_keeps_nothing_of_its_inputs(S):
    g = gen(7)
    x, xs = (t.cuda() for t in R.random_codes(g, 20, 144, "e8m0"))
    w, ws = (t.cuda() for t in R.random_codes(g, 90, 144, "e8m0", matrix=True))
    m = S.E4M3Matrix(w, ws)
    want = m.matmul(x, xs)
    w.view(torch.uint8).fill_(0x7f)
    ws.view(torch.uint8).fill_(0xff)
    assert torch.equal(m.matmul(x, xs), want)
