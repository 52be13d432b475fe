"""How exact the 8-bit product's sums are: in fp32 for up to 16 rows and for fp32 results; for bf16 results of more rows the bound of
the matrix cores' cut, result by result and as a whole."""
import pytest
import torch

import e4m3_ref as R
import test_gpu_e4m3_layer as L

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    return sdd


def ones(rows, K, matrix=False, scale="f32"):
    shape = (R.blocks(rows), R.blocks(K)) if matrix else (R.blocks(K), rows)
    return torch.ones(shape) if scale == "f32" else torch.full(shape, 127, dtype=torch.uint8).view(torch.float8_e8m0fnu)


def product(S, x, w, out, scale="f32"):
    """Codes with scales of 1."""
    m = S.E4M3Matrix(w.cuda(), ones(*w.shape, matrix=True, scale=scale).cuda())
    return m.matmul(x.cuda(), ones(*x.shape, scale=scale).cuda(), dtype=DT[out]).cpu().double()


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(1, 20), (4, 300), (4, 9000), (3, 6000), (5, 300), (16, 33000), (17, 300), (64, 300), (100, 33000), (130, 300),
                                 (300, 2100)])
def test_small_products_beside_large_ones_that_cancel(S, M, N, out, scale):
    """Two groups of 8 columns with 448 x 448 and -448 x 448 and seven products of 1 each: 14, where sums are fp32's."""
    K = 144
    x, w = torch.zeros(M, K), torch.zeros(N, K)
    x[:, :16], w[:, :16] = 1, 1
    x[:, 0], x[:, 8], w[:, 0], w[:, 8] = 448, -448, 448, 448
    x, w = x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn)
    got = product(S, x, w, out, scale)
    if M <= 16 or out == "f32":
        assert (got == 14).all()
    else:  # 7 * 2^-13 of 448^2, twice
        assert ((got - 14).abs() <= 2 * 7 * 2.0 ** -13 * 448 ** 2).all()


def cancelling(M, N, K, seed):
    """Codes of rows with loud channels and of a matrix, K columns, and behind them the same columns in another order with the
    matrix's signs turned: every result is 0 exactly, what comes out is the sums' error and no rounding of a result hides it."""
    g = torch.Generator()
    g.manual_seed(seed)
    x = R.random_rows(g, M, K)
    x = (x * 448 / x.abs().amax(1, keepdim=True)).to(torch.float8_e4m3fn).float()
    w = (torch.randn(N, K, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).float()
    p = torch.randperm(K, generator=g)
    f8 = lambda t: t.to(torch.float8_e4m3fn)  # noqa: E731
    return f8(torch.cat([x, x[:, p]], 1)), f8(torch.cat([w, -w[:, p]], 1))


def exponent(v):
    """Of codes as values, -6 for the subnormal ones."""
    return (torch.frexp(v.abs())[1] - 1).clamp(min=-6)


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(4, 96, 2560), (16, 96, 12800), (33, 96, 2560), (33, 48, 12800), (64, 64, 9472), (130, 96, 12800), (264, 272, 2560)])
def test_error_as_a_whole(S, M, N, K, out, scale):
    """The mean square of the error over all results.

    Signs are random, so that the errors of a sum's parts add up as squares.  Of bf16 results of more than 16 rows each product p
    loses its bits below u = 2^(E - 13), E the largest sum of two codes' exponents among the eight products of its group: (|p| mod u)^2;
    a quarter more for a mean over 1500 results and more (a standard deviation of their squares is the mean times 1.5, of the mean of
    1500 4%).  Each of the at most K / 4 + K / 64 + 1 additions of groups, blocks and parts is off by a step, 2^-23 of a partial
    sum, whose mean square is no larger than the sum of the products' squares.  (fp32 results and fewer rows: 384 results and more, a
    deviation of 8%, against a bound of a whole step each time.)"""
    x, w = cancelling(M, N, K, M + N + K)
    assert ((x.double() @ w.double().t()) == 0).all()
    got = product(S, x, w, out, scale)
    a, b = x.double().cuda(), w.double().cuda()
    ea, eb = exponent(a), exponent(b)
    squares = float(((a * a) @ (b * b).t().contiguous()).mean())
    cut = 0.0
    if out == "bf16" and M > 16:
        lost = torch.zeros(M, N, dtype=torch.float64, device="cuda")
        for k in range(0, 2 * K, 8):
            p = (a[:, None, k:k + 8] * b[None, :, k:k + 8]).abs()
            e = torch.where(p > 0, ea[:, None, k:k + 8] + eb[None, :, k:k + 8], -100).amax(2, keepdim=True)
            lost += (torch.remainder(p, torch.ldexp(torch.ones_like(p[:, :, :1]), e - 13)) ** 2).sum(2)
        cut = 1.25 * float(lost.mean())
    bound = cut + (2 * K / 8 + 2 * K / 128 + 1) * 2.0 ** -46 * squares
    error = float((got ** 2).mean())
    print(f"error {(error / squares) ** 0.5:.2e} of such sums, both as root mean squares; bound {(bound / squares) ** 0.5:.2e}")
    assert error <= bound


@pytest.mark.parametrize("wscale", ["f32", "e8m0"])
@pytest.mark.parametrize("M", [1, 2, 4, 5, 16])
def test_few_rows_with_far_scales(S, M, wscale):
    """bf16 results of up to 16 rows have fp32's sums with scales of any size too."""
    g = torch.Generator()
    g.manual_seed(M)
    x, _ = R.random_codes(g, M, 256, "f32")
    w, ws = R.random_codes(g, 200, 256, wscale, matrix=True)
    for kind in ("f32", "e8m0"):
        xb = torch.full((2, M), 127, dtype=torch.uint8)
        xb[0, 0], xb[1, M // 2], xb[0, M - 1] = 0, 200, 27
        xs = xb.view(torch.float8_e8m0fnu)
        xs = xs.float() if kind == "f32" else xs
        got = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda()).cpu()
        want, mag = R.matmul(x, xs, w, ws)
        assert ((got.double() - want).abs() <= R.matmul_tol(want, mag, 256, torch.bfloat16)).all()


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("B,rows", [(3, 1), (4, 4)])
def test_layer_of_few_rows(S, B, rows, scale):
    """A decode step of a layer (up to 16 rows): each product in fp32's sums."""
    layer = L.Layer(S, scale, seed=4)
    g = torch.Generator()
    g.manual_seed(B)
    pool = S.PagePool(B * 16, L.HKV, L.HD, L.PAGE, "bf16")
    pool.buf.zero_()
    table = torch.arange(B * 16, dtype=torch.int32, device="cuda").view(B, 16)
    lens, n, t = torch.tensor([7 * i for i in range(B)], dtype=torch.int32, device="cuda"), B * rows, {}
    layer.run(pool, torch.randn(n, L.D, generator=g).bfloat16().cuda(), (3 * torch.randn(n, L.D, generator=g)).cuda(), table, lens, B, rows, trace=t)
    t = {k: v.cpu() for k, v in t.items()}
    for nm, c, s, out in (("qkv", "c1", "s1", "qkv"), ("o", "c2", "s2", "o"), ("gate_up", "c3", "s3", "gu"), ("down", "c4", "s4", "y")):
        x, w = L.values(t[c], t[s]), layer.values[nm]
        want, mag = x @ w.t(), x.abs() @ w.abs().t()
        tol = R.matmul_tol(want, mag, x.shape[1], torch.bfloat16)
        assert ((t[out].double() - want).abs() <= tol).all(), nm
