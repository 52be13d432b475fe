"""Values at the ends of fp32's range in the 8-bit operators: tiny blocks, norms whose squares leave it, far gates, far scales."""
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


NORM_ROWS = {  # factor of rows of size 1, eps
    "large": (1e20, 2.0 ** -20), "largest": (2.0 ** 124, 2.0 ** -20), "one_large": (1.0, 2.0 ** -20), "small": (1e-25, 0.0),
    "smallest": (2.0 ** -130, 0.0), "small_beside_eps": (2.0 ** -70, 2.0 ** -140), "eps_above": (2.0 ** -90, 2.0 ** -149),
    "border": (2.0 ** 63, 2.0 ** -20), "low_border": (2.0 ** -53, 0.0)}


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("res", [None, "bf16", "f32"])
@pytest.mark.parametrize("what", NORM_ROWS)
@pytest.mark.parametrize("M,K,dtype", [(1, 16, "f32"), (3, 400, "bf16"), (2, 3584, "bf16"), (2, 40000, "f32")])
def test_rmsnorm_squares_out_of_range(S, M, K, dtype, what, res, scale):
    """Rows of finite values whose squares are none: the same y as of rows of size 1."""
    size, eps = NORM_ROWS[what]
    g = gen(M, K, len(what))
    x = torch.randn(M, K, generator=g).clamp(-4, 4) * size
    if what == "one_large":
        x[:, K // 3] = 1e30
    x = x.to(DT[dtype])
    gain = 1 + 0.1 * torch.randn(K, generator=g)
    r = None if res is None else (2 * size * torch.randn(M, K, generator=g).clamp(-4, 4)).to(DT[res])
    held = None if r is None else r.cuda()
    codes, scales, ro, yo = S.e4m3_rmsnorm(x.cuda(), gain.cuda(), eps=eps, residual=held, y=True, scale=scale)
    codes, scales, yo = codes.cpu(), scales.cpu(), yo.cpu()
    wr, wy, rel_r, rel_y = R.rmsnorm(x, r, gain, eps)
    # a value far below its row's largest is a subnormal number, as it is in the row itself: half of 2^-149 times at most 1.5 * 256
    R.check_codes(wy, codes, scales.t(), scale, rel=rel_y, least=2.0 ** -140)
    assert ((yo.double() - wy).abs() <= wy.abs() * (rel_y + R.HALF[torch.bfloat16] * 1.01) + 2.0 ** -133).all()
    if r is not None:
        assert ((ro.cpu().double() - wr).abs() <= wr.abs() * (rel_r + R.HALF[DT[res]] * 1.01) + 2.0 ** -133).all()


def test_rmsnorm_zero_rows_beside_far_ones(S):
    """A row of zeros has no size: zeros with any eps above 0, no number with 0 (0 / 0); rows beside it do not matter."""
    x = torch.zeros(4, 160)
    x[1], x[3] = 1e25, 1e-30
    gain = torch.ones(160).cuda()
    codes, scales, _, y = (t if t is None else t.cpu() for t in S.e4m3_rmsnorm(x.cuda(), gain, eps=2.0 ** -120, y=True))
    assert (codes[0::2].float() == 0).all() and (scales[:, 0::2] == 1).all() and (y[0::2] == 0).all()
    assert ((y[1].float() - 1).abs() <= 2.0 ** -8).all() and ((y[3].float() - 1e-30 * 2.0 ** 60).abs() <= 2.0 ** -39 * 2.0 ** -8).all()
    codes, scales, _, y = (t if t is None else t.cpu() for t in S.e4m3_rmsnorm(x.cuda(), gain, eps=0.0, y=True))
    assert torch.isnan(y[0::2].float()).all() and torch.isnan(codes[0::2].float()).all() and (scales[:, 0::2] == 1).all()
    assert ((y[1::2].float() - 1).abs() <= 2.0 ** -8).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_swiglu_gates_next_to_the_end(S, dtype):
    """Gates for which 1 + e^-g is next to fp32's largest number, with values that bring the result back: not zero."""
    gates = [-86.0, -87.0, -87.5, -88.0, -88.5]
    x = torch.zeros(len(gates), 2 * 256)
    for m, g in enumerate(gates):
        x[m, 3], x[m, 256 + 3] = g, 1e30
        x[m, 200], x[m, 256 + 200] = g, -2.0
    x = x.to(DT[dtype])
    codes, scales = (t.cpu() for t in S.e4m3_swiglu(x.cuda()))
    y, rel, _ = R.swiglu(x)
    # the reciprocal's quarter may be a subnormal number of 22 bits; 2^-149: a step of products among the smallest numbers
    R.check_codes(y, codes, scales.t(), "f32", rel=rel + 2.0 ** -22, least=2.0 ** -148)
    v = codes.double() * R.spread(scales.double().t(), len(gates), 256, 1)
    assert (v[:, 3] != 0).all() and ((v - y).abs() <= y.abs() * 2.0 ** -4 * 1.01 + 2.0 ** -135).all()


@pytest.mark.parametrize("top", [-124, -118, -116, -114, -110, -106, -100, -94, -60, 0, 100])
def test_codes_are_the_nearest_of_fp32s_quotient(S, top):
    """y / s next to every border between two codes, with the block's maximum between 2^top and 2^(top + 1): the codes that IEEE's
    division and one rounding give, in blocks of the smallest numbers too."""
    g = gen(top + 200)
    M, K = 64, 1024
    a = torch.ldexp(1 + torch.rand(M, K // 128, generator=g), torch.tensor(top))
    s = torch.maximum(a / torch.full_like(a, 448), torch.tensor(2.0 ** -126))
    c = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    mid = ((c[1:] + c[:-1]) / 2)[torch.randint(0, 126, (M, K), generator=g)]
    x = (mid * s.double().repeat_interleave(128, 1)).float()
    x = (x.view(torch.int32) + torch.randint(-2, 3, (M, K), generator=g).int()).clamp(min=0).view(torch.float32)
    x = torch.minimum(x, a.repeat_interleave(128, 1))
    x[:, ::128] = a
    want = (x / s.repeat_interleave(128, 1)).to(torch.float8_e4m3fn).view(torch.uint8)
    codes, scales = S.e4m3_quantize(x.cuda())
    assert torch.equal(scales.cpu().t(), s)
    assert torch.equal(codes.cpu().view(torch.uint8), want)
    # a matrix of one block a tile of 128 rows: the same rule with the tile's maximum
    xm = x[:, :128]
    sm = torch.maximum(xm.max() / torch.tensor(448.0), torch.tensor(2.0 ** -126))
    codes, scales = S.e4m3_quantize_matrix(xm.cuda())
    assert scales.item() == sm.item()
    assert torch.equal(codes.cpu().view(torch.uint8), (xm / sm).to(torch.float8_e4m3fn).view(torch.uint8))


def far_pairs(M, N, K):
    """Codes and power-of-two scales: block 0 has pairs of scales whose product passes fp32's range at either end, block 1 ordinary ones.
    Rows by m % 4: zeros in block 0, one product of the smallest codes, two that cancel, scales far down."""
    g = gen(M, N, K)
    x = torch.zeros(M, K)
    x[:, 128:] = torch.randint(-4, 5, (M, K - 128), generator=g).float()
    w = torch.zeros(N, K)
    w[:, 128:] = torch.randint(-4, 5, (N, K - 128), generator=g).float()
    w[:, 1], w[:, 5], w[:, 9] = 2.0 ** -9, 1.5, 1.5
    w[:, 16:128] = 448.0
    xb = torch.full((R.blocks(K), M), 127)
    x[1::4, 1] = 2.0 ** -9
    x[2::4, 5], x[2::4, 9] = 3.0, -3.0
    x[3::4, 16:128] = 448.0
    x[3::4, 128:] = 0
    xb[0, :] = 127 + 100
    xb[0, 3::4] = 127 - 100 - 80
    wb = torch.full((R.blocks(N), R.blocks(K)), 127)
    wb[:, 0] = 127 + 30
    f8 = lambda t: t.to(torch.float8_e4m3fn)  # noqa: E731
    e8 = lambda t: t.clamp(0, 254).to(torch.uint8).view(torch.float8_e8m0fnu)  # noqa: E731
    return f8(x), e8(xb), f8(w), e8(wb)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(1, 40), (4, 300), (4, 9000), (4, 6000), (16, 300), (33, 300), (33, 33000), (64, 1040), (100, 33000), (70, 200), (200, 300),
                                 (300, 2100)])
def test_powers_of_two_whose_product_is_out_of_range(S, M, N, out):
    """Scales of 2^100 and 2^30 (and of 2^-127 and 2^-23): a block's sum times
    both is what counts, however many rows there are."""
    K = 272
    x, xs, w, ws = far_pairs(M, N, K)
    for wb0 in (157, 127 - 23):  # 2^30, 2^-23
        b = ws.view(torch.uint8).clone()
        b[:, 0] = wb0
        ws = b.view(torch.float8_e8m0fnu)
        got = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
        want, mag = R.matmul(x, xs, w, ws)
        assert torch.isfinite(got).all()
        tol = R.matmul_tol(want, mag, K, DT[out], R.group_max(x, xs, w, ws) if out == "bf16" and M > 16 else None)
        err = (got.double() - want).abs()
        assert (err <= tol).all(), (err / tol).max()
    b[:, 0] = 227  # 2^100 both: zeros and sums that cancel stay what they are, what passes the type's range is infinite
    got = S.E4M3Matrix(w.cuda(), b.view(torch.float8_e8m0fnu).cuda()).matmul(x.cuda(), xs.cuda(), dtype=DT[out]).cpu()
    plain, _ = R.matmul(x[:, 128:], xs[1:], w[:, 128:], ws[:, 1:])
    plain = plain.to(DT[out])  # (whole numbers under 2^12, which every sum holds)
    assert torch.equal(got[0::4], plain[0::4]) and torch.equal(got[2::4], plain[2::4])
    assert (got[1::4] == float("inf")).all()
