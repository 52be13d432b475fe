"""How far paged attention of few rows is from the 64-bit result on the whole: by its outputs' rounding to bf16 and that of the
weights below the largest, which is 1 and is not rounded."""
import pytest
import torch

from test_gpu_paged import S, check_attention, fill, randn  # noqa: F401

pytestmark = pytest.mark.gpu

# A bf16 rounding is off by 2^-8 / sqrt(3) of the binade's lower end, root mean square; over values spread evenly within a binade's
# logarithm 1 / x^2 is 3 / (8 ln 2) on average.
EPS2 = (2.0 ** -8) ** 2 / 3 * 0.5410


@pytest.mark.parametrize("hq, hkv, page, R, at", [(28, 4, 64, 1, [512, 300, 700]), (64, 8, 64, 1, [3000, 1900]), (64, 8, 32, 2, [200, 90, 33])])
@pytest.mark.parametrize("spread", [1.0, 2.5, 6.0])
def test_error_is_that_of_the_roundings(S, hq, hkv, page, R, at, spread):  # noqa: F811
    """Over all values of a call, from flat rows to rows that one position carries.  A tenth is for the mean of that many roundings
    (thousands), and for the parts of a sequence, each of which has a largest weight of its own."""
    hd = 128
    c, k, v = fill(S, "bf16", hkv, hd, page, R, at, seed=17)
    q = (spread * randn(23, len(at), R, hq, hd)).to(torch.bfloat16)
    got = check_attention(S, c, k, v, q, at).cpu().double()
    off = expected = 0.0
    for b, a in enumerate(at):
        for r in range(R):
            for h in range(hq):
                kk, vv = k[b][:a + r + 1, h * hkv // hq], v[b][:a + r + 1, h * hkv // hq]
                w = torch.softmax(kk @ q[b, r, h].double() * hd ** -0.5, 0)
                o = w @ vv
                off += ((got[b, r, h] - o) ** 2).sum().item()
                rounded = w ** 2
                rounded[w.argmax()] = 0
                expected += EPS2 * ((o ** 2).sum() + (rounded[:, None] * vv ** 2).sum()).item()
    assert off <= 1.1 ** 2 * expected, (off / expected) ** 0.5
