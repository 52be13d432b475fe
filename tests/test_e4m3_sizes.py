"""Sizes past 32 bits, which the C side's ints cannot hold, are refused by the binding of the 8-bit operators (no GPU)."""
import pytest
import torch

from test_abi import S  # noqa: F401  (the built library)

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def meta(*shape, dtype=torch.bfloat16):
    """A tensor of which only the shape exists."""
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.fixture
def reached(S, monkeypatch):  # noqa: F811
    """What the C side would be called with, of operators that launch something."""
    real, calls = S.lib(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith(("_bytes", "_error")):
                return getattr(real, name)
            return lambda *a: calls.append((name, a)) or 0

    monkeypatch.setattr(S, "lib", lambda: Library())
    monkeypatch.setattr(S, "_here", lambda *t: 0)
    return calls


def matrix(S, N, K):  # noqa: F811
    return S.E4M3Matrix(meta(N, K, dtype=F8), meta(-(-N // 128), -(-K // 128), dtype=torch.float32))


BIG = 1 << 32


@pytest.mark.parametrize("rows", [BIG + 33, BIG, 1 << 31, (1 << 31) + 5, -1, 0, 33 - BIG])
def test_workspace_rows(S, reached, rows):  # noqa: F811
    with pytest.raises(S.SDDError) as e:
        matrix(S, 300, 4096).workspace(rows)
    assert e.value.code == S.EINVAL


@pytest.mark.parametrize("N,K", [(1, BIG + 16), (BIG + 16, 16), (1 << 31, 16), (16, 1 << 31), (BIG + 16, 1 << 20)])
def test_matrix(S, reached, N, K):  # noqa: F811
    with pytest.raises(S.SDDError) as e:
        matrix(S, N, K)
    assert e.value.code == S.EINVAL and not reached


@pytest.mark.parametrize("M", [BIG + 33, BIG + 1, 1 << 31])
def test_rows_of_a_product(S, reached, M):  # noqa: F811
    m = matrix(S, 300, 256)
    reached.clear()
    for ws in (None, meta(64, dtype=torch.uint8)):
        with pytest.raises(S.SDDError) as e:
            m.matmul(meta(M, 256, dtype=F8), meta(2, M, dtype=torch.float32), ws=ws)
        assert e.value.code == S.EINVAL and not reached


@pytest.mark.parametrize("M,K", [(BIG + 33, 16), (1 << 31, 256), (1, BIG + 16), (3, 1 << 31)])
@pytest.mark.parametrize("what", ["quantize", "quantize_matrix", "swiglu", "rmsnorm"])
def test_rows(S, reached, what, M, K):  # noqa: F811
    with pytest.raises(S.SDDError) as e:
        if what == "rmsnorm":
            S.e4m3_rmsnorm(meta(M, K), meta(K, dtype=torch.float32), residual=meta(M, K))
        else:
            getattr(S, "e4m3_" + what)(meta(M, 2 * K if what == "swiglu" else K))
    assert e.value.code == S.EINVAL and not reached


def test_sizes_within_reach_the_library(S, reached):  # noqa: F811
    """The largest ones that an int holds are the C side's to refuse."""
    S.e4m3_quantize(meta((1 << 31) - 1, 16))
    assert reached[-1][0] == "sdd_e4m3_quantize" and reached[-1][1][3] == (1 << 31) - 1
    m = matrix(S, 1 << 24, 16)
    m.matmul(meta(5, 16, dtype=F8), meta(1, 5, dtype=E8))
    assert reached[-1][0] == "sdd_e4m3_matmul" and reached[-1][1][4] == 5
