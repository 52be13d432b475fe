"""Host-side refusals of the 8-bit products' operators: found before anything is launched (no GPU)."""
import ctypes as C

import pytest
import torch

from test_abi import S  # noqa: F401  (the built library)

A = 1 << 20  # an aligned address that is never followed


def rows(S, what="quantize", **kw):  # noqa: F811
    a = dict(x=A, dt=S.BF16, stride=512 if what == "swiglu" else 256, M=3, K=256, codes=A, scales=A, sd=S.F32)
    a.update(kw)
    f = getattr(S.lib(), "sdd_e4m3_" + what)
    return f(a["x"], a["dt"], a["stride"], a["M"], a["K"], a["codes"], a["scales"], a["sd"], None)


BAD_ROWS = [
    dict(x=None), dict(codes=None), dict(scales=None), dict(M=0), dict(M=-1), dict(M=(1 << 24) + 1), dict(K=0), dict(K=-16), dict(K=24),
    dict(K=255), dict(K=(1 << 20) + 16, stride=1 << 22), dict(K=1 << 30, stride=1 << 32), dict(K=(1 << 31) - 16, stride=1 << 32),
    dict(dt=2), dict(dt=3), dict(dt=-1), dict(sd=1), dict(sd=2), dict(sd=9), dict(stride=248), dict(stride=517), dict(stride=1 << 40),
    dict(x=A + 8), dict(codes=A + 4), dict(scales=A + 2)]


@pytest.mark.parametrize("what", ["quantize", "quantize_matrix", "swiglu"])
@pytest.mark.parametrize("kw", BAD_ROWS)
def test_row_refusals(S, what, kw):  # noqa: F811
    assert rows(S, what, **kw) == S.EINVAL, kw


def test_swiglu_needs_both_halves(S):  # noqa: F811
    assert rows(S, "swiglu", stride=256 + 248) == S.EINVAL


def norm(S, **kw):  # noqa: F811
    a = dict(x=A, dt=S.BF16, stride=256, res=A, ro=A, rd=S.F32, gain=A, eps=1e-6, M=3, K=256, codes=A, scales=A, sd=S.F32, y=A)
    a.update(kw)
    return S.lib().sdd_e4m3_rmsnorm(a["x"], a["dt"], a["stride"], a["res"], a["ro"], a["rd"], a["gain"], a["eps"], a["M"], a["K"],
                                    a["codes"], a["scales"], a["sd"], a["y"], None)


@pytest.mark.parametrize("kw", BAD_ROWS + [
    dict(gain=None), dict(gain=A + 4), dict(res=None), dict(ro=None), dict(rd=2), dict(rd=3), dict(res=A + 8), dict(ro=A + 2), dict(y=A + 8),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_rmsnorm_refusals(S, kw):  # noqa: F811
    assert norm(S, **kw) == S.EINVAL, kw


def test_rmsnorm_rows_too_long(S):  # noqa: F811
    assert norm(S, K=65536 + 16, stride=70000) == S.EUNSUPPORTED


@pytest.mark.parametrize("N,K,code", [(1, 16, 0), (1000, 400, 0), (1 << 24, 16, 0), (16, 1 << 20, 0), (0, 16, -1), (-5, 16, -1),
                                      ((1 << 24) + 1, 16, -1), (16, 0, -1), (16, 24, -1), (16, (1 << 20) + 16, -1), (16, -16, -1)])
def test_matrix_shapes(S, N, K, code):  # noqa: F811
    out = C.c_size_t(77)
    d = S.MatrixDesc(N, K, S.F32, None)
    assert S.lib().sdd_e4m3_matrix_bytes(C.byref(d), C.byref(out)) == code
    if code == 0:
        kb, scales = -(-K // 128), -(-N // 128) * -(-K // 128) * 4
        assert out.value == -(-N // 16) * kb * 2048 + -(-scales // 256) * 256
    assert S.lib().sdd_e4m3_matrix_bytes(None, C.byref(out)) == S.EINVAL
    assert S.lib().sdd_e4m3_matrix_bytes(C.byref(S.MatrixDesc(16, 16, S.F32, None)), None) == S.EINVAL


@pytest.mark.parametrize("kw", [dict(data=None), dict(codes=None), dict(scales=None), dict(sd=1), dict(sd=2), dict(data=A + 128), dict(codes=A + 8),
                                dict(scales=A + 2), dict(N=0), dict(K=20)])
def test_matrix_load_refusals(S, kw):  # noqa: F811
    a = dict(N=100, K=256, data=A, codes=A, scales=A, sd=S.F32)
    a.update(kw)
    d = S.MatrixDesc(a["N"], a["K"], a["sd"], a["data"])
    assert S.lib().sdd_e4m3_matrix_load(C.byref(d), a["codes"], a["scales"], None) == S.EINVAL, kw


def matmul(S, **kw):  # noqa: F811
    a = dict(N=100, K=256, wd=S.F32, data=A, x=A, xs=A, sd=S.F32, M=7, out=A, od=S.BF16, stride=100, ws=A, n=1 << 40)
    a.update(kw)
    d = S.MatrixDesc(a["N"], a["K"], a["wd"], a["data"])
    return S.lib().sdd_e4m3_matmul(C.byref(d), a["x"], a["xs"], a["sd"], a["M"], a["out"], a["od"], a["stride"], a["ws"], a["n"], None)


@pytest.mark.parametrize("kw", [
    dict(data=None), dict(x=None), dict(xs=None), dict(out=None), dict(wd=1), dict(wd=2), dict(sd=1), dict(sd=2), dict(M=0), dict(M=-3), dict(M=(1 << 24) + 1), dict(od=2),
    dict(od=3), dict(stride=99), dict(stride=0), dict(stride=1 << 40), dict(data=A + 64), dict(x=A + 8), dict(out=A + 1), dict(out=A + 2, od=0),
    dict(xs=A + 1), dict(N=0), dict(K=17), dict(N=1 << 24, M=1 << 24, stride=1 << 24)])
def test_matmul_refusals(S, kw):  # noqa: F811
    assert matmul(S, **kw) == S.EINVAL, kw


def test_matmul_workspace(S):  # noqa: F811
    """More rows never need less; sizes asked for without a device."""
    out = C.c_size_t()
    for N, K in ((4608, 3584), (5120, 25600), (51200, 5120), (3584, 18944), (100, 16), (17, 4096)):
        d = S.MatrixDesc(N, K, S.F32, None)
        last = 0
        for M in (1, 16, 33, 64, 65, 100, 128, 129, 264, 511, 1000, 4095, 100000):
            assert S.lib().sdd_e4m3_matmul_workspace_bytes(C.byref(d), M, C.byref(out)) == S.OK
            assert out.value >= last
            last = out.value
    d = S.MatrixDesc(100, 256, S.E8M0, None)
    for args in ((None, 5, C.byref(out)), (C.byref(d), 0, C.byref(out)), (C.byref(d), 5, None), (C.byref(S.MatrixDesc(100, 250, S.F32, None)), 5, C.byref(out))):
        assert S.lib().sdd_e4m3_matmul_workspace_bytes(*args) == S.EINVAL


# ---- the binding's own checks --------------------------------------------------------------------------


def f8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8).view(torch.float8_e4m3fn)


@pytest.mark.parametrize("call", [
    lambda S: S.e4m3_quantize(torch.zeros(2, 3, 16)),
    lambda S: S.e4m3_quantize(torch.zeros(16, 2).t()),
    lambda S: S.e4m3_quantize(torch.zeros(0, 16)),
    lambda S: S.e4m3_quantize(torch.zeros(2, 16), scale="f16"),
    lambda S: S.e4m3_quantize(torch.zeros(2, 16), out=(f8(2, 17), torch.zeros(1, 2))),
    lambda S: S.e4m3_quantize(torch.zeros(2, 16), out=(torch.zeros(2, 16), torch.zeros(1, 2))),
    lambda S: S.e4m3_quantize(torch.zeros(2, 16), out=(f8(2, 16), torch.zeros(2, 1))),
    lambda S: S.e4m3_quantize(torch.zeros(2, 16), scale="e8m0", out=(f8(2, 16), torch.zeros(1, 2))),
    lambda S: S.e4m3_swiglu(torch.zeros(2, 33)),
    lambda S: S.e4m3_rmsnorm(torch.zeros(2, 16), torch.ones(15)),
    lambda S: S.e4m3_rmsnorm(torch.zeros(2, 16), torch.ones(16).bfloat16()),
    lambda S: S.e4m3_rmsnorm(torch.zeros(2, 16), torch.ones(16), residual=torch.zeros(2, 17)),
    lambda S: S.e4m3_rmsnorm(torch.zeros(2, 16), torch.ones(16), residual=torch.zeros(2, 16), residual_out=torch.zeros(2, 16).bfloat16()),
    lambda S: S.e4m3_rmsnorm(torch.zeros(2, 16), torch.ones(16), residual_out=torch.zeros(2, 16)),
    lambda S: S.e4m3_rmsnorm(torch.zeros(2, 16), torch.ones(16), y=torch.zeros(2, 16)),
    lambda S: S.E4M3Matrix(torch.zeros(3, 16), torch.zeros(1, 1)),
    lambda S: S.E4M3Matrix(f8(3, 16), torch.zeros(1, 2)),
])
def test_binding_refusals(S, call):  # noqa: F811
    with pytest.raises(ValueError, match="^(?!tensors must be on)"):  # (CPU tensors come that far otherwise)
        call(S)


def test_binding_types(S):  # noqa: F811
    with pytest.raises(TypeError):
        S.e4m3_quantize(torch.zeros(2, 16).half())
    with pytest.raises(TypeError):
        S.E4M3Matrix(f8(3, 16), torch.zeros(1, 1).bfloat16())
