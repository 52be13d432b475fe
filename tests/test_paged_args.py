"""Host-side refusals of the paged cache's operators and of sdd_token_logprobs: found before anything is launched (no GPU)."""
import ctypes as C
import os

import pytest

from test_abi import S  # noqa: F401  (the built library)

A = 1 << 20  # an aligned address that is never followed


def pages(S, hkv=8, hd=128, page=64, dtype=None, n=10, at=A):
    return S.PagesDesc(hkv, hd, page, S.BF16 if dtype is None else dtype, n, at)


@pytest.mark.parametrize("kw, code", [
    (dict(), 0), (dict(dtype=2), 0), (dict(hd=64, page=32), 0), (dict(page=1024), 0),
    (dict(page=16), -1), (dict(page=48), -1), (dict(page=2048), -1), (dict(page=0), -1), (dict(page=-64), -1),
    (dict(hd=96), -5), (dict(hd=0), -5), (dict(dtype=0), -1), (dict(dtype=7), -1), (dict(n=0), -1), (dict(n=-1), -1),
    (dict(hkv=0), -1), (dict(hkv=-8), -1)])
def test_pool_shapes(S, kw, code):  # noqa: F811
    out = C.c_size_t(77)
    d = pages(S, **kw)
    assert S.lib().sdd_pages_bytes(C.byref(d), C.byref(out)) == code
    if code == 0:
        es = 1 if d.dtype == S.E4M3 else 2
        assert out.value == d.n_pages * d.n_kv_heads * d.page_size * (2 * d.head_dim * es + (2 if es == 1 else 0))
    assert S.lib().sdd_pages_bytes(None, C.byref(out)) == S.EINVAL
    assert S.lib().sdd_pages_bytes(C.byref(pages(S)), None) == S.EINVAL


def test_bytes_past_32_bits(S):  # noqa: F811
    out = C.c_size_t()
    assert S.lib().sdd_pages_bytes(C.byref(pages(S, n=1 << 20)), C.byref(out)) == S.OK
    assert out.value == (1 << 20) * 8 * 64 * 2 * 128 * 2


def append(S, d=None, **kw):  # noqa: F811
    a = dict(table=A, width=4, len=A, B=2, R=3, hq=64, qkv=A, dt=S.BF16, stride=80 * 128, qg=A, kg=A, eps=1e-6, rope=A,
             max_pos=100, out=A, err=None)
    a.update(kw)
    d = pages(S) if d is None else d
    return S.lib().sdd_paged_append(C.byref(d), a["table"], a["width"], a["len"], a["B"], a["R"], a["hq"], a["qkv"], a["dt"],
                                    a["stride"], a["qg"], a["kg"], a["eps"], a["rope"], a["max_pos"], a["out"], a["err"], None)


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(len=None), dict(qkv=None), dict(out=None), dict(B=0), dict(R=0), dict(R=-1), dict(R=1 << 25), dict(width=0),
    dict(hq=0), dict(hq=12), dict(hq=-8), dict(dt=2), dict(stride=80 * 128 - 8), dict(stride=80 * 128 + 4), dict(qkv=A + 8),
    dict(out=A + 2), dict(qg=None), dict(kg=None), dict(qg=A + 4), dict(rope=A + 8), dict(max_pos=0), dict(eps=-1.0)])
def test_append_refusals(S, kw):  # noqa: F811
    assert append(S, **kw) == S.EINVAL, kw


def test_append_pool_refusals(S):  # noqa: F811
    assert append(S, pages(S, at=0)) == S.EINVAL
    assert append(S, pages(S, at=A + 64)) == S.EINVAL
    assert append(S, pages(S, hd=32)) == S.EUNSUPPORTED


def attend(S, d=None, **kw):  # noqa: F811
    a = dict(table=A, width=4, len=A, B=2, R=3, hq=64, q=A, scale=0.1, max_len=200, out=A, ws=A, n=1 << 40)
    a.update(kw)
    d = pages(S) if d is None else d
    return S.lib().sdd_paged_attention(C.byref(d), a["table"], a["width"], a["len"], a["B"], a["R"], a["hq"], a["q"], a["scale"],
                                       a["max_len"], a["out"], None, a["ws"], a["n"], None)


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(len=None), dict(q=None), dict(out=None), dict(B=0), dict(R=0), dict(width=0), dict(hq=0), dict(hq=9),
    dict(max_len=0), dict(max_len=-5), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=A + 8), dict(out=A + 4),
    dict(ws=None), dict(ws=A + 16), dict(R=1 << 21)])
def test_attention_refusals(S, kw):  # noqa: F811
    assert attend(S, **kw) == S.EINVAL, kw


def test_attention_workspace(S):  # noqa: F811
    out = C.c_size_t()
    d = pages(S)
    size = S.lib().sdd_paged_attention_workspace_bytes
    assert size(C.byref(d), 2, 3, 64, 200, C.byref(out)) == S.OK and out.value > 0
    need = out.value
    assert attend(S, n=need - 1) == S.ENOMEM
    assert size(C.byref(d), 2, 3, 64, 100, C.byref(out)) == S.OK and out.value == 0  # one chunk: written directly
    for bad in [(0, 3, 64, 200), (2, 0, 64, 200), (2, 3, 63, 200), (2, 3, 64, 0)]:
        assert size(C.byref(d), *bad, C.byref(out)) == S.EINVAL
    assert size(C.byref(d), 2, 3, 64, 200, None) == S.EINVAL


@pytest.mark.parametrize("kw", [dict(start=None), dict(table=None), dict(k=None), dict(v=None), dict(k=A + 8), dict(B=0), dict(n=0),
                                dict(n=-3), dict(width=0)])
def test_read_refusals(S, kw):  # noqa: F811
    a = dict(table=A, width=4, start=A, B=2, n=3, k=A, v=A)
    a.update(kw)
    assert S.lib().sdd_paged_read(C.byref(pages(S)), a["table"], a["width"], a["start"], a["B"], a["n"], a["k"], a["v"], None,
                                  None) == S.EINVAL


@pytest.mark.parametrize("kw, code", [
    (dict(z=None), -1), (dict(dt=2), -1), (dict(B=0), -1), (dict(R=0), -1), (dict(V=0), -1), (dict(V=(1 << 28) + 1), -1),
    (dict(tokens=None), -1), (dict(lp=None), -1), (dict(n=33), -1), (dict(n=-1), -1), (dict(top=None), -1), (dict(tlp=None), -1),
    (dict(stride=2999), -1), (dict(ws=None), -1), (dict(ws=A + 8), -1), (dict(z=A + 2), -1), (dict(bytes=1000), -2)])
def test_logprobs_refusals(S, kw, code):  # noqa: F811
    a = dict(z=A, dt=0, stride=3000, B=2, R=3, V=1000, tokens=A, n=5, lp=A, ent=A, top=A, tlp=A, ws=A, bytes=1 << 40)
    a.update(kw)
    assert S.lib().sdd_token_logprobs(a["z"], a["dt"], a["stride"], a["B"], a["R"], a["V"], a["tokens"], a["n"], a["lp"], a["ent"],
                                      a["top"], a["tlp"], a["ws"], a["bytes"], None) == code


def test_rope_table_refusals(S):  # noqa: F811
    f = S.lib().sdd_rope_table
    for args in [(None, 4, 64, 1e4), (A, 0, 64, 1e4), (A, 4, 63, 1e4), (A, 4, 0, 1e4), (A, 4, 64, 0.0), (A, 4, 64, float("nan"))]:
        assert f(*args, None) == S.EINVAL


def test_binding_refusals(S):  # noqa: F811
    import torch
    buf = torch.empty(2 * 2 * 32 * 2 * 64 * 2, dtype=torch.uint8)
    pool = S.PagePool(2, 2, 64, 32, "bf16", device="cpu", buf=buf)
    t, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        S.PagePool(3, 2, 64, 32, "bf16", device="cpu", buf=buf)  # too small
    with pytest.raises(ValueError):
        S.PagePool(2, 2, 64, 32, "fp8", device="cpu", buf=buf)
    with pytest.raises(ValueError):
        pool.attention(q.float(), t, n)
    with pytest.raises(ValueError):
        pool.attention(q, t.long(), n)
    with pytest.raises(ValueError):
        pool.attention(q, t, n.repeat(2))
    with pytest.raises(ValueError):
        pool.append(torch.zeros(1, 1, 7 * 64, dtype=torch.bfloat16), 4, t, n)
    with pytest.raises(ValueError):
        pool.append(torch.zeros(1, 1, 8 * 64, dtype=torch.bfloat16), 4, t, n, q_norm=torch.zeros(65))
    with pytest.raises(ValueError):
        S.token_logprobs(torch.zeros(1, 2, 8), torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        S.token_logprobs(torch.zeros(1, 8, 2).transpose(1, 2))
    assert os.path.exists(S.LIB_PATH)


@pytest.mark.parametrize("B, n", [(2 ** 31 - 1, 1 << 24), (1 << 30, 3), (65, 1 << 24)])
def test_more_positions_than_an_index_holds(S, B, n):  # noqa: F811
    d = pages(S)
    assert S.lib().sdd_paged_read(C.byref(d), A, 4, A, B, n, A, A, None, None) == S.EINVAL
    assert append(S, B=B, R=n) == S.EINVAL


def test_attention_workspace_of_extreme_shapes(S):  # noqa: F811
    """Sizes stay in range where the product of all factors would pass 64 bits."""
    out = C.c_size_t()
    hkv = 1024
    big = pages(S, hkv=hkv)
    size = S.lib().sdd_paged_attention_workspace_bytes
    for B, R, hq in ((1 << 24, 1, hkv), (1, 1 << 20, hkv), (1 << 12, 1 << 12, 64 * hkv)):
        assert size(C.byref(big), B, R, hq, 1 << 30, C.byref(out)) == S.OK
        assert 0 < out.value <= B * 512 * 16 * 130 * 4 + 2048 * 128 * 130 * 4
