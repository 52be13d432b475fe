"""Buffer sizes of caches at the ends of their arguments' ranges: exact, or refused (no GPU)."""
import ctypes as C

import pytest

from test_abi import S  # noqa: F401  (the built library)


def config(S, n_layers=2, hkv=8, hd=128):  # noqa: F811
    return S.ModelConfig(n_layers, 512, hkv, hkv, hd, 1024, 2048, 1e-6, 1e6, 0, S.BF16)


def up(x):
    return (x + 255) // 256 * 256


@pytest.mark.parametrize("max_batch", [1, 77, (1 << 30) - 1, 1 << 30, (1 << 31) - 1])
def test_paged_cache_of_many_sequences(S, max_batch):  # noqa: F811
    """Two words a sequence: the header is as large as what the constructor writes into it."""
    out, cfg = C.c_size_t(), config(S)
    assert S.lib().sdd_paged_kv_bytes(C.byref(cfg), max_batch, 100, 64, S.E4M3, 10, C.byref(out)) == S.OK
    assert out.value == up((2 * max_batch + 1) * 4) + up(100 * 128 * 4) + 2 * up(10 * 8 * 64 * (2 * 128 + 2))


@pytest.mark.parametrize("max_batch", [1, 77, (1 << 30) - 1, 1 << 30, (1 << 31) - 1])
def test_contiguous_cache_of_many_sequences(S, max_batch):  # noqa: F811
    out, cfg = C.c_size_t(), config(S, hkv=1, hd=64)
    assert S.lib().sdd_kv_bytes(C.byref(cfg), max_batch, 10, C.byref(out)) == S.OK
    assert out.value == up((2 * max_batch + 1) * 4) + up(10 * 64 * 4) + 4 * up(max_batch * 64 * 64 * 2)


@pytest.mark.parametrize("n_layers, n_pages, code", [(9, (1 << 31) - 1, -1), (8, (1 << 31) - 1, 0), (64, (1 << 31) - 1, -1),
                                                   ((1 << 31) - 1, 1 << 16, -1), (80, 1 << 20, 0)])
def test_paged_cache_past_the_address_range(S, n_layers, n_pages, code):  # noqa: F811
    """Pools of up to 2^60 - 2^29 bytes a layer (so eight are 2^63 - 2^32): layers past 2^63 bytes in all are refused, not counted modulo 2^64."""
    out, cfg = C.c_size_t(5), config(S, n_layers, hkv=1024)
    assert S.lib().sdd_paged_kv_bytes(C.byref(cfg), 1, 100, 1024, S.BF16, n_pages, C.byref(out)) == code
    if code == 0:
        assert out.value == 256 + up(100 * 128 * 4) + n_layers * n_pages * 1024 * 1024 * 128 * 4
