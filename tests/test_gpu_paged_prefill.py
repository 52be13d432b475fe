"""Prefill into a paged cache: what its workspace decides, and what it does not."""
import pytest
import torch

import workloads as W
from gpu_helpers import to_dev_i32

pytestmark = pytest.mark.gpu

SHAPES = {"hd64": W.ModelShape(2, 512, 8, 2, 64, 1024, 2048, 1e-6, 1e6, True, "bf16"),
          "hd128": W.ModelShape(2, 384, 7, 1, 128, 1088, 2176, 1e-6, 1e6, False, "bf16"),
          "many": W.ModelShape(2, 512, 16, 8, 64, 1024, 2048, 1e-6, 1e6, True, "bf16")}


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    assert sdd.device_ok(), "needs a gfx950 device"
    return sdd


@pytest.mark.parametrize("rows", [1, 2, 9, 15, 16])
@pytest.mark.parametrize("max_len", [600, 40000])
def test_a_workspace_for_few_rows_serves_prefill(S, rows, max_len):
    """As the contiguous cache's does: a decode step's workspace is enough to prefill with."""
    shape = SHAPES["many"]
    m = S.Model(shape)
    m.init_random(22, W.WEIGHT_SIGMA)
    toks = to_dev_i32(W.prompt(3, 100, shape.vocab))
    kv = S.PagedKVCache(m, 1, max_len, 8, 32)
    kv.assign(0, 128)
    kv.prefill(0, toks, kv.workspace(rows))
    cv = S.KVCache(m, 1, max_len)
    cv.prefill(0, toks, cv.workspace(rows))
    assert kv.state()[2] == 0 and kv.state()[0][0] == 99 == cv.state()[0][0]


def cached(S, m, dtype, toks, ws_rows):
    """K/V of the prompt's positions in every layer, after a prefill with a workspace for ws_rows rows."""
    n = len(toks)
    kv = S.PagedKVCache(m, 1, n + 8, n // 32 + 2, 32, dtype)
    kv.assign(0, n)
    kv.prefill(0, to_dev_i32(toks), kv.workspace(ws_rows))
    assert kv.state()[2] == 0
    return [kv.pool(layer).read(kv.table, to_dev_i32([0]), n - 1) for layer in range(2)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("n", [130, 402, 1000, 2861])
def test_bits_do_not_depend_on_the_workspace(S, name, dtype, n):
    """Workspaces for 256 rows or more leave the same bits in the pages, however many chunks they make of the prompt."""
    m = S.Model(SHAPES[name])
    m.init_random(21, W.WEIGHT_SIGMA)
    toks = W.prompt(n, n, SHAPES[name].vocab)
    want = cached(S, m, dtype, toks, 256)
    for rows in (300, 512, 1024, 4096):
        for (k, v), (wk, wv) in zip(cached(S, m, dtype, toks, rows), want):
            assert torch.equal(k, wk) and torch.equal(v, wv), rows
