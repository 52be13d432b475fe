"""A paged cache driven on a stream of its own, while the current one is busy."""
import numpy as np
import pytest
import torch

import workloads as W
from gpu_helpers import to_dev_i32

pytestmark = pytest.mark.gpu

SHAPE = W.ModelShape(2, 512, 8, 2, 64, 1024, 2048, 1e-6, 1e6, True, "bf16")


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    assert sdd.device_ok(), "needs a gfx950 device"
    return sdd


@pytest.fixture(scope="module")
def model(S):
    m = S.Model(SHAPE)
    m.init_random(31, W.WEIGHT_SIGMA)
    torch.cuda.synchronize()
    return m


def busy(n=12):
    """Some milliseconds of work on the current stream, from tensors that stay."""
    x = torch.randn(8192, 8192, device="cuda")
    for _ in range(n):
        x = x @ x * 1e-4
    return x


def rounds(S, m, stream, gap):
    """A sequence prefilled, verified, released, and another one in its pages; `gap` before each call."""
    V = SHAPE.vocab
    toks = [to_dev_i32(W.prompt(40 + i, 60 + 20 * i, V)) for i in range(2)]
    drafts = to_dev_i32(W.prompt(50, 8, V).reshape(1, 8))
    ids = [to_dev_i32([i]) for i in range(2)]
    logits = [torch.full((1, 9, V), float("nan"), device="cuda") for _ in range(3)]
    kept = [torch.full((1 << 14,), 3, dtype=torch.int32, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    del kept  # (freed blocks whose contents look like page ids)
    keep = [gap()]
    on = {} if stream is None else {"stream": stream}
    kv = S.PagedKVCache(m, 2, 160, 5, 32, "bf16", **on)
    ws = kv.workspace(16, **on)
    keep.append(gap())
    kv.assign(0, 70, **on)
    kv.prefill(0, toks[0], ws, **on)
    kv.verify(ids[0], drafts, logits[0], None, ws, **on)
    keep.append(gap())
    kv.release(0, **on)
    kv.assign(1, 90, **on)
    kv.prefill(1, toks[1], ws, **on)
    kv.verify(ids[1], drafts, logits[1], None, ws, **on)
    keep.append(gap())
    kv.assign(1, 100, **on)
    kv.verify(ids[1], drafts, logits[2], None, ws, **on)
    torch.cuda.synchronize()
    assert kv.state()[2] == 0
    return [t.cpu().numpy() for t in logits]


def test_a_cache_on_a_stream_of_its_own(S, model):
    """The table's fill, assignments and releases are ordered with the calls on the stream that is given for them, whatever the
    current stream is busy with."""
    want = rounds(S, model, None, lambda: None)
    got = rounds(S, model, torch.cuda.Stream(), busy)
    for a, b in zip(want, got):
        assert np.array_equal(a, b)


def test_a_cache_made_for_a_stream_and_used_within_it(S, model):
    """The constructor's stream, then assign() with that stream current."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy()
    kv = S.PagedKVCache(model, 1, 160, 5, 32, "bf16", stream=side)
    with torch.cuda.stream(side):
        kv.assign(0, 70)
        table = kv.table.clone()
    torch.cuda.synchronize()
    assert keep.shape == (8192, 8192)
    assert torch.equal(kv.table, table) and (kv.table[0, :3] >= 0).all() and (kv.table[0, 3:] == -1).all()
