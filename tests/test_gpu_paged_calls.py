"""The paged decoder called as a server calls it: captured and replayed, its lengths and block table on the device, and with
sequence ids that are not there."""
import numpy as np
import pytest
import torch

import workloads as W
from gpu_helpers import to_dev_i32

pytestmark = pytest.mark.gpu

SHAPES = {"hd64": W.ModelShape(2, 512, 8, 2, 64, 1024, 2048, 1e-6, 1e6, True, "bf16"),
          "hd128": W.ModelShape(2, 512, 16, 8, 128, 1088, 2176, 1e-6, 1e6, False, "bf16")}


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    assert sdd.device_ok(), "needs a gfx950 device"
    return sdd


def cache(S, m, dtype, lens, room):
    n = len(lens)
    kv = S.PagedKVCache(m, n, room, sum(-(-room // 32) for _ in lens) + 3, 32, dtype)
    ws = kv.workspace(n * 33)
    for s, L in enumerate(lens):
        kv.assign(s, L)
        kv.prefill(s, to_dev_i32(W.prompt(60 + s, L, m.shape.vocab)), ws)
    return kv, ws


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name, lens, gamma", [("hd64", [60, 3, 200], 4), ("hd64", [40], 0), ("hd128", [100, 31, 64, 7, 350], 32)])
def test_rounds_captured_and_replayed(S, name, lens, gamma, dtype):
    """Verify and commit as one graph, replayed while sequences grow into pages that are assigned between the replays: every
    round equals the eager calls'.  Eager work of the program's own runs between them."""
    m = S.Model(SHAPES[name])
    m.init_random(41, W.WEIGHT_SIGMA)
    n, V, room = len(lens), SHAPES[name].vocab, max(lens) + 6 * (gamma + 1)
    a, ws_a = cache(S, m, dtype, lens, room)
    b, ws_b = cache(S, m, dtype, lens, room)
    ids, acc = to_dev_i32(list(range(n))), to_dev_i32([min(gamma, i + 1) for i in range(n)])
    drafts, nxt = torch.zeros(n, gamma, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    lg_a, lg_b = (torch.zeros(n, gamma + 1, V, device="cuda") for _ in range(2))
    am_a, am_b = (torch.zeros(n, gamma + 1, dtype=torch.int32, device="cuda") for _ in range(2))

    def step(kv, ws, lg, am):
        kv.verify(ids, drafts, lg, am, ws)
        kv.commit(ids, acc, nxt)

    def feed(r):
        drafts.copy_(torch.from_numpy(W.prompt(70 + r, n * gamma, V).reshape(n, gamma)))
        nxt.copy_(torch.from_numpy(W.prompt(80 + r, n, V)))
        for kv in (a, b):
            for s, L in enumerate(lens):
                kv.assign(s, min(room, L + r * (min(gamma, s + 1) + 1) + gamma + 1))

    feed(0)
    step(b, ws_b, lg_b, am_b)  # (the first round of both is eager)
    step(a, ws_a, lg_a, am_a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, ws_a, lg_a, am_a)
    for r in range(1, 5):
        feed(r)
        lg_a.fill_(float("nan"))
        g.replay()
        step(b, ws_b, lg_b, am_b)
        (lg_b[0, :1] @ lg_b[0, :1].T).sum()  # eager work of the program's own
        torch.cuda.synchronize()
        assert torch.equal(lg_a, lg_b) and torch.equal(am_a, am_b), r
    sa, sb = a.state(), b.state()
    assert sa[2] == sb[2] == 0 and np.array_equal(sa[0], sb[0]) and np.array_equal(sa[1], sb[1])


@pytest.mark.parametrize("gamma", [0, 8, 32])
def test_sequence_ids_that_are_not_there(S, gamma):
    """Refused and reported; the others' logits are those of a call of the same shape with ids that are, and their pages stay."""
    m = S.Model(SHAPES["hd128"])
    m.init_random(42, W.WEIGHT_SIGMA)
    V, lens = SHAPES["hd128"].vocab, [50, 90, 20, 33]
    kv, ws = cache(S, m, "bf16", lens, 160)
    for s, L in enumerate(lens):
        kv.assign(s, L + gamma + 1)
    drafts = to_dev_i32(W.prompt(90, 4 * gamma, V).reshape(4, gamma))
    want, got = (torch.full((4, gamma + 1, V), 5.0, device="cuda") for _ in range(2))
    kv.verify(to_dev_i32([3, 1, 2, 0]), drafts, want, None, ws)
    assert kv.state()[2] == 0
    before = kv.buf.clone()
    kv.verify(to_dev_i32([3, -1, 4, 0]), drafts, got, None, ws)
    assert kv.state()[2] == 4
    assert torch.equal(got[[0, 3]], want[[0, 3]]) and (got[[1, 2]] == 5).all()
    head = 256  # (lengths, pending tokens, the error word)
    assert torch.equal(kv.buf[head:], before[head:])
