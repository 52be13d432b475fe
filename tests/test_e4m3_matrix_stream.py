"""A matrix in 8 bits that is laid out on another stream than its inputs' own: their memory stays theirs until that stream has read it."""
import contextlib

import pytest
import torch

import e4m3_ref as R
from test_abi import S  # noqa: F401  (the built library)


class Library:
    """Stands for libsdd where no device is: every call succeeds."""

    def sdd_e4m3_matrix_bytes(self, desc, out):
        out._obj.value = 4096
        return 0

    def sdd_e4m3_matrix_load(self, *a):
        return 0


@pytest.mark.parametrize("stream", [None, object()])
def test_inputs_are_recorded_on_the_stream(S, monkeypatch, stream):  # noqa: F811
    """(CPU) The allocator hears of both inputs' use on a stream that is given, after the layout was queued there."""
    used = []

    def load(self, *a):
        used.append("load")
        return 0

    class Tensor(torch.Tensor):
        def record_stream(self, s):
            used.append((self.dtype, s))

    monkeypatch.setattr(Library, "sdd_e4m3_matrix_load", load)
    monkeypatch.setattr(S, "lib", lambda: Library())
    monkeypatch.setattr(S, "_here", lambda *t: 0)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    codes = torch.zeros(16, 128, dtype=torch.uint8).view(torch.float8_e4m3fn).as_subclass(Tensor)
    scales = torch.ones(1, 1).as_subclass(Tensor)
    S.E4M3Matrix(codes, scales, stream=stream)
    if stream is None:
        assert used == ["load"]
    else:
        assert used[0] == "load" and set(used[1:]) == {(torch.float8_e4m3fn, stream), (torch.float32, stream)}


@pytest.mark.gpu
def test_inputs_dropped_while_the_stream_is_busy(S):  # noqa: F811
    """A loading loop: codes made on the current stream, laid out on another behind queued work, dropped, their memory asked for again
    and filled."""
    g = torch.Generator()
    g.manual_seed(1)
    N, K = 2048, 4096
    x, xs = (t.cuda() for t in R.random_codes(g, 20, K, "f32"))
    w, ws = R.random_codes(g, N, K, "f32", matrix=True)
    want = S.E4M3Matrix(w.cuda(), ws.cuda()).matmul(x, xs)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    made, others = [], []
    torch.cuda.synchronize()
    for _ in range(4):
        codes, scales = w.cuda(), ws.cuda()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(8):
                busy = busy @ busy * 1e-4
        made.append(S.E4M3Matrix(codes, scales, stream=side))
        del codes, scales
        others.append([torch.full((N, K), 0x7f, dtype=torch.uint8, device="cuda"), torch.full(ws.shape, float("nan"), device="cuda")])
    side.synchronize()
    for m in made:
        assert torch.equal(m.matmul(x, xs), want)
