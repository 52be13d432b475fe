"""The decoder over a paged KV cache: prefill, verify, decode and commit against the oracle and a 64-bit decoder, next to the
contiguous cache.  Logits agree per row within 2e-2 of the row's largest (bf16 models' tolerance throughout the tests)."""
import numpy as np
import pytest
import torch

import oracle
import paged_ref as ref
import workloads as W
from gpu_helpers import row_tol_ok, to_dev_i32

pytestmark = pytest.mark.gpu

TOL = 2e-2
SHAPES = {"hd64": W.ModelShape(2, 512, 8, 2, 64, 1024, 2048, 1e-6, 1e6, True, "bf16"),
          "hd128": W.ModelShape(2, 384, 6, 2, 128, 1088, 2176, 1e-6, 1e6, False, "bf16")}


@pytest.fixture(scope="module")
def S():
    from paper_2608_14787_amd import sdd
    assert sdd.device_ok(), "needs a gfx950 device"
    return sdd


def verify(kv, seqs, drafts, V, ws):
    drafts = np.asarray(drafts, np.int32)
    lg = torch.full((len(seqs), drafts.shape[1] + 1, V), float("nan"), device="cuda")
    kv.verify(to_dev_i32(seqs), to_dev_i32(drafts), lg, None, ws)
    return lg


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("prompt, gamma", [(1, 0), (2, 4), (70, 8), (200, 32), (399, 33)])
def test_rounds_against_the_oracle(S, name, prompt, gamma):
    """Three rounds of verify and commit; pages handed out as the sequence grows, in an order of their own."""
    shape = SHAPES[name]
    m = S.Model(shape)
    m.init_random(0, W.WEIGHT_SIGMA)
    n = prompt + 3 * (gamma + 1) + 8
    kv = S.PagedKVCache(m, 1, n, 20, 32, "bf16")
    kv.free = [7, 3, 19, 0, 12, 1, 18, 5, 2, 16, 9, 4, 11, 17, 6, 8, 10, 13, 14, 15]
    kv.buf[256 + -(-n * shape.head_dim * 4 // 256) * 256:].fill_(255)  # NaN wherever nothing is written
    ws = kv.workspace(max(64, gamma + 1))
    om = oracle.Model(shape)
    okv = oracle.KV(om, n)
    toks = W.prompt(prompt, prompt, shape.vocab)
    kv.assign(0, prompt + gamma + 1)
    kv.prefill(0, to_dev_i32(toks), ws)
    okv.prefill(toks)
    for r in range(3):
        drafts = W.prompt(1000 + r, gamma, shape.vocab).reshape(1, gamma)
        kv.assign(0, int(kv.state()[0][0]) + gamma + 1)
        got = verify(kv, [0], drafts, shape.vocab, ws)[0].cpu().numpy()
        want = okv.verify(drafts[0])
        ok, rel = row_tol_ok(got, want, TOL)
        assert ok.all(), rel
        L = min(gamma, 2 + r)
        nxt = int(want[L].argmax())
        kv.commit(to_dev_i32([0]), to_dev_i32([L]), to_dev_i32([nxt]))
        okv.commit(L, nxt)
    ln, pd, err = kv.state()
    assert err == 0 and ln[0] == prompt - 1 + sum(min(gamma, 2 + r) + 1 for r in range(3))


def weights(shape, seed):
    g = torch.Generator().manual_seed(seed)
    bf = lambda *s, scale=0.05: (torch.randn(*s, generator=g) * scale).to(torch.bfloat16)  # noqa: E731
    d, hd, hq, hkv = shape.d_model, shape.head_dim, shape.n_q_heads, shape.n_kv_heads
    w = {"embed": bf(shape.vocab, d, scale=1.0), "lm": bf(shape.vocab, d), "layers": []}
    for _ in range(shape.n_layers):
        w["layers"].append(dict(q=bf(hq * hd, d), k=bf(hkv * hd, d), v=bf(hkv * hd, d), o=bf(d, hq * hd), gate=bf(shape.d_ff, d),
                                up=bf(shape.d_ff, d), down=bf(d, shape.d_ff)))
    return w


def load(S, m, w):
    m.init_random(0, 0.02)  # norm gains of 1
    m.load_tensor(S.T_EMBED, 0, w["embed"].cuda())
    m.load_tensor(S.T_LM_HEAD, 0, w["lm"].cuda())
    for i, l in enumerate(w["layers"]):
        for name, kind in (("q", S.T_WQ), ("k", S.T_WK), ("v", S.T_WV), ("o", S.T_WO), ("gate", S.T_WGATE), ("up", S.T_WUP), ("down", S.T_WDOWN)):
            m.load_tensor(kind, i, l[name].cuda())


def forward64(shape, w, tokens, cached):
    """Logits of all positions, attention reading `cached` (k, v [n, hkv, hd] a layer) instead of its own K/V; and its own."""
    hd, hq, hkv, eps = shape.head_dim, shape.n_q_heads, shape.n_kv_heads, shape.rms_eps
    rms = lambda x: x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)  # noqa: E731
    n = len(tokens)
    pos = torch.arange(n)
    x = w["embed"][torch.from_numpy(tokens).long()].double()
    own = []
    for l, (k, v) in zip(w["layers"], cached):
        W64 = {a: b.double() for a, b in l.items()}
        h = rms(x)
        one = torch.ones(hd) if shape.qk_norm else None
        q = ref.norm_rope((h @ W64["q"].T).view(n, hq, hd), one, eps, pos, shape.rope_theta)
        kk = ref.norm_rope((h @ W64["k"].T).view(n, hkv, hd), one, eps, pos, shape.rope_theta)
        own.append((kk, (h @ W64["v"].T).view(n, hkv, hd)))
        o = torch.stack([ref.attention(q[i:i + 1], k, v, i, hd ** -0.5)[0][0] for i in range(n)])
        x = x + o.flatten(1) @ W64["o"].T
        h = rms(x)
        x = x + (torch.nn.functional.silu(h @ W64["gate"].T) * (h @ W64["up"].T)) @ W64["down"].T
    return rms(x) @ w["lm"].double().T, own


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_logits_from_what_the_pages_hold(S, name, dtype):
    """The logits are those of the values that the pages stand for (read back), and those are the layers' K/V rounded once."""
    shape, gamma, n = SHAPES[name], 6, 75
    w = weights(shape, 3)
    m = S.Model(shape)
    load(S, m, w)
    kv = S.PagedKVCache(m, 2, 128, 9, 32, dtype)
    ws = kv.workspace(64)
    toks, drafts = W.prompt(5, n, shape.vocab), W.prompt(6, gamma, shape.vocab)
    kv.assign(1, n + gamma)
    kv.prefill(1, to_dev_i32(toks), ws)
    got = verify(kv, [1], drafts.reshape(1, gamma), shape.vocab, ws)[0].cpu().numpy()
    assert kv.state()[2] == 0
    every = n + gamma
    cached = []
    for layer in range(2):
        k, v = kv.pool(layer).read(kv.table[1:].contiguous(), to_dev_i32([0]), every)
        cached.append((k[0].cpu().double(), v[0].cpu().double()))
    want, own = forward64(shape, w, np.concatenate([toks, drafts]), cached)
    ok, rel = row_tol_ok(got, want[n - 1:].numpy(), TOL)
    assert ok.all(), rel
    for have, mine in zip(cached, own):
        for a, b in zip(have, mine):
            # the bf16 model's own error (a row's tolerance) and half a step of the cache's type
            half = 2.0 ** -4 if dtype == "e4m3" else 2.0 ** -8
            row = b.abs().amax(-1, keepdim=True)
            assert ((a - b).abs() <= 2 * TOL * row + half * b.abs().maximum(row * 2.0 ** -15) * (1 + TOL)).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_batched_ragged_and_many_rows(S, name, dtype):
    """Eight ragged sequences, 66 and more rows a call (the many-row kernel), one after the other and together: the same bits;
    a prompt of several chunks; full recompute; against the contiguous cache."""
    shape = SHAPES[name]
    m = S.Model(shape)
    m.init_random(11, W.WEIGHT_SIGMA)
    n, R, V = 8, 33, shape.vocab
    lens = [5 + 41 * s for s in range(n)]
    kv, cv = S.PagedKVCache(m, n, 400, 110, 32, dtype), S.KVCache(m, n, 400)
    ws = kv.workspace(n * R)
    for s in range(n):
        kv.assign(s, lens[s] + R)
        for c in (kv, cv):
            c.prefill(s, to_dev_i32(W.prompt(s, lens[s], V)), ws)
    drafts = W.prompt(50, n * (R - 1), V).reshape(n, R - 1)
    both = verify(kv, list(range(n)), drafts, V, ws)
    plain = verify(cv, list(range(n)), drafts, V, ws)
    # (8-bit K and V: their values are off by up to 2^-4 each, and scores and outputs by less than twice that)
    ok, rel = row_tol_ok(both.flatten(0, 1).cpu().numpy(), plain.flatten(0, 1).cpu().numpy(), TOL if dtype == "bf16" else TOL + 2.0 ** -3)
    assert ok.all(), rel.max()
    for seqs in ([0, 1], [6, 2, 4], [7, 5, 3, 1, 0]):
        assert torch.equal(verify(kv, seqs, drafts[seqs], V, ws), both[seqs]), seqs
    assert kv.state()[2] == 0
    # the whole of sequence 7 again without its cache, into slot 0's pages
    kv.assign(0, lens[7] + R)
    toks = np.concatenate([W.prompt(7, lens[7], V), drafts[7]])
    full = torch.empty((R, V), device="cuda")
    kv.verify_full(to_dev_i32(toks), R - 1, full, None, ws)
    ok, rel = row_tol_ok(full.cpu().numpy(), both[7].cpu().numpy(), TOL if dtype == "bf16" else TOL + 2.0 ** -3)
    assert ok.all(), rel.max()
    assert kv.state()[2] == 0


def test_pages_run_out_and_come_back(S):
    shape = SHAPES["hd64"]
    m = S.Model(shape)
    m.init_random(1, W.WEIGHT_SIGMA)
    kv = S.PagedKVCache(m, 3, 128, 5, 32, "bf16")
    ws, V = kv.workspace(64), shape.vocab
    kv.assign(0, 64)
    kv.assign(1, 96)
    with pytest.raises(S.SDDError) as e:
        kv.assign(2, 1)
    assert e.value.code == S.ECAPACITY
    with pytest.raises(ValueError):
        kv.assign(0, 129)
    prompt = W.prompt(3, 90, V)
    kv.prefill(1, to_dev_i32(prompt), ws)
    want = verify(kv, [1], np.zeros((1, 3), np.int32), V, ws)
    kv.release(0)
    kv.assign(2, 64)
    kv.prefill(2, to_dev_i32(W.prompt(4, 60, V)), ws)
    assert torch.equal(verify(kv, [1], np.zeros((1, 3), np.int32), V, ws), want)
    assert kv.state()[2] == 0
    # sequence 2 grows past its pages: reported, and sequence 1 keeps its results
    verify(kv, [2, 1], np.zeros((2, 20), np.int32), V, kv.workspace(64))
    assert kv.state()[2] == 4
    assert torch.equal(verify(kv, [1], np.zeros((1, 3), np.int32), V, ws), want)


def test_refusals(S):
    shape = SHAPES["hd64"]
    m = S.Model(shape)
    m.init_random(1, W.WEIGHT_SIGMA)
    kv = S.PagedKVCache(m, 1, 100, 4, 32)
    lg = torch.empty((1, 1, shape.vocab), device="cuda")
    with pytest.raises(S.SDDError) as e:  # a contiguous cache's workspace has no room for the paged part
        kv.verify(to_dev_i32([0]), torch.empty((1, 0), dtype=torch.int32, device="cuda"), lg, None, m.workspace(1))
    assert e.value.code == S.ECAPACITY
    for kw in (dict(page_size=33), dict(page_size=16), dict(n_pages=0)):
        with pytest.raises(S.SDDError):
            S.PagedKVCache(m, 1, 100, **{**dict(n_pages=4, page_size=32), **kw})
    with pytest.raises(S.SDDError) as e:
        kv.pool(2)
    assert e.value.code == S.EINVAL
    tiny = S.Model(W.TINY)
    with pytest.raises(S.SDDError) as e:
        S.PagedKVCache(tiny, 1, 100, 4)
    assert e.value.code == S.EUNSUPPORTED


MANY = {"hd64": W.ModelShape(2, 512, 16, 8, 64, 1024, 2048, 1e-6, 1e6, True, "bf16"),
        "hd128": W.ModelShape(2, 512, 16, 8, 128, 1088, 2176, 1e-6, 1e6, False, "bf16")}


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(MANY))
def test_many_query_vectors(S, name, dtype):
    """Calls that take the attention kernel of many query vectors (20 x 8 and 21 x 8 workgroups of 128): a batch of 20 sequences,
    and a prompt's chunk of 1300 rows, against the contiguous cache and against the sequences one by one."""
    shape = MANY[name]
    m = S.Model(shape)
    m.init_random(12, W.WEIGHT_SIGMA)
    n, R, V = 20, 33, shape.vocab
    assert n * 8 * -(-R * 2 // 128) >= 160 and 8 * -(-1300 * 2 // 128) >= 160
    tol = TOL if dtype == "bf16" else TOL + 2.0 ** -3  # (8-bit K and V, as above)
    lens = [3 + 31 * s for s in range(n)]
    kv, cv = S.PagedKVCache(m, n, 1400, 600, 32, dtype), S.KVCache(m, n, 1400)
    ws = kv.workspace(1400)
    for s in range(n):
        kv.assign(s, lens[s] + R)
        for c in (kv, cv):
            c.prefill(s, to_dev_i32(W.prompt(s, lens[s], V)), ws)
    drafts = W.prompt(51, n * (R - 1), V).reshape(n, R - 1)
    both = verify(kv, list(range(n)), drafts, V, ws)
    assert torch.equal(both, verify(kv, list(range(n)), drafts, V, ws))
    plain = verify(cv, list(range(n)), drafts, V, ws)
    ok, rel = row_tol_ok(both.flatten(0, 1).cpu().numpy(), plain.flatten(0, 1).cpu().numpy(), tol)
    assert ok.all(), rel.max()
    for s in (0, 7, 19):
        one = verify(kv, [s], drafts[s:s + 1], V, ws)[0].cpu().numpy()
        ok, rel = row_tol_ok(both[s].cpu().numpy(), one, TOL)
        assert ok.all(), (s, rel.max())
    for s in range(1, n):
        kv.release(s)
    kv.assign(0, 1301 + R)
    toks = to_dev_i32(W.prompt(77, 1301, V))
    for c in (kv, cv):
        c.prefill(0, toks, ws)
    got, want = (verify(c, [0], drafts[:1], V, ws)[0].cpu().numpy() for c in (kv, cv))
    ok, rel = row_tol_ok(got, want, tol)
    assert ok.all(), rel.max()
    assert kv.state()[2] == 0 and cv.state()[2] == 0


def test_a_batch_with_a_refused_sequence(S):
    """A sequence without room among many: reported, its rows' attention left alone, the others' results as without it."""
    shape = MANY["hd64"]
    m = S.Model(shape)
    m.init_random(13, W.WEIGHT_SIGMA)
    n, R, V = 20, 33, shape.vocab
    kv = S.PagedKVCache(m, n, 128, 70, 32, "bf16")
    ws = kv.workspace(n * R)
    for s in range(n):
        kv.assign(s, 96)
        kv.prefill(s, to_dev_i32(W.prompt(s, 60, V)), ws)
    drafts = W.prompt(52, n * (R - 1), V).reshape(n, R - 1)
    want = verify(kv, list(range(n)), drafts, V, ws)
    kv.commit(to_dev_i32([5]), to_dev_i32([50]), to_dev_i32([1]))  # 110 positions: 33 more pass max_len
    got = verify(kv, list(range(n)), drafts, V, ws)
    rest = [s for s in range(n) if s != 5]
    assert kv.state()[2] & 1
    assert torch.equal(got[rest], want[rest])
