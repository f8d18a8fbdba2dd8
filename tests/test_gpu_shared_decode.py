"""Shared prefixes, weighed pages and rules on logits as they are used: in the layers and in prefill_decode."""
import math

import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, step, up
from test_gpu_kv8_decode import CFG, SCALE, SIZES, d, dec, models, tables, weights  # noqa: F401 (fixtures among them)
from test_gpu_logits import plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("what", ["nothing", "groups", "weights", "both"])
def test_the_layer_is_the_layer_whatever_a_step_says(d, models, quantized, what):  # noqa: F811
    """Bytes of rows and cache as without; weights are those of the attention call on the layer's own queries."""
    m = models(quantized)
    c = m.cfg
    H, Hq, Hkv, N = c.H, c.Hq, c.Hkv, (c.Hq + 2 * c.Hkv) * 128
    pages, S = 9, 6
    cos, sin = tables(pages * 64)
    lc = d.layer_cfg(H, Hq, Hkv, 128, c.F, pages * 64, c.eps, SCALE)
    rng = np.random.default_rng(3)
    host = rng.permutation(S * pages).reshape(S, pages).astype(np.int32)
    host[1:4, :5] = host[0, :5]          # the first four sequences share 320 tokens
    host[4, 2] = -1                      # and one has given up a page
    table, pos = up(host), up(np.array([330, 321, 400, 500, 300, 77], np.int32))
    x0 = ds.normal_bf16_torch(8600, (S, H), 1.0, 0.0, DEV)
    pool0 = d.kv8_pool(1, S * pages, Hkv)[0]
    old = ds.normal_bf16_torch(8601, (S * pages * 64, N), 1.0, 0.0, DEV)
    every = torch.arange(S * pages * 64, dtype=torch.int32, device=DEV)
    q = torch.empty((S * pages * 64, Hq, 128), dtype=torch.bfloat16, device=DEV)
    whole = up(np.arange(S * pages, dtype=np.int32).reshape(S, pages))
    d.det_kv8_rope_append(old, q, pool0, whole, every % (pages * 64), every // (pages * 64), cos, sin)
    _, struct = m.layers[0]
    ws = torch.empty(m.layer_workspace_bytes(lc, S), dtype=torch.uint8, device=DEV).fill_(0xFF)
    want, wpool = x0.clone(), pool0.clone()
    step(f"layer with {what}, quantized {quantized}")
    m.layer(struct, lc, want, wpool, table, pos, None, cos, sin, ws)
    groups = (up(np.array([0, 4, 6], np.int32)), up(np.array([320, 0], np.int32))) if what in ("groups", "both") else (None, None)
    given = torch.rand(table.shape, device=DEV) if what in ("weights", "both") else None
    add = None if given is None else given.clone()
    st = d.kv8_step(*groups, add)
    ws = torch.empty(m.layer_workspace_bytes(lc, S, step=st), dtype=torch.uint8, device=DEV).fill_(0xFF)
    x, pool = x0.clone(), pool0.clone()
    m.layer(struct, lc, x, pool, table, pos, None, cos, sin, ws, step=st)
    assert torch.equal(x, want) and torch.equal(pool, wpool)
    if add is not None:  # the queries: norm, projection and rotation as the layer does them
        packed = m.layers[0][0]
        h, qkv, qb = torch.empty((S, H), dtype=torch.bfloat16, device=DEV), torch.empty((S, N), dtype=torch.bfloat16, device=DEV), q[:S].clone()
        if quantized:
            codes, scales = torch.empty((S, H), dtype=torch.int8, device=DEV), torch.empty(d.det_quant_act_scales_bytes(S, H) // 4, device=DEV)
            d.det_rmsnorm_quant_q8(x0, packed["norm1"], codes, scales, c.eps)
            d.det_qgemm_w4a8(codes, scales, packed["wqkv"], qkv, N)
        else:
            d.det_rmsnorm(x0, packed["norm1"], h, c.eps)
            d.det_gemm_bf16(h, packed["wqkv"], qkv, N, H)
        d.det_kv8_rope_append(qkv, qb, pool0.clone(), table, pos, None, cos, sin)
        aws = torch.empty(d.det_attn_decode_kv8_weights_workspace_bytes(S, Hq, Hkv, 128, pages), dtype=torch.uint8, device=DEV)
        w = torch.empty_like(given)
        d.det_attn_decode_kv8_weights(qb, pool, table, pos + 1, None, None, None, given, w, torch.empty_like(qb), aws, SCALE)
        assert torch.equal(add, w)


def test_layer_steps_that_are_refused(d, models):  # noqa: F811
    m = models()
    c = m.cfg
    lc = d.layer_cfg(c.H, c.Hq, c.Hkv, 128, c.F, 64, c.eps, SCALE)
    cos, sin = tables(64)
    x, pos = torch.zeros((2, c.H), dtype=torch.bfloat16, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    pool, table = d.kv8_pool(1, 4, c.Hkv)[0], up(np.array([[0], [1]], np.int32))
    ws = torch.empty(m.layer_workspace_bytes(lc, 2), dtype=torch.uint8, device=DEV)
    rows, shared = up(np.array([0, 1, 2, 2], np.int32)), up(np.array([0, 0, 0], np.int32))
    with pytest.raises(d.api.DetError):                 # more groups than rows
        m.layer(m.layers[0][1], lc, x, pool, table, pos, None, cos, sin, ws, step=d.kv8_step(rows, shared))
    st = d.kv8_step(weights=torch.zeros(table.shape, device=DEV))
    with pytest.raises(d.api.DetError):                 # a workspace that is too small for weights
        m.layer(m.layers[0][1], lc, x, pool, table, pos, None, cos, sin, ws[:m.layer_workspace_bytes(lc, 2, step=st) - 1], step=st)
    with pytest.raises(ValueError):
        m.layer(m.layers[0][1], lc, x, pool, table, pos, None, cos, sin, ws, step=d.kv8_step(weights=torch.zeros((2, 2), device=DEV)))
    assert not x.any() and not pool.any()


@pytest.mark.parametrize("quantized", [False, True])
def test_continuations_of_long_prompts(dec, models, quantized, monkeypatch):  # noqa: F811
    """What shares whole chunks goes through the shared kernels; tokens and logits as from prompts that stand there several times."""
    m = models(quantized)
    lens = np.array([530, 256, 700, 40], dtype=np.int32)
    prompts = up(ds.uniform_int(8700, (4, 700), 0, CFG["V"] - 1))
    cos, sin = tables(760)
    policy = dec.SamplingPolicy(1.0, 50, 0.95, 77, torch.arange(20, dtype=torch.int32, device=DEV))
    step("five continuations of four prompts")
    monkeypatch.setattr(dec, "GROUPS_FROM", 1)
    shared, logits = dec.prefill_decode(m, prompts, up(lens), 50, cos, sin, policy=policy, keep_logits=True, samples=5)
    apart, want = dec.prefill_decode(m, prompts.repeat_interleave(5, 0), up(np.repeat(lens, 5)), 50, cos, sin, policy=policy, keep_logits=True)
    assert torch.equal(shared, apart) and all(torch.equal(a, b) for a, b in zip(logits, want))


def grammar(dec, V, seed):  # noqa: F811
    """Tokens in five classes; a state lets two or three of them through, -1 after the last."""
    rng = np.random.default_rng(seed)
    of = rng.integers(0, 5, V).astype(np.int32)
    lets = np.array([[1, 1, 0, 0, 1], [0, 1, 1, 0, 0], [0, 0, 1, 1, 1], [1, 0, 0, 1, 0]], bool)
    to = np.array([[1, 2, -1, -1, 3], [-1, 0, 2, -1, -1], [-1, -1, 3, 0, 1], [2, -1, -1, 1, -1]], np.int32)
    bits = np.zeros((4, -(-V // 32) * 32), np.uint32)
    bits[:, :V] = lets[:, of]
    words = (bits.reshape(4, -1, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return dec.Grammar(up(words.view(np.int32)), up(to), up(of)), lets, to, of


@pytest.mark.parametrize("samples", [1, 3])
def test_rules_between_the_head_and_the_token(dec, models, samples):  # noqa: F811
    """Every token is what the plain rules and the largest logit give on the head's own logits; a sequence alone gets the same."""
    m, V, n_new = models(), CFG["V"], 24
    lens = np.array([9, 70, 31], dtype=np.int32)
    host = ds.uniform_int(8800, (3, 70), 0, 60)
    prompts, (cos, sin) = up(host), tables(160)
    g, lets, to, of = grammar(dec, V, 5)
    biases = {3: 2.5, 700: -1.0, 41: 0.75}
    rules = dec.LogitsPolicy(1.3, 0.4, 0.2, biases, g)
    step(f"rules, {samples} samples")
    got, logits = dec.prefill_decode(m, prompts, up(lens), n_new, cos, sin, keep_logits=True, samples=samples, rules=rules)
    got, logits = got.cpu().numpy(), [x.cpu().numpy() for x in logits]
    for b in range(3 * samples):
        ids, state = host[b // samples, :lens[b // samples]].tolist(), 0
        start = len(ids)
        for j in range(n_new):
            h = dict(history=np.array([ids], np.int32), history_lens=np.array([len(ids)], np.int32), generated_from=np.array([start], np.int32),
                     penalties=np.array([[1.3, 0.4, 0.2]], np.float32), bias_begin=np.array([0, 3], np.int32), bias_tokens=np.array(list(biases), np.int32),
                     bias_values=np.array(list(biases.values()), np.float32))
            z, _ = plain(logits[j][b:b + 1], h, np.float32)
            if state >= 0:
                z[0, ~lets[state, of]] = -np.inf
            assert int(z[0].argmax()) == got[b, j], (b, j)
            state = int(to[state, of[got[b, j]]]) if state >= 0 else -1
            ids.append(int(got[b, j]))
    step("rules without kept logits, and a sequence alone")
    again, _ = dec.prefill_decode(m, prompts, up(lens), n_new, cos, sin, samples=samples, rules=rules)
    assert np.array_equal(again.cpu().numpy(), got)
    alone, _ = dec.prefill_decode(m, prompts[1:2], up(lens[1:2]), n_new, cos, sin, rules=rules)
    assert np.array_equal(alone[0].cpu().numpy(), got[samples])
    none, _ = dec.prefill_decode(m, prompts, up(lens), n_new, cos, sin, rules=dec.LogitsPolicy())
    plainly, _ = dec.prefill_decode(m, prompts, up(lens), n_new, cos, sin)
    assert torch.equal(none, plainly)


def test_rules_with_a_bf16_cache_and_sampling(dec, models):  # noqa: F811
    """Tokens that a bias bars are never drawn; draws do not depend on the batch."""
    m = dec.DecodeModel(dec.ModelCfg(**CFG), weights(8000, n_layers=2, **SIZES))
    prompts, lens, (cos, sin) = up(ds.uniform_int(8900, (4, 20), 0, CFG["V"] - 1)), up(np.array([20, 7, 13, 1], np.int32)), tables(64)
    policy = lambda ids: dec.SamplingPolicy(1.2, 40, 0.9, 5, torch.tensor(ids, dtype=torch.int32, device=DEV))  # noqa: E731
    step("sampling with biases")
    free, _ = dec.prefill_decode(m, prompts, lens, 30, cos, sin, policy=policy([0, 1, 2, 3]))
    barred = {int(t): -math.inf for t in free.unique().tolist()[::2]}
    rules = dec.LogitsPolicy(repetition=1.1, biases=barred)
    got, _ = dec.prefill_decode(m, prompts, lens, 30, cos, sin, policy=policy([0, 1, 2, 3]), rules=rules)
    assert not set(got.unique().tolist()) & set(barred)
    one, _ = dec.prefill_decode(m, prompts[2:3], lens[2:3], 30, cos, sin, policy=policy([2]), rules=rules)
    assert torch.equal(one[0], got[2])


@pytest.mark.parametrize("samples", [1, 3])
def test_sequences_that_give_up_pages(dec, models, samples, monkeypatch):  # noqa: F811
    """They come back to their budgets, alone as in a batch; with room for all pages nothing changes."""
    m = models()
    lens = np.array([600, 90, 330], dtype=np.int32)
    prompts, (cos, sin) = up(ds.uniform_int(9000, (3, 600), 0, CFG["V"] - 1)), tables(700)
    run = lambda p, n, s=samples, **more: dec.prefill_decode(m, p, up(n), 60, cos, sin, keep_logits=True, samples=s, **more)  # noqa: E731
    monkeypatch.setattr(dec, "GROUPS_FROM", 1)
    step("evict nothing")
    want, logits = run(prompts, lens)
    got, same = run(prompts, lens, evict=dec.EvictPolicy(keep=11, every=8))
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(logits, same))
    seen = []
    policy = dec.EvictPolicy(keep=6, every=16, first=1, recent=2)
    original = dec.KVPages.evict

    def spy(self, w, n, keep, *rest):
        gone = original(self, w, n, keep, *rest)
        seen.append([sum(x >= 0 for x in self.pages(s)[:-(-int(n[s]) // 64)]) for s in range(len(gone))])
        assert all(x >= 0 for s in range(len(gone)) for x in self.pages(s)[:1])
        return gone
    dec.KVPages.evict = spy
    try:
        step("evict to six pages")
        got, some = run(prompts, lens, evict=policy)
        for b in (0, 2):
            alone, one = run(prompts[b:b + 1], lens[b:b + 1], 1, evict=policy)
            assert torch.equal(alone[0], got[b * samples]) and all(torch.equal(o[0], l[b * samples]) for o, l in zip(one, some))
    finally:
        dec.KVPages.evict = original
    assert len(seen) == 9 and all(n <= 6 for counts in seen for n in counts)
    assert all(torch.equal(a[samples:2 * samples], b[samples:2 * samples]) for a, b in zip(some, logits))     # three pages: nothing to give up
    assert torch.equal(some[15][0], logits[15][0]) and not torch.equal(some[16][0], logits[16][0])             # ten pages: from the sixteenth step on
    with pytest.raises(ValueError):
        run(prompts, lens, evict=dec.EvictPolicy(keep=0))
    with pytest.raises(ValueError):
        dec.prefill_decode(dec.DecodeModel(dec.ModelCfg(**CFG), weights(8000, n_layers=2, **SIZES)), prompts, up(lens), 2, cos, sin, evict=policy)


def test_a_captured_step_follows_the_tables(dec, models, monkeypatch):  # noqa: F811
    """Groups, weights and workspace of a captured step stay where they are; after the tables have changed `tell` is enough."""
    m = models()
    B, T = 5, 700
    cos, sin = tables(T)
    st = m.new_state(B, T, cos, sin, reserve=False, n_pages=B * 11)
    st.pages.reserve([0], [400], [0])
    fill = ds.uniform_int(9300, (B, 399), 0, CFG["V"] - 1)
    rows = st.of_rows(torch.zeros(399, dtype=torch.int32, device=DEV))
    rows.tokens.copy_(up(fill[0]))
    rows.positions.copy_(torch.arange(399, dtype=torch.int32, device=DEV))
    step("a prompt")
    rows.forward()
    st.pages.fork(0, range(1, B), 399)
    tokens, positions = torch.arange(B, dtype=torch.int32, device=DEV), torch.full((B,), 399, dtype=torch.int32, device=DEV)
    st.pages.reserve(range(B), [T] * B, [399] * B)

    def forward(groups, weights):
        st.groups, st.weights = groups, weights
        st.tokens.copy_(tokens)
        st.positions.copy_(positions)
        st.forward()
        return st.logits.clone()

    with pytest.raises(ValueError):
        forward([0, 3], None)
    with pytest.raises(ValueError):
        forward([], None)
    with monkeypatch.context() as to, pytest.raises(RuntimeError):
        to.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
        st.groups = [0, B]
        st.tell()
    few = st.of_rows(torch.zeros(2, dtype=torch.int32, device=DEV))
    few.groups = [0, 2]
    with pytest.raises(ValueError):
        few.tell()
    step("eager")
    want = forward(None, None)
    weights = torch.zeros(st.pages.table.shape, device=DEV)
    assert torch.equal(forward([0, B], weights), want)
    once = weights.clone()
    assert once.sum() > 0
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.forward()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        st.forward()
    for _ in range(3):
        step("replay")
        weights.zero_()
        st.logits.zero_()
        graph.replay()
        assert torch.equal(st.logits, want) and torch.equal(weights, once)
        assert torch.equal(forward(None, None), want)     # another workspace
        st.groups, st.weights = [0, B], weights
    # two sequences go on in pages of their own: what all share ends at the first page
    old = st.pages.table.clone()
    for s in (1, 3):
        st.pages.release(s)
    st.pages.reserve([1, 3], [T] * 2, [0] * 2)
    for pool in st.kcache:
        pool[st.pages.table[[1, 3], :7].flatten().long()] = pool[old[[1, 3], :7].flatten().long()]
    st.tell()
    step("replay with other tables")
    weights.zero_()
    graph.replay()
    assert torch.equal(st.logits, want) and torch.equal(weights, once)
    assert int(st._told[0, B][1][0]) == 0 and torch.equal(forward([0, B], weights), want)
