"""Penalties, biases and masks on logits, and the bookkeeping behind them, against a plain implementation in fp64 and the exact fp32 steps."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, step, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    import paper_2602_00182_amd as d
    return d


def rules_of(rng, B, V, T, penalties=True, biases=6, masks=3, rows=None):
    """Host arrays of a call with everything in it: ids outside the vocabulary, repeated tokens and biases, rows without history, masks that allow nothing."""
    h = {}
    n = B if rows is None else rows
    if penalties:
        h["history"] = np.where(rng.random((n, T)) < 0.1, rng.integers(-5, V + 5, (n, T)), (rng.random((n, T)) ** 4 * V).astype(np.int64)).astype(np.int32)
        h["history_lens"] = rng.integers(0, T + 1, B).astype(np.int32)
        h["history_lens"][0], h["history_lens"][-1] = T, max(0, T // 2)
        h["generated_from"] = rng.integers(0, T + 1, B).astype(np.int32)
        h["penalties"] = np.stack([1 + rng.random(B), rng.normal(0, 0.5, B), rng.normal(0, 0.7, B)], 1).astype(np.float32)
        if rows is not None:
            h["history_rows"] = rng.integers(-1, n + 1, B).astype(np.int32)
    if biases:
        counts = rng.integers(0, biases + 1, B)
        h["bias_begin"] = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        total = int(counts.sum())
        h["bias_tokens"] = rng.integers(-1, V + 1, total).astype(np.int32)
        h["bias_tokens"][total // 2:] = h["bias_tokens"][:total - total // 2]  # some tokens twice
        h["bias_values"] = rng.normal(0, 3, total).astype(np.float32)
    if masks:
        words = -(-V // 32) + 1
        bits = rng.integers(0, 2 ** 32, (masks, words), dtype=np.uint32)
        bits[0] = 0
        h["masks"] = bits.view(np.int32)
        h["mask_rows"] = rng.integers(-1, masks + 1, B).astype(np.int32)
    return h


def plain(z, h, dtype):
    """The written steps on z [B, V] in `dtype`."""
    z = z.astype(dtype).copy()
    B, V = z.shape
    n_allowed = np.ones((B, V), bool)
    touched = np.zeros((B, V), bool)
    for b in range(B):
        if "penalties" in h:
            rep, freq, pres = h["penalties"][b].astype(dtype)
            row = h["history_rows"][b] if "history_rows" in h else b
            if 0 <= row < len(h["history"]):
                ids = h["history"][row, :min(h["history_lens"][b], h["history"].shape[1])]
                keep = (ids >= 0) & (ids < V)
                made = np.bincount(ids[keep & (np.arange(len(ids)) >= h["generated_from"][b])], minlength=V)
                seen = np.zeros(V, bool)
                seen[ids[keep]] = True
                z[b, seen] = np.where(z[b, seen] > 0, z[b, seen] / rep, z[b, seen] * rep)
                on = made > 0
                z[b, on] = (z[b, on] - freq * made[on].astype(dtype)) - pres
                touched[b] |= seen
        if "bias_begin" in h:
            last = {}
            for i in range(h["bias_begin"][b], h["bias_begin"][b + 1]):
                last[int(h["bias_tokens"][i])] = h["bias_values"][i].astype(dtype)
            for t, v in last.items():
                if 0 <= t < V:
                    z[b, t] = z[b, t] + v
                    touched[b, t] = True
        if "masks" in h:
            m = h["mask_rows"][b]
            if 0 <= m < len(h["masks"]):
                t = np.arange(V)
                n_allowed[b] = (h["masks"][m].view(np.uint32)[t // 32] >> (t % 32).astype(np.uint32)) & 1 != 0
    z[~n_allowed] = -np.inf
    return z, touched & n_allowed


def run(d, z, h, out=None, stream=None):
    keep = {k: up(v) for k, v in h.items()}
    rules = d.logits_rules(**keep)
    out = torch.full_like(z, 77.0) if out is None else out
    d.det_logits_process(z, out, rules, stream)
    return out


SIZES = [(1, 1, 1), (1, 31, 5), (2, 33, 9), (3, 1023, 40), (5, 1025, 300), (4, 4097, 50), (1, 32000, 200), (7, 32001, 700), (64, 8190, 33), (66, 32003, 300), (2, 128000, 4001)]


@pytest.mark.parametrize("B,V,T", SIZES)
@pytest.mark.parametrize("parts", ["all", "penalties", "biases", "masks", "none"])
def test_fp32_logits_bit_for_bit(d, B, V, T, parts):
    rng = np.random.default_rng(B * 1000 + V)
    on = lambda w: parts in ("all", w)
    h = rules_of(rng, B, V, T, on("penalties"), 6 * on("biases"), 3 * on("masks"))
    z = rng.normal(0, 3, (B, V)).astype(np.float32)
    z.ravel()[::7] = 0.0
    z.ravel()[3::11] = -0.0
    step(f"{B} rows of {V}, {parts}")
    got = run(d, up(z), h).cpu().numpy()
    want, _ = plain(z, h, np.float32)
    assert np.array_equal(got.view(np.int32), want.view(np.int32))
    exact, _ = plain(z, h, np.float64)
    fine = np.isfinite(exact)
    assert np.array_equal(fine, np.isfinite(got))
    # up to five roundings (the quotient, frequency * count, two subtractions, the bias), each 2^-24 of the largest number that enters
    most = np.abs(exact[fine]).max(initial=0) + np.abs(z).max() * 2 + 0.5 * 6 * T + 20
    assert np.abs(got[fine] - exact[fine]).max(initial=0) <= 5 * 2.0 ** -24 * most


@pytest.mark.parametrize("B,V,T", SIZES)
def test_bf16_logits(d, B, V, T):
    """The fp32 steps, rounded once; what no rule reaches keeps its bits."""
    rng = np.random.default_rng(B * 1000 + V + 1)
    h = rules_of(rng, B, V, T)
    bits = ds.f32_to_bf16_bits(rng.normal(0, 3, (B, V)).astype(np.float32))
    bits.ravel()[::13] = 0x7FA1  # a NaN with a payload
    step(f"bf16 {B} rows of {V}")
    z = ds.to_torch_bf16(bits, DEV)
    got = ds.from_torch_bf16(run(d, z, h))
    with np.errstate(invalid="ignore"):
        want, touched = plain(ds.bf16_bits_to_f32(bits), h, np.float32)
    rounded = np.where(np.isnan(want), np.uint16(0x7FC0), ds.f32_to_bf16_bits(want))  # the library's rounding; the helper is for numbers
    expect = np.where(touched, rounded, np.where(np.isneginf(want), np.uint16(0xFF80), bits))
    assert np.array_equal(got, expect)


def test_rows_that_name_histories_strides_and_in_place(d):
    rng = np.random.default_rng(9)
    B, V, T = 12, 5003, 120
    h = rules_of(rng, B, V, T, rows=4)
    z = rng.normal(0, 3, (B, V)).astype(np.float32)
    want, _ = plain(z, h, np.float32)
    wide = torch.full((B, V + 37), 5.0, device=DEV)
    wide[:, :V] = up(z)
    step("strided rows")
    out = torch.full((B, V + 9), 6.0, device=DEV)
    run(d, wide[:, :V], h, out[:, :V])
    assert np.array_equal(out[:, :V].cpu().numpy(), want) and (out[:, V:] == 6).all() and (wide[:, V:] == 5).all()
    step("in place")
    run(d, wide[:, :V], h, wide[:, :V])
    assert np.array_equal(wide[:, :V].cpu().numpy(), want) and (wide[:, V:] == 5).all()


def test_what_is_not_finite(d):
    V = 100
    z = np.zeros((1, V), np.float32)
    z[0, :6] = [np.nan, np.inf, -np.inf, 3e38, -3e38, 1e-42]
    h = dict(history=np.array([[0, 1, 2, 3, 4, 5, 5]], np.int32), history_lens=np.array([7], np.int32), generated_from=np.array([0], np.int32),
             penalties=np.array([[1.5, 0.25, 0.5]], np.float32))
    step("not finite")
    got = run(d, up(z), h).cpu().numpy()
    with np.errstate(all="ignore"):
        want, _ = plain(z, h, np.float32)
    assert np.isnan(got[0, 0]) and np.array_equal(got[0, 1:], want[0, 1:]) and got[0, 4] == -np.inf


def test_a_row_does_not_depend_on_its_batch(d):
    rng = np.random.default_rng(21)
    B, V, T = 70, 32001, 100
    h = rules_of(rng, B, V, T)
    z = rng.normal(0, 3, (B, V)).astype(np.float32)
    step("70 rows")
    all_rows = run(d, up(z), h)
    for b in (0, 33, 69):
        one = {k: v[b:b + 1] for k, v in h.items() if k in ("history", "history_lens", "generated_from", "penalties", "mask_rows")}
        one["masks"], one["bias_tokens"], one["bias_values"] = h["masks"], h["bias_tokens"], h["bias_values"]
        one["bias_begin"] = h["bias_begin"][b:b + 2]
        step(f"row {b} alone")
        assert torch.equal(run(d, up(z[b:b + 1]), one)[0], all_rows[b])


def test_a_masked_row_and_the_choice_of_a_token(d):
    """A mask that allows one token, and one that allows none: det_argmax gives that token, and 0."""
    V = 777
    z = torch.randn((2, V), device=DEV)
    masks = np.zeros((2, -(-V // 32)), np.uint32)
    masks[0, 500 // 32] = 1 << (500 % 32)
    out = run(d, z, dict(masks=masks.view(np.int32), mask_rows=np.array([0, 1], np.int32)))
    tokens = torch.full((2,), -1, dtype=torch.int32, device=DEV)
    step("argmax of masked rows")
    d.det_argmax(out, tokens)
    assert tokens.tolist() == [500, 0] and torch.isneginf(out[1]).all()


def test_the_bookkeeping_of_a_step(d):
    B, most, n_states, classes, V = 300, 6, 5, 4, 50
    rng = np.random.default_rng(31)
    tokens = rng.integers(-2, V + 2, B).astype(np.int32)
    history = rng.integers(0, V, (B, most)).astype(np.int32)
    lens = rng.integers(-1, most + 2, B).astype(np.int32)
    transitions = rng.integers(-1, n_states + 1, (n_states, classes)).astype(np.int32)
    of = rng.integers(-1, classes + 1, V).astype(np.int32)
    states = rng.integers(-2, n_states + 2, B).astype(np.int32)

    def want(of, V):
        h, n, s = history.copy(), np.maximum(lens, 0), np.full(B, -1, np.int32)
        for b in range(B):
            if n[b] < most:
                h[b, n[b]] = tokens[b]
                n[b] += 1
            if 0 <= states[b] < n_states and 0 <= tokens[b] < V:
                c = tokens[b] if of is None else of[tokens[b]]
                if 0 <= c < classes:
                    s[b] = transitions[states[b], c]
            if not 0 <= s[b] < n_states:
                s[b] = -1
        return h, n, s

    for classes_of in (of, None):
        h, n, s = want(classes_of, V if classes_of is not None else classes)
        dh, dn, dt = up(history), up(lens), up(states)
        new_n, new_s = torch.empty_like(dn), torch.empty_like(dt)
        step("advance")
        d.det_logits_advance(up(tokens), dh, dn, new_n, up(transitions), None if classes_of is None else up(classes_of), dt, new_s)
        assert np.array_equal(dh.cpu().numpy(), h) and np.array_equal(new_n.cpu().numpy(), n) and np.array_equal(new_s.cpu().numpy(), s)
        dh = up(history)
        d.det_logits_advance(up(tokens), dh, dn, dn, up(transitions), None if classes_of is None else up(classes_of), dt, dt)  # in place
        assert np.array_equal(dh.cpu().numpy(), h) and np.array_equal(dn.cpu().numpy(), n) and np.array_equal(dt.cpu().numpy(), s)
        only = torch.empty_like(dt)
        d.det_logits_advance(up(tokens), None, None, None, up(transitions), None if classes_of is None else up(classes_of), up(states), only)
        assert np.array_equal(only.cpu().numpy(), s)


def test_graphs_and_streams(d):
    """A captured step of bookkeeping and rules, replayed while the history grows: every replay is the eager one."""
    rng = np.random.default_rng(41)
    B, V, T = 6, 4001, 40
    z = up(rng.normal(0, 3, (B, V)).astype(np.float32))
    h = rules_of(rng, B, V, T)
    keep = {k: up(v) for k, v in h.items()}
    keep["history_lens"].fill_(3)
    tokens, out = torch.zeros(B, dtype=torch.int32, device=DEV), torch.empty_like(z)
    rules = d.logits_rules(**keep)

    def both():
        d.det_logits_advance(tokens, keep["history"], keep["history_lens"], keep["history_lens"])
        d.det_logits_process(z, out, rules)
    start = {k: v.clone() for k, v in keep.items()}
    results = []
    for mode in ("eager", "graph"):
        for k, v in start.items():
            keep[k].copy_(v)
        side, got = torch.cuda.Stream(), []
        if mode == "graph":
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                both()
            torch.cuda.synchronize()
        for i in range(5):
            step(f"{mode} {i}")
            tokens.copy_(torch.arange(B, device=DEV, dtype=torch.int32) * 7 + i // 2)
            out.zero_()
            both() if mode == "eager" else graph.replay()
            torch.cuda.synchronize()
            got.append(out.clone())
        results.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*results)) and not torch.equal(results[0][0], results[0][4])
