"""What the calls of shared prefixes, page weights and logit rules refuse, without a launch (this runs without a GPU)."""
import ctypes

import pytest
import torch

import paper_2602_00182_amd as d
from paper_2602_00182_amd._lib import Kv8Step, LayerWeights, LogitsRules

EINVAL, ESHAPE, EALIGN, EWORKSPACE = 1, 2, 3, 4
P = 4096  # a 16-byte aligned address that is never read: every call below ends before a launch


def lib():
    return d.api.lib()


SHARED = dict(q=P, pool=P, table=P, n_pages=4, n_slots=4, max_pages=2, seqlens=P, slots=0, group_rows=P, shared=P, n_groups=1, out=P, ws=P,
              ws_bytes=1 << 40, R=2, Hq=4, Hkv=2, D=128, scale=0.1, stream=0)
WEIGHTS = dict(q=P, pool=P, table=P, n_pages=4, n_slots=4, max_pages=2, seqlens=P, slots=0, group_rows=P, shared=P, n_groups=1, weights_in=P,
               weights_out=P, out=P, ws=P, ws_bytes=1 << 40, R=2, Hq=4, Hkv=2, D=128, scale=0.1, stream=0)
PICK = dict(weights=P, table=P, n_pages=4, n_slots=2, max_pages=2, lengths=P, keep=P, first=1, recent=1, dropped=P, stream=0)
ADVANCE = dict(tokens=P, history=P, ld=8, lens_in=P, lens_out=P, transitions=P, n_states=2, n_classes=3, token_class=P, V=9, states_in=P, states_out=P, B=2,
               stream=0)
POINTERS = {"q", "pool", "table", "seqlens", "slots", "group_rows", "shared", "out", "ws", "weights_in", "weights_out", "weights", "lengths", "keep", "dropped",
            "tokens", "history", "lens_in", "lens_out", "transitions", "token_class", "states_in", "states_out", "stream"}
ATTENTION = [
    (dict(q=0), EINVAL), (dict(pool=0), EINVAL), (dict(table=0), EINVAL), (dict(seqlens=0), EINVAL), (dict(out=0), EINVAL), (dict(ws=0), EINVAL),
    (dict(group_rows=0), EINVAL), (dict(shared=0), EINVAL), (dict(n_groups=-1), EINVAL), (dict(n_groups=3), ESHAPE), (dict(R=0), EINVAL),
    (dict(Hq=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(max_pages=-1), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(D=64), ESHAPE), (dict(Hq=5), ESHAPE), (dict(Hq=34), ESHAPE),
    (dict(R=5), ESHAPE), (dict(R=65536, slots=P), ESHAPE), (dict(max_pages=131073), ESHAPE), (dict(q=P + 2), EALIGN), (dict(out=P + 4), EALIGN),
    (dict(ws=P + 8), EALIGN), (dict(pool=P + 8), EALIGN), (dict(ws_bytes=0), EWORKSPACE)]
CASES = [("det_attn_decode_kv8_shared", SHARED, *c) for c in ATTENTION]
CASES += [("det_attn_decode_kv8_weights", WEIGHTS, *c) for c in ATTENTION + [(dict(weights_out=0), EINVAL), (dict(n_slots=65536), ESHAPE)]]
CASES += [("det_kv8_pick_pages", PICK, change, code) for change, code in [
    (dict(weights=0), EINVAL), (dict(table=0), EINVAL), (dict(lengths=0), EINVAL), (dict(keep=0), EINVAL), (dict(dropped=0), EINVAL),
    (dict(n_pages=0), EINVAL), (dict(n_slots=0), EINVAL), (dict(max_pages=0), EINVAL), (dict(first=-1), EINVAL), (dict(recent=-1), EINVAL),
    (dict(max_pages=131073), ESHAPE)]]
CASES += [("det_logits_advance", ADVANCE, change, code) for change, code in [
    (dict(tokens=0), EINVAL), (dict(B=0), EINVAL), (dict(history=0, transitions=0), EINVAL), (dict(lens_in=0), EINVAL), (dict(lens_out=0), EINVAL),
    (dict(ld=0), EINVAL), (dict(states_in=0), EINVAL), (dict(states_out=0), EINVAL), (dict(n_states=0), EINVAL), (dict(n_classes=0), EINVAL),
    (dict(V=0), EINVAL), (dict(token_class=0), EINVAL)]]


@pytest.mark.parametrize("name,args,change,code", CASES, ids=lambda x: str(x) if isinstance(x, dict) and len(x) <= 2 else "")
def test_a_call_that_is_refused_says_why(name, args, change, code):
    call = {**args, **change}
    assert getattr(lib(), name)(*[None if isinstance(v, int) and v == 0 and k in POINTERS else v for k, v in call.items()]) == code


LAYER = dict(x=P, pool=P, table=P, n_pages=4, n_slots=4, max_pages=2, positions=P, slots=None, cos=P, sin=P, step={}, ws=P, ws_bytes=1 << 40, R=2)


@pytest.mark.parametrize("name", ["det_decoder_layer_kv8_step", "det_qdecoder_layer_kv8_step"])
@pytest.mark.parametrize("change,code", [
    (dict(step=dict(group_rows=0)), EINVAL), (dict(step=dict(shared=0)), EINVAL), (dict(step=dict(n_groups=-1)), EINVAL), (dict(step=dict(n_groups=3)), ESHAPE),
    (dict(R=65536, slots=P), ESHAPE), (dict(step=dict(weights=P), n_slots=65536), ESHAPE), (dict(step=dict(n_groups=0, weights=P), R=65536, slots=P), ESHAPE),
    (dict(ws_bytes="size - 1"), EWORKSPACE), (dict(step=dict(weights=P), max_pages=200, ws_bytes="size"), EWORKSPACE), (dict(R=5), ESHAPE), (dict(x=None), EINVAL),
    (dict(pool=P + 8), EALIGN), (dict(ws=P + 8), EALIGN)])
def test_a_layers_step_that_is_refused_says_why(name, change, code):
    a = {**LAYER, **change}
    cfg, w = d.layer_cfg(512, 4, 2, 128, 1024, 256, 1e-5, 0.1), LayerWeights(*[P] * 6)
    step = Kv8Step(**{**dict(group_rows=P, shared=P, n_groups=1), **a["step"]})
    size = getattr(d, name + "_workspace_bytes")(cfg, a["R"], a["max_pages"], False)
    n_bytes = {"size - 1": size - 1, "size": size}.get(a["ws_bytes"], a["ws_bytes"])
    call = [a[k] for k in ("x", "pool", "table", "n_pages", "n_slots", "max_pages", "positions", "slots", "cos", "sin")]
    assert getattr(lib(), name)(ctypes.byref(w), ctypes.byref(cfg), *call, ctypes.byref(step), a["ws"], n_bytes, a["R"], None) == code


def test_a_layers_workspace():
    cfg = d.layer_cfg(512, 4, 2, 128, 1024, 256, 1e-5, 0.1)
    for name in ("det_decoder_layer_kv8", "det_qdecoder_layer_kv8"):
        size = lambda weights, R=3, pages=9: getattr(d, name + "_step_workspace_bytes")(cfg, R, pages, weights)  # noqa: E731, B023
        assert getattr(d, name + "_workspace_bytes")(cfg, 3, 9) == size(False) < size(True) and size(False, 0) == size(True, 3, 0) == size(True, 3, 131073) == 0


FULL = dict(penalties=P, history=P, history_lens=P, bias_begin=P, bias_tokens=P, bias_values=P, masks=P, mask_rows=P, ld_history=10, n_history=2, n_biases=3,
            n_masks=1, mask_words=4)


@pytest.mark.parametrize("change,rules,code", [
    (dict(logits=0), {}, EINVAL), (dict(out=0), {}, EINVAL), (dict(rules=None), {}, EINVAL), (dict(B=0), {}, EINVAL), (dict(V=0), {}, EINVAL),
    (dict(ld_in=99), {}, EINVAL), (dict(ld_out=99), {}, EINVAL), (dict(dtype=2), {}, EINVAL), ({}, dict(history=0), EINVAL),
    ({}, dict(history_lens=0), EINVAL), ({}, dict(ld_history=0), EINVAL), ({}, dict(n_history=0), EINVAL), ({}, dict(n_history=1), EINVAL),
    ({}, dict(ld_history=(1 << 30) + 1), ESHAPE), ({}, dict(n_biases=(1 << 30) + 1), ESHAPE), ({}, dict(bias_tokens=0), EINVAL), ({}, dict(bias_values=0), EINVAL), ({}, dict(n_biases=-1), EINVAL), ({}, dict(n_masks=0), EINVAL),
    ({}, dict(mask_words=0), EINVAL), ({}, dict(mask_words=3), ESHAPE), (dict(B=65536), dict(n_history=70000), ESHAPE),
    (dict(V=(1 << 30) + 1, ld_in=1 << 31, ld_out=1 << 31), dict(masks=0), ESHAPE), (dict(logits=P + 4), {}, EALIGN), (dict(out=P + 8), {}, EALIGN),
    (dict(out=P, ld_out=101), {}, EINVAL),      # in place with another stride
    (dict(out=P + 16), {}, EINVAL), (dict(out=P + 784), {}, EINVAL), (dict(logits=P + 784, out=P), {}, EINVAL)])  # rows that overlap
def test_rules_that_are_refused(change, rules, code):
    call = {**dict(logits=P, ld_in=100, out=1 << 40, ld_out=100, dtype=1, B=2, V=100), **change}
    r = LogitsRules()
    for k, v in {**FULL, **rules}.items():
        setattr(r, k, v or None if k in FULL and FULL[k] == P else v)
    given = call.pop("rules", r)
    assert lib().det_logits_process(*[v or None if k in ("logits", "out") else v for k, v in call.items()],
                                    None if given is None else ctypes.byref(given), None) == code


def test_sizes():
    assert d.det_attn_decode_kv8_shared_workspace_bytes(3, 32, 8, 128, 9) == d.det_attn_decode_kv8_workspace_bytes(3, 32, 8, 128, 9)
    assert d.det_attn_decode_kv8_weights_workspace_bytes(3, 32, 8, 128, 9) == 3 * 32 * 3 * (132 + 4) * 4
    for of in (d.det_attn_decode_kv8_shared_workspace_bytes, d.det_attn_decode_kv8_weights_workspace_bytes):
        assert of(1, 32, 8, 64, 4) == 0 and of(1, 32, 7, 128, 4) == 0 and of(1, 34, 2, 128, 4) == 0 and of(1, 32, 8, 128, 131073) == 0 and of(0, 32, 8, 128, 4) == 0
        assert of(65535, 128, 8, 128, 131072) > 1 << 40  # no 32-bit product


def test_the_binding_refuses_what_does_not_fit():
    pool, table = d.kv8_pool(1, 4, 2, device="cpu")[0], torch.zeros((3, 2), dtype=torch.int32)
    bf, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    q, out, lens = torch.zeros((3, 4, 128), **bf), torch.zeros((3, 4, 128), **bf), torch.zeros(3, **i32)
    ws, rows, shared = torch.zeros(64, dtype=torch.uint8), torch.zeros(2, **i32), torch.zeros(1, **i32)
    weights = torch.zeros(3, 2)
    for bad in [dict(rows=rows[:1]), dict(lens=lens[:2]), dict(out=out[:2]), dict(table=table[:2]), dict(slots=lens[:2]), {}]:  # {}: host tensors
        a = {**dict(q=q, pool=pool, table=table, lens=lens, slots=None, rows=rows, shared=shared, out=out), **bad}
        with pytest.raises(ValueError):
            d.det_attn_decode_kv8_shared(a["q"], a["pool"], a["table"], a["lens"], a["slots"], a["rows"], a["shared"], a["out"], ws, 0.1)
        with pytest.raises(ValueError):
            d.det_attn_decode_kv8_weights(a["q"], a["pool"], a["table"], a["lens"], a["slots"], a["rows"], a["shared"], None, weights, a["out"], ws, 0.1)
    for given in [(weights[:2], weights), (None, weights[:, :1])]:
        with pytest.raises(ValueError):
            d.det_attn_decode_kv8_weights(q, pool, table, lens, None, None, None, *given, out, ws, 0.1)
    drop = torch.zeros((3, 2), dtype=torch.uint8)
    for bad in [dict(w=weights[:2]), dict(n=lens[:2]), dict(k=lens[:2]), dict(o=drop[:, :1]), {}]:
        a = {**dict(w=weights, n=lens, k=lens, o=drop), **bad}
        with pytest.raises(ValueError):
            d.det_kv8_pick_pages(a["w"], table, 4, a["n"], a["k"], 1, 1, a["o"])
    with pytest.raises(ValueError):
        d.logits_rules(penalties=torch.ones(2, 3))                                                     # no history
    with pytest.raises(ValueError):
        d.logits_rules(bias_begin=torch.zeros(3, **i32), bias_tokens=torch.zeros(2, **i32), bias_values=torch.zeros(1))
    with pytest.raises(ValueError):
        d.logits_rules(masks=torch.zeros(4, **i32))
    with pytest.raises(ValueError):
        d.logits_rules(masks=torch.zeros((2, 4), **i32))                                               # host tensors
    with pytest.raises(ValueError):
        d.det_logits_process(torch.zeros(2, 9), torch.zeros(2, 8), d.logits_rules())
    with pytest.raises(ValueError):
        d.det_logits_process(torch.zeros(2, 9), torch.zeros(2, 9), d.logits_rules())                     # host tensors
    with pytest.raises(ValueError):
        d.det_logits_advance(lens, torch.zeros((2, 5), **i32), lens, lens)
    with pytest.raises(ValueError):
        d.det_logits_advance(lens, None, None, None, torch.zeros((2, 5), **i32), None, lens[:1], lens)
