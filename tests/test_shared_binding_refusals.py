"""Arguments that belong together, of which a caller gives one: refused by the bindings with a ValueError, other types of logits with a TypeError (this runs
without a GPU)."""
import pytest
import torch

import paper_2602_00182_amd as d

I32 = dict(dtype=torch.int32)


def test_groups_are_first_rows_and_what_they_share():
    rows, shared = torch.zeros(2, **I32), torch.zeros(1, **I32)
    pool, table = d.kv8_pool(1, 4, 2, device="cpu")[0], torch.zeros((3, 2), **I32)
    q, lens, ws = torch.zeros((3, 4, 128), dtype=torch.bfloat16), torch.zeros(3, **I32), torch.zeros(64, dtype=torch.uint8)
    for given in ((rows, None), (None, shared), (rows, shared[0]), (rows, torch.zeros((1, 1), **I32)), (rows[:1], shared)):
        with pytest.raises(ValueError):
            d.kv8_step(*given)
        with pytest.raises(ValueError):
            d.det_attn_decode_kv8_weights(q, pool, table, lens, None, *given, None, torch.zeros(3, 2), q.clone(), ws, 0.1)
        with pytest.raises(ValueError):
            d.det_attn_decode_kv8_shared(q, pool, table, lens, None, *given, q.clone(), ws, 0.1)


def test_a_history_and_a_state_machine_are_whole():
    tokens, history, to = torch.zeros(3, **I32), torch.zeros((3, 5), **I32), torch.zeros((2, 4), **I32)
    for given in ((history, None, tokens), (history, tokens, None), (None, None, None, to, None, None, tokens), (None, None, None, to, None, tokens, None)):
        with pytest.raises(ValueError):
            d.det_logits_advance(tokens, *given)


def test_rules_of_one_value_a_row():
    with pytest.raises(ValueError):
        d.logits_rules(masks=torch.zeros((2, 4), **I32), mask_rows=torch.tensor(1, **I32))
    with pytest.raises(ValueError):
        d.logits_rules(bias_begin=torch.tensor(1, **I32), bias_tokens=torch.zeros(0, **I32), bias_values=torch.zeros(0))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32])
def test_other_types_of_logits(dtype):
    z = torch.zeros((2, 9), dtype=dtype)
    with pytest.raises(TypeError):
        d.det_logits_process(z, z, d.logits_rules())
