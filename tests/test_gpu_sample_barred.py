"""Rows that rules on logits leave without any token: what the header says det_argmax and det_sample give there, and how a decode loop refuses them."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, step, up
from test_gpu_kv8_decode import CFG, dec, models, tables  # noqa: F401 (fixtures among them)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1, 40, 777, 32000, 32001, 65000, 128000])  # every form of the sampler
@pytest.mark.parametrize("top_k", [1, 50, 100, 1000])
def test_a_row_without_any_token(V, top_k):
    import paper_2602_00182_amd as d
    B = 4
    masks = torch.zeros((2, -(-V // 32)), dtype=torch.int32, device=DEV)
    masks[1, (V - 1) // 32] = 1 << ((V - 1) % 32) if (V - 1) % 32 < 31 else -2 ** 31   # the last token alone
    logits = torch.randn((B, V), device=DEV)
    rules = d.logits_rules(masks=masks, mask_rows=up(np.array([0, 1, 0, 1], np.int32)))
    step(f"barred rows of {V}, top-k {top_k}")
    d.det_logits_process(logits, logits, rules)
    tokens, rows = torch.full((B,), -1, dtype=torch.int32, device=DEV), torch.arange(B, dtype=torch.int32, device=DEV)
    d.det_argmax(logits, tokens)
    assert tokens.tolist() == [0, V - 1, 0, V - 1]
    last = min(top_k, V) - 1
    for seed, temperature, top_p in ((1, 1.0, 1.0), (2, 0.7, 0.9), (3, 50.0, 0.5)):
        d.det_sample(logits, temperature, top_k, top_p, seed, rows, rows + 5, tokens)
        assert tokens.tolist() == [last, V - 1, last, V - 1]


@pytest.mark.parametrize("allowed", [1, 2, 7])
def test_a_barred_token_is_never_drawn_while_there_is_another(allowed):
    """Fewer tokens than top_k are left: the barred ones among the candidates have no weight."""
    import paper_2602_00182_amd as d
    V, B, rng = 5000, 512, np.random.default_rng(allowed)
    mask = np.zeros((1, -(-V // 32)), np.uint32)
    left = rng.choice(V, allowed, replace=False)
    for t in left:
        mask[0, t // 32] |= np.uint32(1 << (int(t) % 32))
    logits = torch.randn((B, V), device=DEV) * 4
    rules = d.logits_rules(masks=up(mask.view(np.int32)), mask_rows=torch.zeros(B, dtype=torch.int32, device=DEV))
    step(f"{allowed} tokens left")
    d.det_logits_process(logits, logits, rules)
    tokens, rows = torch.full((B,), -1, dtype=torch.int32, device=DEV), torch.arange(B, dtype=torch.int32, device=DEV)
    for seed in range(4):
        for top_k, top_p in ((50, 1.0), (200, 0.95), (1000, 1.0)):
            d.det_sample(logits, 1.5, top_k, top_p, seed, rows, rows, tokens)
            assert set(tokens.tolist()) <= set(left.tolist())


def test_a_grammar_with_a_dead_end_is_refused_by_the_loop(dec, models):  # noqa: F811
    """Sampled sequences keep to a grammar to the end; one whose states the biases empty does not begin."""
    m, V = models(), CFG["V"]
    of = np.arange(V, dtype=np.int32) % 2
    bits = np.zeros((2, V), np.uint32)
    bits[0, 10:20:2], bits[1, 11:20:2] = 1, 1                 # even tokens, then odd ones, in turn
    words = (bits.reshape(2, -1, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    g = dec.Grammar(up(words.view(np.int32)), up(np.array([[1, -1], [-1, 0]], np.int32)), up(of))
    with pytest.raises(ValueError, match="state 1"):
        dec.Grammar(up(words.view(np.int32) * np.array([[1], [0]], np.int32)), g.transitions, g.token_class)
    prompts, lens, (cos, sin) = up(ds.uniform_int(8950, (3, 20), 0, V - 1)), up(np.array([20, 7, 13], np.int32)), tables(64)
    policy = dec.SamplingPolicy(1.5, 50, 0.95, 3, torch.arange(3, dtype=torch.int32, device=DEV))
    step("a grammar of few tokens, sampled")
    got, _ = dec.prefill_decode(m, prompts, lens, 20, cos, sin, policy=policy, rules=dec.LogitsPolicy(grammar=g))
    got = got.cpu().numpy()
    assert set(got[:, ::2].ravel()) <= set(range(10, 20, 2)) and set(got[:, 1::2].ravel()) <= set(range(11, 20, 2))
    with pytest.raises(ValueError, match="state 1"):
        dec.prefill_decode(m, prompts, lens, 20, cos, sin, rules=dec.LogitsPolicy(grammar=g, biases={t: float("-inf") for t in range(11, 20, 2)}))
