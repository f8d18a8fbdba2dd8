"""speculative_decode against a plain replay: every round's probabilities from a fresh pass over the tokens kept so far, the choices by the plain
verification in extended precision.  Tokens and accepted counts have to be equal, through rejections and full acceptances."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, step, up
from test_gpu_kv8_decode import CFG, SIZES, numbers, tables, weights
from test_gpu_verify import plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantized,n_draft,spread", [(False, 1, 0.05), (False, 3, 0.02), (True, 4, 0.02)])
def test_rounds_replayed_from_the_kept_tokens(quantized, n_draft, spread):
    import paper_2602_00182_amd as d
    from paper_2602_00182_amd import decode as dec

    # the draft model: the model's weights and some noise on its head, so that some of its drafts are taken
    w = weights(8800, n_layers=2, **SIZES)
    near = dict(w, lm_head=(w["lm_head"].float() + ds.normal_bf16_torch(8890, tuple(w["lm_head"].shape), spread, 0.0, DEV).float()).to(torch.bfloat16))
    cfg = dec.ModelCfg(**CFG)
    model = dec.DecodeModel(cfg, w, quantized=quantized, cache8=True)
    draft = dec.DecodeModel(cfg, near, cache8=True)
    lens = np.array([61, 9], dtype=np.int32)
    prompts = ds.uniform_int(8801, (2, 61), 0, CFG["V"] - 1)
    n_new, V = 16, CFG["V"]
    cos, sin = tables(61 + n_new + n_draft)
    step(f"drafts of {n_draft}, quantized {quantized}")
    tokens, counts = dec.speculative_decode(model, draft, up(prompts), up(lens), n_new, n_draft, numbers(3, [0, 1]), cos, sin)
    taken = torch.stack(counts)
    assert (taken < n_draft).any() and (taken > 0).any()

    def probabilities(m, text):
        _, logits = dec.prefill_decode(m, up(np.array([text], np.int32)), up(np.array([len(text)], np.int32)), 1, cos, sin, keep_logits=True)
        out, sums = torch.empty_like(logits[0]), torch.empty((2, 1), device=DEV)
        d.det_softmax_f32(logits[0], up(np.array([V], np.int32)), out, sums[0], sums[1])
        return out.cpu().numpy()[0]

    def pick(p, u):
        return int(plain(p[None, None].repeat(2, 1), None, np.zeros((1, 1), np.int32), [0], np.array([[0, u]], np.float32))[1][0, 0])

    for b in range(2):
        give = numbers(3, [b])
        text = prompts[b, :lens[b]].tolist()
        made = [pick(probabilities(model, text), give(-1, (1, 2)).cpu().numpy()[0, 1])]
        turn = 0
        while len(made) < n_new:
            u = give(turn, (1, 2 * n_draft + 1)).cpu().numpy()[0]
            kept, q = text + made, []
            for i in range(n_draft):
                q.append(probabilities(draft, kept))
                kept = kept + [pick(q[-1], u[i])]
            first = len(text) + len(made)
            p = np.stack([probabilities(model, kept[:first + i]) for i in range(n_draft + 1)])
            took, new = plain(p[None], np.stack(q)[None], np.array([kept[first:]], np.int32), [n_draft], u[None, n_draft:])
            assert took[0] == int(counts[turn][b]), (b, turn)
            made += new[0, :took[0] + 1].tolist()
            turn += 1
        assert made[:n_new] == tokens[b].tolist(), b
