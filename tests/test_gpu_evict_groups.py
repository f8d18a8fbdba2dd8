"""Continuations that give up pages of their own choice: a step reads in groups only while these share whole chunks worth it."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import step, up
from test_gpu_kv8_decode import CFG, dec, models, tables  # noqa: F401 (fixtures among them)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups_from", [1, 2000])
def test_groups_end_with_what_they_share(dec, models, monkeypatch, groups_from):  # noqa: F811
    m, samples, n_new = models(), 3, 50
    lens = np.array([700, 90, 520], dtype=np.int32)
    prompts, (cos, sin) = up(ds.uniform_int(9100, (3, 700), 0, CFG["V"] - 1)), tables(800)
    policy = dec.SamplingPolicy(1.0, 50, 0.95, 7, torch.arange(9, dtype=torch.int32, device=prompts.device))
    run = lambda **more: dec.prefill_decode(m, prompts, up(lens), n_new, cos, sin, samples=samples, policy=policy, keep_logits=True, **more)  # noqa: E731
    evict = dec.EvictPolicy(keep=7, every=12, first=1, recent=2)
    monkeypatch.setattr(dec, "GROUPS_FROM", 10 ** 9)
    step("each for itself")
    want, logits = run(evict=evict)
    monkeypatch.setattr(dec, "GROUPS_FROM", groups_from)
    told, original = [], dec.DecodeState.tell

    def spy(self, stream=None):
        out = original(self, stream)
        if self.weights is not None:
            g = self.groups
            told.append(None if g is None else [self.pages.shared_tokens(range(a, b)) // 256 * 256 for a, b in zip(g, g[1:])])
        return out
    monkeypatch.setattr(dec.DecodeState, "tell", spy)
    step("in groups")
    got, some = run(evict=evict)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(some, logits))
    assert len(told) == n_new - 1 and told[0] == [512, 0, 512]
    print(told[::6])
    for j, shared in enumerate(told, 1):
        if shared is None:
            assert all(x is None for x in told[j:])      # what is shared only becomes less
            break
        saved = (samples - 1) * sum(shared)
        assert saved * CFG["Hkv"] >= groups_from and 2 * saved >= samples * (int(lens.sum()) - sum(shared)) + j * 9
    assert told[-1] is None and told[-1 - n_new // 2] is None
