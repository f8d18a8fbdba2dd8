"""The pool behind several continuations of a prompt: its full pages once, the rest for each (this runs without a GPU)."""
import pytest
import torch

import paper_2602_00182_amd as d
from paper_2602_00182_amd import api, decode


@pytest.mark.parametrize("lens", [[1], [64], [100, 64, 9], [63, 65, 128, 300]])
@pytest.mark.parametrize("samples,n_new", [(2, 1), (4, 40), (3, 200)])
def test_the_pool_holds_what_the_run_takes_and_no_more(monkeypatch, lens, samples, n_new):
    """The run's own bookkeeping with the kernels left out: no page is missing, and in the end none is free."""
    made = []

    class State:
        def __init__(self, model, B, Lmax, cos, sin, reserve=True, n_pages=None):
            each = -(-Lmax // 64)
            self.pages = d.KVPages(1, B * each if n_pages is None else n_pages, 1, B, each, device="cpu")
            self.kcache, self.vcache, self.lcfg = [], [], None
            self.rope_cos, self.rope_sin = cos, sin
            self.x, self.logits = torch.zeros(B, 1), torch.zeros(B, 3)
            self.positions, self.tokens = torch.zeros(B, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
            made.append(self)

        head = forward = lambda self, stream=None: None

    class Model:
        cache8, layers, embed = True, [], torch.zeros(5, 1, dtype=torch.bfloat16)
        cfg = decode.ModelCfg(H=1, Hq=1, Hkv=1, D=128, F=1, V=3, n_layers=1)
        layer_workspace_bytes = lambda self, lcfg, rows, named=False: 16

        def new_state(self, *args, **more):
            return State(self, *args, **more)

    for name in ("det_embed_gather", "det_argmax", "det_decode_advance"):
        monkeypatch.setattr(api, name, lambda *args: None)
    monkeypatch.setattr(api, "det_kv8_copy_pages", lambda *args: None)
    T = max(lens) + n_new - 1
    prompts = torch.zeros((len(lens), max(lens)), dtype=torch.int32)
    decode.prefill_decode(Model(), prompts, torch.tensor(lens, dtype=torch.int32), n_new, torch.zeros(T, 64), torch.zeros(T, 64), samples=samples)
    pages, each = made[0].pages, -(-T // 64)
    assert pages.pool.shape[1] == sum(n // 64 + samples * (each - n // 64) for n in lens) <= len(lens) * samples * each
    for b, n in enumerate(lens):
        held = [pages.pages(b * samples + i) for i in range(samples)]
        assert all(len(h) == each and h[:n // 64] == held[0][:n // 64] for h in held)
        assert len({p for h in held for p in h[n // 64:]}) == samples * (each - n // 64)
    assert pages.free_pages == 0
