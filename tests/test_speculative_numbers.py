"""speculative_decode's use of its random numbers, with models that are tables and the kernels done by torch (this runs without a GPU)."""
import numpy as np
import pytest
import torch

from paper_2602_00182_amd import api, decode

V = 3


class Table:
    """A "model" whose logits for the next token are a row of a table; its state needs no cache."""

    def __init__(self, probabilities):
        self.logp = torch.tensor(probabilities).log()
        self.cfg = decode.ModelCfg(H=1, Hq=1, Hkv=1, D=2, F=1, V=V, n_layers=1)

    def new_state(self, B, Lmax, cos, sin):
        return State(self, B)


class State:
    def __init__(self, model, rows):
        self.model = model
        self.tokens, self.positions = torch.zeros(rows, dtype=torch.int32), torch.zeros(rows, dtype=torch.int32)
        self.logits = torch.zeros(rows, V)

    def of_rows(self, slots):
        return State(self.model, slots.shape[0])

    def forward(self, stream=None):
        self.logits = self.model.logp[self.tokens.long()]


@pytest.fixture(autouse=True)
def by_torch(monkeypatch):
    def fill(model, st, prompts, lens, stream):
        st.tokens.copy_(prompts[torch.arange(len(lens)), lens - 1])
        st.forward()

    def softmax(logits, width, out, m, s, stream=None):
        out.copy_(torch.softmax(logits, -1))

    def verify(p, q, drafts, n, u, accepted, tokens, ws=None, stream=None):
        B, N = drafts.shape
        each, wide = torch.arange(B), drafts.long()
        px = p[:, :N].gather(2, wide[..., None])[..., 0].double()
        qx = torch.ones_like(px) if q is None else q.gather(2, wide[..., None])[..., 0].double()
        count = torch.full((B,), N) if n is None else n.long()
        ok = (u[:, :N].double() * qx < px) & (torch.arange(N) < count[:, None])
        took = ok.int().cumprod(1).sum(1)
        left = p[each, took].double()
        if q is not None:
            left = left - torch.where((took < count)[:, None], q[each, took.clamp(max=N - 1)].double(), 0.0)
        left = left.clamp(min=0)
        left = torch.where(left.sum(1, keepdim=True) > 0, left, p[each, took].double())
        sums = left.cumsum(1)
        token = (sums > u[:, N, None].double() * sums[:, -1:]).int().argmax(1)
        tokens.copy_(torch.where(torch.arange(N + 1) < took[:, None], torch.cat([drafts, drafts[:, :1]], 1), -1))
        tokens[each, took] = token.int()
        accepted.copy_(took)

    monkeypatch.setattr(decode, "_fill_prompts", fill)
    monkeypatch.setattr(api, "det_softmax_f32", softmax)
    monkeypatch.setattr(api, "det_verify_drafts", verify)


@pytest.mark.parametrize("n_draft", [1, 3])
def test_numbers_from_a_stream_of_each_sequence_and_round_draw_from_the_target(n_draft):
    """Each sequence's numbers of a round are the first of a stream of its own, whatever the batch: the natural way to write `uniforms`.  Of B sequences the share that draws a token after a given one is off by
    sqrt(p (1 - p) / n) in one standard deviation, n the times that the given one was there; five of them are allowed."""
    B, n_new = 20000, 5
    target = [[0.6, 0.3, 0.1], [0.1, 0.2, 0.7], [0.3, 0.4, 0.3]]
    drafts = [[0.2, 0.5, 0.3], [0.5, 0.4, 0.1], [0.3, 0.2, 0.5]]
    prompts = torch.arange(B, dtype=torch.int32)[:, None] % V

    def uniforms(turn, shape):
        streams = np.random.default_rng([5, turn + 1]).random((B, 16), dtype=np.float32)
        return torch.from_numpy(np.ascontiguousarray(streams[:, :shape[1]]))

    cos = torch.zeros(1 + n_new + n_draft, 1)
    tokens, counts = decode.speculative_decode(Table(target), Table(drafts), prompts, torch.ones(B, dtype=torch.int32), n_new, n_draft, uniforms, cos, cos)
    assert any((c == 0).any() for c in counts) and any((c == n_draft).any() for c in counts)
    line = torch.cat([prompts, tokens], 1)
    for i in range(n_new):
        for before in range(V):
            after = line[line[:, i] == before, i + 1]
            for token in range(V):
                p = target[before][token]
                assert abs((after == token).double().mean().item() - p) <= 5 * (p * (1 - p) / len(after)) ** 0.5, (i, before, token)


def test_one_request_of_numbers_a_round():
    asked = []

    def uniforms(turn, shape):
        asked.append((turn, tuple(shape)))
        return torch.full(shape, 0.5)

    even = [[0.25, 0.5, 0.25]] * V
    cos = torch.zeros(20, 1)
    _, counts = decode.speculative_decode(Table(even), Table(even), torch.zeros((2, 1), dtype=torch.int32), torch.ones(2, dtype=torch.int32), 8, 3,
                                          uniforms, cos, cos)
    assert asked == [(-1, (2, 2))] + [(t, (2, 7)) for t in range(len(counts))]


@pytest.mark.parametrize("lens", [[0, 2], [2, -1], [3, 1]])
def test_prompts_without_a_token_and_longer_than_their_rows_are_refused(lens):
    """An empty prompt has no row whose logits its first token could be drawn from: it drew from a neighbour's."""
    model, cos = Table([[0.25, 0.5, 0.25]] * V), torch.zeros(20, 1)
    with pytest.raises(ValueError):
        decode.speculative_decode(model, model, torch.zeros((2, 2), dtype=torch.int32), torch.tensor(lens, dtype=torch.int32), 3, 1,
                                  lambda turn, shape: torch.full(shape, 0.5), cos, cos)
