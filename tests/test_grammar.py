"""A grammar says when it is made that a sequence could come to a state in which no token is left (host integers; this runs without a GPU)."""
import math
import random

import pytest
import torch

from paper_2602_00182_amd import decode as dec


def masks(V, *allowed):
    out = torch.zeros((len(allowed), -(-V // 32)), dtype=torch.int64)
    for s, tokens in enumerate(allowed):
        for t in tokens:
            out[s, t // 32] |= 1 << (t % 32)
    return torch.where(out >= 2 ** 31, out - 2 ** 32, out).to(torch.int32)


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def test_a_state_without_tokens_that_can_be_reached_is_refused():
    V, of = 70, ints([t % 3 for t in range(70)])
    to = [[1, 0, 2], [0, 1, 1], [-1, -1, -1]]
    dec.Grammar(masks(V, [0, 3, 69], [1, 2], [5]), ints(to), of)
    with pytest.raises(ValueError, match="state 2"):
        dec.Grammar(masks(V, [0, 2], [1], []), ints(to), of)              # token 2 leads there
    with pytest.raises(ValueError, match="state 0"):
        dec.Grammar(masks(V, [], [1], [2]), ints(to), of)
    with pytest.raises(ValueError, match="state 2"):
        dec.Grammar(masks(V, [0], [1], []), ints(to), of, start=2)
    with pytest.raises(ValueError, match="state 2"):                       # over another state, by the last token of all
        dec.Grammar(masks(V, [0], [68], []), ints([[1, -1, -1], [-1, -1, 2], [0, 0, 0]]), of)


def test_a_state_without_tokens_that_nothing_leads_to_is_none_of_it():
    V, of = 70, ints([t % 3 for t in range(70)])
    dec.Grammar(masks(V, [0, 1], [1], []), ints([[1, 0, 2], [0, 1, 2], [2, 2, 2]]), of)   # only class 2, which is barred, leads there
    dec.Grammar(masks(4, [0, 1], [3], []), ints([[1, -1, 2, 2], [2, 2, 2, 0], [2, 2, 2, 2]]))  # every token its own class


def test_tokens_without_a_class_and_states_that_are_none_end_the_grammar():
    dec.Grammar(masks(3, [0, 1, 2], []), ints([[-1, 7], [0, 0]]), ints([0, 1, 9]))


def test_shapes():
    to, of = ints([[0, 0], [1, 1]]), ints([0, 1, 1])
    for m, t, c, start in ((masks(3, [0]), to, of, 0), (masks(3, [0], [1])[0], to, of, 0), (masks(3, [0], [1]), to[0], of, 0), (masks(3, [0], [1]), to, of, 2),
                           (masks(3, [0], [1]), to, of, -1), (masks(3, [0], [1]), to, ints([0] * 33), 0), (masks(3, [0], [1]), to, ints([[0, 1, 1]]), 0)):
        with pytest.raises(ValueError):
            dec.Grammar(m, t, c, start)


def test_what_biases_bar_and_a_smaller_vocabulary():
    V, of = 70, ints([t % 3 for t in range(70)])
    g = dec.Grammar(masks(V, [0, 3, 69], [1, 4], [5]), ints([[1, 0, 2], [0, 1, 1], [-1, -1, -1]]), of)
    prompts, lens = torch.zeros((2, 4), dtype=torch.int32), torch.tensor([4, 2])
    rules = lambda biases, V=V: dec._Rules(dec.LogitsPolicy(biases=biases, grammar=g), prompts, lens, 8, V, None)  # noqa: E731
    with pytest.raises(ValueError, match="state 1"):
        rules({1: -math.inf, 4: -math.inf})
    with pytest.raises(ValueError, match="state 1"):
        rules({1: -1e39, 4: -math.inf, 200: 1.0})                            # -inf in fp32
    with pytest.raises(ValueError, match="state 1"):
        rules({}, 1)
    for biases in ({1: -math.inf, 4: -5.0}, {0: -math.inf, 3: -math.inf, 69: -math.inf, 1: -math.inf, 4: math.inf}):
        if len(biases) == 2:
            with pytest.raises(ValueError, match="device tensors"):        # past the grammar: the library wants its tensors on the GPU
                rules(biases)
        else:
            with pytest.raises(ValueError, match="state 0"):
                rules(biases)


@pytest.mark.parametrize("seed", range(20))
def test_against_a_walk_over_tokens(seed):
    rng = random.Random(seed)
    n, classes, V = rng.randint(1, 9), rng.randint(1, 5), rng.randint(1, 90)
    of = [rng.randrange(-1, classes + 1) for _ in range(V)]
    to = [[rng.randrange(-1, n + 1) for _ in range(classes)] for _ in range(n)]
    allowed = [[t for t in range(V) if rng.random() < rng.choice([0, 0.02, 0.2])] for _ in range(n)]
    start = rng.randrange(n)
    seen, todo, dead = {start}, [start], False
    while todo:
        s = todo.pop()
        dead |= not allowed[s]
        for t in allowed[s]:
            nxt = to[s][of[t]] if 0 <= of[t] < classes else -1
            if 0 <= nxt < n and nxt not in seen:
                seen.add(nxt)
                todo.append(nxt)
    if dead:
        with pytest.raises(ValueError):
            dec.Grammar(masks(V, *allowed), ints(to), ints(of), start)
    else:
        dec.Grammar(masks(V, *allowed), ints(to), ints(of), start)
