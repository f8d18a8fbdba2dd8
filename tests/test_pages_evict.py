"""Pages that are given up: holes in a slot's table, whatever happens to it afterwards (host integers; this runs without a GPU)."""
import random

import pytest
import torch

from test_pages import copies, make, read, write  # noqa: F401 (copies: page copies by torch)

import paper_2602_00182_amd as d


def give_up(p, slot, places):
    dropped = torch.zeros(p.table.shape, dtype=torch.uint8)
    dropped[slot, places] = 1
    return p._give_up(dropped)[slot]


def test_a_page_that_is_given_up_is_free_unless_others_name_it():
    p = make(n_pages=14)
    p.reserve([0], [300])
    for t in range(300):
        write(p, 0, t, t % 251)
    p.fork(0, [1, 2], 192)
    free = p.free_pages
    assert give_up(p, 0, [1, 2, 3]) == [1, 2, 3]
    assert p.free_pages == free + 1 and p.pages(0)[1:4] == [-1, -1, -1] and p.table[0, 1:4].tolist() == [-1, -1, -1]
    assert read(p, 1, 192) == [t % 251 for t in range(192)]
    assert give_up(p, 0, [1]) == []                                  # there is none any more
    assert p.shared_tokens([1, 2]) == 192 and p.shared_tokens([0, 1]) == 64 and p.shared_tokens([1]) == 192 and p.shared_tokens([0, 3]) == 0
    give_up(p, 1, [1])
    give_up(p, 2, [1])
    assert p.free_pages == free + 2 and p.shared_tokens([1, 2]) == 192  # both have the same hole


def test_a_slot_with_holes_goes_on_forks_and_ends():
    p = make(n_pages=14)
    p.reserve([0], [300])
    give_up(p, 0, [0, 2])
    p.fork(0, [1], 320)
    p.reserve([1], [320], [290])                                     # its last page becomes its own
    assert p.pages(1)[:4] == p.pages(0)[:4] and p.pages(1)[4] != p.pages(0)[4] and p.pages(1)[0] == -1
    p.compact()
    assert p.pages(0)[0] == -1 and p.pages(0)[2] == -1 and all(x >= 0 for i, x in enumerate(p.pages(0)) if i not in (0, 2))
    free = p.free_pages
    p.reserve([0], [300], [128])                                     # written again from a page that is a hole on
    assert p.pages(0)[2] >= 0 and p.pages(0)[0] == -1 and p.free_pages < free
    before = p.pages(0)
    with pytest.raises(ValueError):
        p.reserve([0], [300], [10])                                  # the tokens in front of 10 are gone
    assert p.pages(0) == before
    p.truncate(0, 64)
    assert p.pages(0) == [-1]
    p.release(0)
    p.release(1)
    assert p.free_pages == 14


def test_too_few_pages_for_a_hole_change_nothing():
    p = make(n_pages=5)
    p.reserve([0], [192])
    give_up(p, 0, [1])
    p.reserve([1], [192])
    before = p.pages(0), p.pages(1), p.free_pages
    with pytest.raises(d.OutOfPages):
        p.reserve([0], [192], [64])
    assert (p.pages(0), p.pages(1), p.free_pages) == before


def test_what_evict_refuses():
    p = make(n_pages=5)
    with pytest.raises(ValueError):
        p.evict(torch.zeros(p.table.shape), torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), recent=0)


@pytest.mark.parametrize("seed", range(6))
def test_random_histories_with_holes(seed):
    rng = random.Random(seed)
    p, held, clock = make(n_pages=14), {}, 0
    for _ in range(150):
        what = rng.choice(["grow", "grow", "fork", "release", "cut", "hole", "hole", "compact"])
        live = [s for s in held if held[s]]
        try:
            if what == "grow":
                s = rng.randrange(4)
                have = held.get(s, [])
                n = min(320, len(have) + rng.randrange(1, 90))
                if len(have) % 64 and have[-1] is None:              # its last page is a hole: nothing can go on behind it
                    with pytest.raises(ValueError):
                        p.reserve([s], [n], [len(have)])
                    continue
                p.reserve([s], [n], [len(have)])
                for t in range(len(have), n):
                    clock += 1
                    write(p, s, t, clock % 251)
                    have = have + [clock % 251]
                held[s] = have
            elif what == "fork" and live:
                s, empty = rng.choice(live), [x for x in range(4) if not held.get(x)]
                if empty:
                    n = rng.randrange(1, len(held[s]) + 1)
                    p.fork(s, empty, n)
                    for x in empty:
                        held[x] = held[s][:n]
            elif what == "release" and live:
                s = rng.choice(live)
                p.release(s)
                held[s] = []
            elif what == "cut" and live:
                s = rng.choice(live)
                n = rng.randrange(len(held[s]) + 1)
                p.truncate(s, n)
                held[s] = held[s][:n]
            elif what == "hole" and live:
                s = rng.choice(live)
                i = rng.randrange(-(-len(held[s]) // 64))
                give_up(p, s, [i])
                held[s] = [None if t // 64 == i else x for t, x in enumerate(held[s])]
            elif what == "compact":
                p.compact()
        except d.OutOfPages:
            pass
        for s, tokens in held.items():
            table = p.pages(s)
            for t, x in enumerate(tokens):
                assert (x is None) == (table[t // 64] < 0)
            assert p.table[s, :len(table)].tolist() == table
            got = [None if table[t // 64] < 0 else int(p.pool[0, table[t // 64], 0, t % 64]) for t in range(len(tokens))]
            assert got == tokens
        assert p.free_pages == 14 - len({x for s in range(4) for x in p.pages(s) if x >= 0})
