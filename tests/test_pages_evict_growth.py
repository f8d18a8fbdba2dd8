"""A slot that has given up pages grows as any other: its holes stay holes unless the caller writes there again (host integers; this runs without a GPU)."""
import random

import pytest
import torch

from test_pages import copies, make, read, write  # noqa: F401 (copies: page copies by torch)
from test_pages_evict import give_up

import paper_2602_00182_amd as d


def test_holes_stay_when_a_slot_grows():
    p = make(n_pages=20, max_pages=12)
    p.reserve([0], [300])
    for t in range(300):
        write(p, 0, t, t % 251)
    assert give_up(p, 0, [1, 2]) == [1, 2]
    free, kept = p.free_pages, p.pages(0)
    p.reserve([0], [330])                      # 6 pages: one more than there are
    assert p.pages(0)[:5] == kept == [kept[0], -1, -1, kept[3], kept[4]] and p.pages(0)[5] >= 0
    assert p.free_pages == free - 1 and p.table[0, :6].tolist() == p.pages(0)
    assert [int(p.pool[1, p.pages(0)[t // 64], 0, t % 64]) for t in range(300) if t // 64 not in (1, 2)] == [t % 251 for t in range(300) if t // 64 not in (1, 2)]
    p.reserve([0], [330])                      # and again: nothing
    p.reserve([0], [100])
    assert p.pages(0)[1:3] == [-1, -1] and p.free_pages == free - 1


@pytest.mark.parametrize("length", [64, 100, 128, 192, 250])
def test_holes_stay_when_a_slot_that_was_forked_grows(length):
    """Source and fork, at aligned and unaligned lengths, with a hole at the old boundary too."""
    p = make(n_pages=40, max_pages=12)
    p.reserve([0], [300])
    for t in range(300):
        write(p, 0, t, t % 251)
    p.fork(0, [1], length)
    p.reserve([0, 1], [300, 300])              # both write behind what they share
    for t in range(length, 300):
        write(p, 1, t, t % 241)
    for slot in (0, 1):
        assert give_up(p, slot, [1, 2]) == [1, 2]
    free, kept = p.free_pages, [p.pages(s) for s in (0, 1)]
    p.reserve([0, 1], [520, 450])              # 9 and 8 pages where there were 5
    for slot, n in ((0, 9), (1, 8)):
        assert p.pages(slot)[:5] == kept[slot] and kept[slot][1:3] == [-1, -1] and len(p.pages(slot)) == n
        assert all(x >= 0 for x in p.pages(slot)[5:]) and p.table[slot, :n].tolist() == p.pages(slot)
    assert p.free_pages == free - 7
    p.reserve([0], [600], [200])               # written again from token 200 on: page 3 is there, nothing in front of it comes back
    assert p.pages(0)[1:3] == [-1, -1]
    p.reserve([0], [600], [128])               # from page 2 on
    assert p.pages(0)[1] == -1 and p.pages(0)[2] >= 0


def test_too_few_pages_for_growth_alone():
    """Holes ask for no pages: a slot may grow into the very pages that it gave up."""
    p = make(n_pages=5, max_pages=8)
    p.reserve([0], [320])
    with pytest.raises(d.OutOfPages):
        p.reserve([0], [321])
    give_up(p, 0, [1, 3])
    p.reserve([0], [448])
    assert p.pages(0)[1] == p.pages(0)[3] == -1 and len(p.pages(0)) == 7 and p.free_pages == 0
    with pytest.raises(d.OutOfPages):
        p.reserve([0], [449])


def test_nothing_goes_on_inside_a_hole():
    """A slot that a fork or a truncation left with its last token in a page that was given up: what it writes next would have no page."""
    p = make(n_pages=20, max_pages=8)
    p.reserve([0], [300])
    give_up(p, 0, [1])
    p.fork(0, [1], 100)
    p.fork(0, [2], 128)
    before = p.pages(1), p.free_pages
    with pytest.raises(ValueError):
        p.reserve([1], [200])
    assert (p.pages(1), p.free_pages) == before
    p.reserve([2], [200])                      # ends with the page: goes on in the next one
    assert p.pages(2)[1] == -1 and len(p.pages(2)) == 4
    p.truncate(0, 100)
    with pytest.raises(ValueError):
        p.reserve([0], [200])
    p.reserve([0], [200], [64])                # the page written anew
    assert p.pages(0)[1] >= 0
    p.reserve([0], [300])
    assert give_up(p, 0, [1]) == [1]
    p.reserve([0], [400])                      # long past it now
    assert p.pages(0)[1] == -1


@pytest.mark.parametrize("seed", range(6))
def test_random_growth_by_default(seed):
    """Slots grow without a write_from through forks, truncations to whole pages and holes; a model of the tokens says what each page has to hold."""
    rng = random.Random(seed)
    p, held, clock = make(n_pages=16, max_pages=6), {s: [] for s in range(4)}, 0
    for _ in range(200):
        what, s = rng.choice(["grow", "grow", "grow", "fork", "cut", "hole", "hole", "compact"]), rng.randrange(4)
        have = held[s]
        try:
            if what == "grow":
                n = min(384, len(have) + rng.randrange(1, 100))
                if len(have) % 64 and have[-1] is None:
                    continue
                p.reserve([s], [n])
                for t in range(len(have), n):
                    clock += 1
                    write(p, s, t, clock % 251)
                    have.append(clock % 251)
            elif what == "fork" and have:
                empty = [x for x in range(4) if not held[x]]
                n = rng.randrange(1, len(have) + 1)
                if empty:
                    p.fork(s, empty, n)
                    for x in empty:
                        held[x] = have[:n]
            elif what == "cut":
                n = rng.randrange(len(have) // 64 + 1) * 64
                p.truncate(s, n)
                held[s] = have[:n]
            elif what == "hole" and len(have) > 64:
                i = rng.randrange((len(have) - 1) // 64)
                give_up(p, s, [i])
                held[s] = [None if t // 64 == i else x for t, x in enumerate(have)]
            elif what == "compact":
                p.compact()
        except d.OutOfPages:
            pass
        for slot, tokens in held.items():
            table = p.pages(slot)
            assert p.table[slot, :len(table)].tolist() == table
            assert [None if table[t // 64] < 0 else int(p.pool[0, table[t // 64], 0, t % 64]) for t in range(len(tokens))] == tokens
        assert p.free_pages == 16 - len({x for slot in range(4) for x in p.pages(slot) if x >= 0})
