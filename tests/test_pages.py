"""KVPages' bookkeeping against a plain model of what each slot should hold, with the page copies done by torch (this runs without a GPU)."""
import random

import pytest
import torch

import paper_2602_00182_amd as d
from paper_2602_00182_amd import api, pages


@pytest.fixture(autouse=True)
def copies(monkeypatch):
    def copy(pool, src, dst, stream=None):
        assert len(set(dst.tolist())) == len(dst) and not set(dst.tolist()) & set(src.tolist())
        pool[:, dst.long()] = pool[:, src.long()]

    monkeypatch.setattr(api, "det_kv8_copy_pages", copy)


def make(n_pages=12, slots=4, max_pages=5, layers=2):
    return d.KVPages(layers, n_pages, 1, slots, max_pages, device="cpu")


def write(p, slot, token, value):
    """A token's place holds a number that names it, in every layer."""
    page = int(p.table[slot, token // 64])
    assert page >= 0
    p.pool[:, page, 0, token % 64] = value


def read(p, slot, n):
    return [int(p.pool[1, int(p.table[slot, t // 64]), 0, t % 64]) for t in range(n)]


def test_reserve_gives_pages_and_release_takes_them_back():
    p = make()
    p.reserve([0, 2], [65, 64])
    assert p.free_pages == 9 and [len(p.pages(s)) for s in range(4)] == [2, 0, 1, 0]
    assert p.table[0, :2].tolist() == p.pages(0) and (p.table[0, 2:] == -1).all() and (p.table[1] == -1).all()
    p.reserve([0], [60])  # less than is there: nothing goes
    assert len(p.pages(0)) == 2
    p.truncate(0, 64)
    assert len(p.pages(0)) == 1
    p.truncate(0, 0)
    p.release(2)
    assert p.free_pages == 12 and (p.table == -1).all()


def test_refusals_change_nothing():
    p = make()
    p.reserve([0], [300])
    before = (p.table.clone(), p.free_pages)
    with pytest.raises(d.OutOfPages):
        p.reserve([1, 2], [300, 300])
    for call in (lambda: p.reserve([1, 1], [1, 1]), lambda: p.reserve([1], [321]), lambda: p.reserve([1], [-1]), lambda: p.reserve([1], [1, 2]),
                 lambda: p.reserve([1], [1], [-1]), lambda: p.fork(0, [0], 10), lambda: p.fork(1, [2], 10), lambda: p.fork(0, [1, 1], 10),
                 lambda: p.fork(0, [1], 400), lambda: p.truncate(0, -1), lambda: make(slots=0), lambda: make(max_pages=0)):
        with pytest.raises(ValueError):
            call()
    assert torch.equal(p.table, before[0]) and p.free_pages == before[1]


def test_a_fork_shares_pages_until_someone_writes():
    p = make()
    p.reserve([0], [100])
    for t in range(100):
        write(p, 0, t, t % 251)
    p.fork(0, [1, 3], 100)
    assert p.free_pages == 10 and p.pages(1) == p.pages(0) == p.pages(3)
    p.reserve([0, 1, 3], [101] * 3, [100] * 3)
    assert len({p.pages(s)[1] for s in (0, 1, 3)}) == 3 and len({p.pages(s)[0] for s in (0, 1, 3)}) == 1 and p.free_pages == 8
    for s in (0, 1, 3):
        write(p, s, 100, 200 + s)
    for s in (0, 1, 3):
        assert read(p, s, 101) == [t % 251 for t in range(100)] + [200 + s]
    p.release(0)
    assert read(p, 1, 101)[-1] == 201 and p.free_pages == 9


@pytest.mark.parametrize("seed", range(6))
def test_random_histories(seed):
    rng = random.Random(seed)
    p, held, clock = make(n_pages=14), {}, 0
    for _ in range(150):
        what = rng.choice(["grow", "grow", "fork", "release", "cut", "rewrite", "compact"])
        live = [s for s in held if held[s]]
        try:
            if what == "grow":
                s = rng.randrange(4)
                have = held.get(s, [])
                n = min(320, len(have) + rng.randrange(1, 90))
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
            elif what == "rewrite" and live:  # rejected drafts: the places from some token on are written again
                s = rng.choice(live)
                n = rng.randrange(len(held[s]))
                p.reserve([s], [len(held[s])], [n])
                for t in range(n, len(held[s])):
                    clock += 1
                    write(p, s, t, clock % 251)
                    held[s] = held[s][:t] + [clock % 251] + held[s][t + 1:]
            elif what == "compact":
                used = p.compact()
                assert used == len({x for s in range(4) for x in p.pages(s)}) and all(x < used for s in range(4) for x in p.pages(s))
        except d.OutOfPages:
            pass
        for s, tokens in held.items():
            assert read(p, s, len(tokens)) == tokens
        assert p.free_pages == 14 - len({x for s in range(4) for x in p.pages(s)})
    assert isinstance(p, pages.KVPages)


@pytest.mark.parametrize("shared", [1, 63, 64, 65, 100, 128])
def test_a_shared_last_page_is_copied_without_write_from_too(shared):
    """The source had room for more than it shared, a first copy holds just the shared tokens, a second is cut before it goes on."""
    p = make()
    p.reserve([0], [shared + 40])
    for t in range(shared):
        write(p, 0, t, t % 251)
    p.fork(0, [1, 2], shared)
    cut = max(1, shared - 30)
    p.truncate(2, cut)
    p.reserve([0, 1], [shared + 1] * 2)
    p.reserve([2], [cut + 1])
    for s, n in ((0, shared), (1, shared), (2, cut)):
        write(p, s, n, 200 + s)
    for s, n in ((0, shared), (1, shared), (2, cut)):
        assert read(p, s, n + 1) == [t % 251 for t in range(n)] + [200 + s]
    full = shared // 64
    assert p.pages(0)[:full] == p.pages(1)[:full]  # pages that no one writes stay shared


def test_the_longest_fork_of_a_slot_is_what_it_goes_on_behind():
    p = make(n_pages=20)
    p.reserve([0], [200])
    for t in range(200):
        write(p, 0, t, t % 251)
    p.fork(0, [1], 200)
    p.fork(0, [2], 70)
    p.reserve([0, 2], [201, 71])
    write(p, 0, 200, 201)
    write(p, 2, 70, 202)
    p.reserve([1], [200])                     # no longer than what is shared: nothing is written
    assert p.free_pages == 20 - 4 - 2 and p.pages(1)[:3] == p.pages(0)[:3] and p.pages(2)[0] == p.pages(0)[0]
    p.reserve([1], [201])
    write(p, 1, 200, 203)
    p.release(2)
    p.fork(1, [2], 10)
    p.reserve([2], [20])
    write(p, 2, 10, 204)
    text = [t % 251 for t in range(200)]
    assert read(p, 0, 201) == text + [201] and read(p, 1, 201) == text + [203] and read(p, 2, 11) == text[:10] + [204]


def test_slots_that_are_none_are_refused():
    p = make()
    p.reserve([0, 3], [70, 5])
    before = (p.table.clone(), p.free_pages)
    for call in (lambda: p.reserve([3, -1], [10, 300]), lambda: p.reserve([-4], [300]), lambda: p.reserve([4], [1]), lambda: p.fork(-4, [1], 10),
                 lambda: p.fork(0, [-2], 10), lambda: p.fork(0, [2, -2], 10), lambda: p.fork(4, [1], 0), lambda: p.truncate(-1, 0), lambda: p.release(4),
                 lambda: p.release(-4), lambda: p.pages(-1), lambda: p.pages(4)):
        with pytest.raises(ValueError):
            call()
    assert torch.equal(p.table, before[0]) and p.free_pages == before[1]
