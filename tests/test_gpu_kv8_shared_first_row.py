"""Groups whose first rows do not hold what the group shares: rows without a slot or a token, rows that end inside it and whose own pages go on elsewhere."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import step, up, up_bf16
from kv8_ref import D, PAGE
from kv8_shared_ref import SharedCache
from test_gpu_kv8_shared import d, grouped, plain, same_bytes, weighed  # noqa: F401 (fixture among them)

pytestmark = pytest.mark.gpu

# what each group shares, the lengths of its rows in the order of the call
ORDERS = [
    ("a short row first", [512], [[300, 700, 600]]),
    ("an empty row first", [768], [[0, 800, 769, 1000]]),
    ("a row of a chunk and less first", [512, 0], [[256, 512, 513], [17, 90]]),
    ("two groups, many short rows first", [512, 1024], [[0, 17, 511, 0, 300, 256, 512, 900], [257, 1023, 1024, 1025, 1500]]),
    ("all end inside: the longest", [1280], [[300, 500, 900, 1088, 700, 1088, 64]]),
    ("rows of a wave and more first", [768], [[0] * 30 + [400] * 30 + [767] * 10 + [768, 1000, 0, 900]]),
    ("more short rows than a wave has lanes", [1024, 0, 512], [[1 + 7 * i for i in range(140)] + [1500, 1030], [300], [0] * 65 + [511] * 3 + [600]]),
]


def build(seed, Hkv, common, lengths):
    """The call's rows: whose tokens, table and lengths; short rows have pages of other sequences behind their own (reserved, not written yet)."""
    orders = [sorted(range(len(of)), key=lambda i, of=of: -of[i]) for of in lengths]
    longest = [max(of) for of in lengths]
    cut = [min(n, top // PAGE * PAGE) for n, top in zip(common, longest)]          # what SharedCache can build: its first row holds all of it
    c = SharedCache(seed, Hkv, cut, [[of[i] for i in order] for of, order in zip(lengths, orders)])
    begin = c.group_rows
    rows = np.concatenate([b + np.argsort(order) for b, order in zip(begin, orders)])
    table, lens = c.table[rows].copy(), np.concatenate([np.asarray(of) for of in lengths]).astype(np.int32)
    rng = np.random.default_rng(seed)
    for r, n in enumerate(lens):
        count = -(-int(n) // PAGE)
        behind = table.shape[1] - count
        table[r, count:] = rng.integers(0, len(c.pool), behind) if r % 2 else -1
    return c, table, lens, np.asarray(common, np.int32)


@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (5, 1), (8, 1), (16, 1), (16, 8)])
@pytest.mark.parametrize("what,common,lengths", ORDERS, ids=[s[0] for s in ORDERS])
def test_whichever_row_is_the_first(d, what, common, lengths, Hq, Hkv):  # noqa: F811
    c, table, lens, shared = build(1300 + Hq, Hkv, common, lengths)
    q, pool, rows = up_bf16(ds.normal_bf16(1301, (len(lens), Hq, D), 1.5)), up(c.pool), up(c.group_rows)
    step(f"{what}, {Hq}/{Hkv} heads")
    want = plain(d, q, pool, up(table), up(lens))
    assert same_bytes(grouped(d, q, pool, up(table), up(lens), rows, up(shared)), want)
    out, weights = weighed(d, q, pool, up(table), up(lens), None, rows, up(shared))
    _, others = weighed(d, q, pool, up(table), up(lens), None)
    assert same_bytes(out, want) and torch.equal(weights, others)


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (16, 1), (16, 8)])
@pytest.mark.parametrize("n", [5, 40, 130])
def test_a_batch_whose_first_sequences_have_ended(d, Hq, Hkv, n):  # noqa: F811
    """Rows that name slots; the slots of those that have ended are none, and the groups stay as they were."""
    c = SharedCache(1400 + n, Hkv, [768, 512], [[800 + 13 * i % 500 for i in range(n)], [600, 513, 700]])
    q, pool, table, rows, shared = up_bf16(ds.normal_bf16(1401, (n + 3, Hq, D), 1.5)), up(c.pool), up(c.table), up(c.group_rows), up(c.shared)
    lens = up(np.asarray(c.lengths, np.int32))
    for ended in ([0], [0, 1, 3], list(range(n - 1)), list(range(n)), [n], [0, n, n + 1]):
        slots = np.arange(n + 3, dtype=np.int32)[::-1].copy()
        slots[ended] = [-1, len(slots), 10 ** 6][len(ended) % 3]
        inverse = up(np.arange(n + 3)[::-1].copy()).long()
        step(f"{len(ended)} of {n} rows ended, {Hq}/{Hkv} heads")
        want = plain(d, q, pool, table[inverse].contiguous(), lens, up(slots))
        assert not want[ended].any()
        assert same_bytes(grouped(d, q, pool, table[inverse].contiguous(), lens, rows, shared, up(slots)), want)
        out, weights = weighed(d, q, pool, table[inverse].contiguous(), lens, None, rows, shared, up(slots))
        _, others = weighed(d, q, pool, table[inverse].contiguous(), lens, None, slots=up(slots))
        assert same_bytes(out, want) and torch.equal(weights, others)
