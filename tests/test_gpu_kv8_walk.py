"""Attention over the 8-bit cache by calls of so many rows that their tiles walk the chunks, with the inputs where such a walk can go wrong: holes in the
page table, rows without a slot, tokens that are not finite, queries that are not, lengths of zero.  Against fp64, and byte for byte against a row alone."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, bits_to_f64, down_bf16, step, up, up_bf16
from kv8_ref import D, SCALE, Cache, attend

pytestmark = pytest.mark.gpu
LENGTHS = [700, 513, 130, 300, 1000, 64, 259]
S = len(LENGTHS)


@pytest.fixture(scope="module")
def d():
    import paper_2602_00182_amd as d
    return d


def make(Hkv, seed):
    """Holes: whole chunks, a first page, the last page, single pages.  Token 100 of slot 0 has a NaN key in the first KV head, token 270 of slot 3 an
    infinite value in the last one, token 6 of slot 4 (in a missing page) a NaN key that no one sees."""
    def edit(k, v):
        k[0, 0, 100, 3] = 0x7FC0
        v[3, -1, 270, 9] = 0x7F80
        k[4, :, 6] = 0x7FC0
    cache = Cache(seed, LENGTHS, Hkv, edit=edit)
    gone = np.zeros((S, max(LENGTHS)), dtype=bool)
    table = cache.table.copy()
    for s, pages in ((0, [3, 8]), (1, [0, 8]), (2, [1]), (4, [0, 4, 5, 6, 7, 10]), (6, [4])):
        for i, page in enumerate(pages):
            gone[s, 64 * page:64 * page + 64] = True
            table[s, page] = (-1, -7, cache.pool.shape[0], 2 ** 31 - 1)[(s + i) % 4]
    return cache, table, gone


def rows_of(R, mixed, rng):
    """Rows of every slot, most of them in the order of a prompt, or all in no order; some name slots that are none."""
    slots = np.sort(rng.integers(0, S, R)).astype(np.int32)
    lens = np.array([rng.integers(0, LENGTHS[s] + 1) for s in slots], dtype=np.int32)
    for s in range(S):
        at = slots == s
        lens[at] = np.sort(lens[at])
    lens[rng.integers(0, R, 20)] = 0
    at = rng.integers(0, R, 12)
    slots[at[:6]], slots[at[6:]] = -1, S
    lens[at] = 200
    if mixed:
        order = rng.permutation(R)
        slots, lens = slots[order], lens[order]
    return slots, lens


def kinds(slots, rows):
    """How many slots a workgroup's rows name, at most and at least."""
    each = [len(set(slots[i:i + rows].tolist())) for i in range(0, len(slots) - rows + 1, rows)]
    return max(each), min(each)


def call(d, q, pool, table, lens, slots):
    R, Hq, _ = q.shape
    ws = torch.empty(d.det_attn_decode_kv8_workspace_bytes(R, Hq, pool.shape[1], D, table.shape[1]), dtype=torch.uint8, device=DEV).fill_(0xFF)
    out = torch.full_like(q, float("nan"))
    d.det_attn_decode_kv8(q, pool, table, lens, slots, out, ws, SCALE)
    return out


@pytest.mark.parametrize("R,Hq,Hkv", [(500, 32, 8), (1800, 8, 1), (930, 15, 5), (1900, 8, 8), (900, 16, 4)])
@pytest.mark.parametrize("mixed", [False, True])
def test_walks_over_holes_and_rows_that_are_not_finite(d, R, Hq, Hkv, mixed):
    G = Hq // Hkv
    tile = 16 // G
    assert -(-R // tile) * Hkv >= 896  # the rows walk
    rng = np.random.default_rng(R + mixed)
    cache, table, gone = make(Hkv, 7500 + Hq)
    slots, lens = rows_of(R, mixed, rng)
    most, least = kinds(slots, 4 * tile)
    if mixed and tile > 2:
        assert most > 4   # tiles that go alone
    if not mixed:
        assert least <= 4  # and tiles that go together
    q = ds.normal_bf16(7600 + Hq, (R, Hq, D), 1.5)
    odd = rng.choice(R, 8, replace=False)
    for i, r in enumerate(odd):
        q[r, (5 * i) % Hq, i] = (0xFF80, 0x7FC0)[i % 2]
    step(f"walk of {R} rows, {Hq}/{Hkv} heads, mixed {mixed}")
    pool, dev, qd = up(cache.pool), up(table), up_bf16(q)
    got = down_bf16(call(d, qd, pool, dev, up(lens), up(slots)))
    val = bits_to_f64(got)

    none = (slots < 0) | (slots >= S)
    sees = np.array([0 if n else int((~gone[s, :L]).sum()) for n, s, L in zip(none, slots, lens)])
    bad = np.zeros((R, Hq), dtype=bool)
    bad[(slots == 0) & (lens > 100), :G] = True
    bad[(slots == 3) & (lens > 270), Hq - G:] = True
    for i, r in enumerate(odd):
        bad[r, (5 * i) % Hq] = True
    bad[sees == 0] = False
    assert (val[sees == 0] == 0).all() and (sees == 0).sum() >= 12
    assert np.isnan(val[bad]).all() and np.isfinite(val[~bad]).all() and bad.any()

    pick = sorted(set(range(0, R, max(1, R // 40))) | set(odd.tolist()) | {R - 1} | set(np.flatnonzero(none)[:2].tolist()))
    q0 = q.copy()
    q0[odd] = np.where((q0[odd] & 0x7F80) == 0x7F80, 0, q0[odd])
    with np.errstate(invalid="ignore"):
        ref, tol = attend(cache, q0[pick], np.where(none, 0, lens)[pick], np.clip(slots, 0, S - 1)[pick], gone=gone)
    good = ~bad[pick]
    assert (np.abs(val[pick] - ref) <= tol)[good].all()
    # a row alone, by the forms that take a chunk at a time: rows that name their slot, and rows that are their slot
    for r in pick[::3]:
        one = down_bf16(call(d, qd[r:r + 1], pool, dev, up(lens[r:r + 1]), up(slots[r:r + 1])))[0]
        same = (one == got[r]) | (np.isnan(val[r]) & np.isnan(bits_to_f64(one)))
        assert same.all(), (r, slots[r], lens[r])
        if not none[r]:
            s = int(slots[r])
            one = down_bf16(call(d, qd[r:r + 1], pool, dev[s:s + 1], up(lens[r:r + 1]), None))[0]
            same = (one == got[r]) | (np.isnan(val[r]) & np.isnan(bits_to_f64(one)))
            assert same.all(), (r, slots[r], lens[r])


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 1), (8, 2), (8, 1)])
def test_rows_that_are_their_slots_where_tokens_are_not_finite(d, Hq, Hkv):
    """Slots NULL, up to four heads a KV head (all digits in one operand) and more."""
    G = Hq // Hkv
    cache, table, gone = make(Hkv, 7700 + Hq)
    q = ds.normal_bf16(7710 + Hq, (S, Hq, D), 1.5)
    q[2, 1, 5] = 0x7F80
    step(f"{S} rows without named slots, {Hq}/{Hkv} heads")
    got = bits_to_f64(down_bf16(call(d, up_bf16(q), up(cache.pool), up(table), up(np.array(LENGTHS, np.int32)), None)))
    bad = np.zeros((S, Hq), dtype=bool)
    bad[0, :G] = bad[3, Hq - G:] = True
    bad[2, 1] = True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    q[2, 1, 5] = 0
    with np.errstate(invalid="ignore"):
        ref, tol = attend(cache, q, LENGTHS, range(S), gone=gone)
    assert (np.abs(got - ref) <= tol)[~bad].all()
