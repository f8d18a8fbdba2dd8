"""Attention that reads shared pages once (byte for byte what every row gets for itself, and against fp64), the weights of the pages against fp64, and the
choice of the pages that go against a plain sort."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, bits_to_f64, down_bf16, step, up, up_bf16
from kv8_ref import D, PAGE, SCALE, Cache, attend, parts
from kv8_shared_ref import SharedCache, page_weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    import paper_2602_00182_amd as d
    return d


def space(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV).fill_(0xFF)


def plain(d, q, pool, table, lens, slots=None):
    """det_attn_decode_kv8, every row for itself."""
    out = torch.full_like(q, float("nan"))
    ws = space(d.det_attn_decode_kv8_workspace_bytes(q.shape[0], q.shape[1], pool.shape[1], D, table.shape[1]))
    d.det_attn_decode_kv8(q, pool, table, lens, slots, out, ws, SCALE)
    return out


def grouped(d, q, pool, table, lens, group_rows, shared, slots=None):
    out = torch.full_like(q, float("nan"))
    ws = space(d.det_attn_decode_kv8_shared_workspace_bytes(q.shape[0], q.shape[1], pool.shape[1], D, table.shape[1]))
    d.det_attn_decode_kv8_shared(q, pool, table, lens, slots, group_rows, shared, out, ws, SCALE)
    return out


def weighed(d, q, pool, table, lens, before, group_rows=None, shared=None, slots=None):
    out, weights = torch.full_like(q, float("nan")), torch.full(table.shape, float("nan"), device=DEV)
    ws = space(d.det_attn_decode_kv8_weights_workspace_bytes(q.shape[0], q.shape[1], pool.shape[1], D, table.shape[1]))
    d.det_attn_decode_kv8_weights(q, pool, table, lens, slots, group_rows, shared, before, weights, out, ws, SCALE)
    return out, weights


def same_bytes(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def fill(cache, seed, Hq, lens=None):
    q = ds.normal_bf16(seed, (len(cache.lengths), Hq, D), 1.5)
    return q, up_bf16(q), up(cache.pool), up(cache.table), up(np.asarray(cache.lengths if lens is None else lens, np.int32))


# lengths of each group's rows; what they share
SHAPES = [
    ("one chunk and a tail", [256], [[300, 257, 511]]),
    ("all of a row is shared", [512], [[512, 300, 256, 17, 600]]),            # rows that end inside what their group shares
    ("less than a chunk", [192], [[200, 193, 450, 192]]),
    ("three groups and a row alone", [768, 0, 256, 1024], [[769, 1000, 1100, 800], [700], [257, 300], [1025] * 5]),
    ("a chunk that is shared in part", [320], [[321, 640, 1000]]),
    ("empty rows", [512], [[600, 0, 513, 0, 700]]),
    ("many rows", [1280], [[1281 + 7 * i for i in range(37)]]),
]


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (6, 2), (8, 2), (5, 1), (8, 1), (16, 1), (32, 8)])
@pytest.mark.parametrize("what,common,lengths", SHAPES, ids=[s[0] for s in SHAPES])
def test_a_row_gets_the_bytes_that_it_gets_alone(d, what, common, lengths, Hq, Hkv):
    c = SharedCache(100 + Hq, Hkv, common, lengths)
    _, q, pool, table, lens = fill(c, 200 + Hq, Hq)
    step(f"{what}, {Hq}/{Hkv} heads")
    got = grouped(d, q, pool, table, lens, up(c.group_rows), up(c.shared))
    want = plain(d, q, pool, table, lens)
    assert same_bytes(got, want)
    out, weights = weighed(d, q, pool, table, lens, None, up(c.group_rows), up(c.shared))
    alone, others = weighed(d, q, pool, table, lens, None)
    assert same_bytes(out, want) and same_bytes(alone, want)
    assert torch.equal(weights, others)  # a page's weight does not depend on who read it


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (5, 1), (16, 8)])
def test_outputs_and_weights_against_fp64(d, Hq, Hkv):
    c = SharedCache(300 + Hq, Hkv, [512, 0], [[513, 700, 600, 530], [130]])
    bits, q, pool, table, lens = fill(c, 301 + Hq, Hq)
    before = np.random.default_rng(5).random(c.table.shape).astype(np.float32)
    step(f"fp64, {Hq}/{Hkv} heads")
    out, weights = weighed(d, q, pool, table, lens, up(before), up(c.group_rows), up(c.shared))
    slots = np.arange(len(c.lengths))
    ref, tol = attend(c, bits, c.lengths, slots)
    assert (np.abs(bits_to_f64(down_bf16(out)) - ref) <= tol).all()
    ref, tol = page_weights(c, bits, c.lengths, slots, *c.table.shape, before)
    err = np.abs(weights.cpu().numpy().astype(np.float64) - ref)
    print("weights: largest error over its allowance", (err / tol).max())
    assert (err <= tol).all()


@pytest.mark.parametrize("length", [1, 2, 63, 64, 65, 255, 256, 257, 511, 512, 513, 1025])
def test_single_rows_at_every_kind_of_length(d, length):
    c = Cache(400 + length, [length], 2)
    bits, q, pool, table, lens = fill(c, 401, 8)
    step(f"{length} tokens")
    out, weights = weighed(d, q, pool, table, lens, None)
    assert same_bytes(out, plain(d, q, pool, table, lens))
    ref, tol = page_weights(c, bits, c.lengths, [0], *c.table.shape, 0.0)
    assert (np.abs(weights.cpu().numpy() - ref) <= tol).all()
    assert abs(float(weights.double().sum()) - 8) < 8 * 1e-5


def test_rows_that_name_slots_and_several_rows_of_one(d):
    """Rows of drafted tokens: five of each slot at growing lengths; their weights meet in the slot's pages."""
    c = Cache(500, [900, 300, 1400], 2)
    slots = np.repeat(np.array([2, 0, 1], np.int32), 5)
    lens = np.array([c.lengths[s] - 4 + i for s in (2, 0, 1) for i in range(5)], np.int32)
    bits = ds.normal_bf16(501, (15, 8, D), 1.5)
    args = up_bf16(bits), up(c.pool), up(c.table), up(lens)
    step("rows that name slots")
    want = plain(d, *args, slots=up(slots))
    group_rows, shared = up(np.array([0, 5, 10, 15], np.int32)), up(np.array([1400, 900, 300], np.int32))  # a slot's rows share all of it
    for groups in ((None, None), (group_rows, shared)):
        out, weights = weighed(d, *args, None, *groups, slots=up(slots))
        assert same_bytes(out, want)
        ref, tol = page_weights(c, bits, lens, slots, *c.table.shape, 0.0)
        assert (np.abs(weights.cpu().numpy() - ref) <= tol).all()
    assert same_bytes(grouped(d, *args, group_rows, shared, slots=up(slots)), want)


def test_groups_that_name_some_of_the_rows_only(d):
    c = SharedCache(600, 2, [512, 256], [[700, 600, 800], [300, 400, 900, 270]])
    _, q, pool, table, lens = fill(c, 601, 8)
    want = plain(d, q, pool, table, lens)
    for rows, shared in [([0, 3], [512]), ([3, 7], [256]), ([1, 3, 5], [512, 256]), ([2, 2, 3, 3, 7], [0, 512, 9999, 256]), ([7], []), ([0, 0], [512])]:
        step(f"groups {rows}")
        if len(shared) == 0:
            got = grouped(d, q, pool, table, lens, None, None)
        else:
            got = grouped(d, q, pool, table, lens, up(np.array(rows, np.int32)), up(np.array(shared, np.int32)))
        assert same_bytes(got, want)


def test_more_groups_than_a_wave_has_lanes(d):
    n = 150
    c = SharedCache(650, 1, [256 if g % 3 else 0 for g in range(n)], [[257 + g] * (1 + g % 3) for g in range(n)])
    _, q, pool, table, lens = fill(c, 651, 2)
    step("150 groups")
    got = grouped(d, q, pool, table, lens, up(c.group_rows), up(c.shared))
    assert same_bytes(got, plain(d, q, pool, table, lens))


def test_what_the_first_rows_table_names_counts(d):
    """The shared chunks are read through the table of the group's first row, whatever the others name there; lengths past the table are cut."""
    c = SharedCache(700, 2, [512], [[600, 700, 800]])
    _, q, pool, table, lens = fill(c, 701, 8)
    want = plain(d, q, pool, table, lens)
    other = table.clone()
    other[1:, :8] = -1
    step("tables without the shared pages")
    assert same_bytes(grouped(d, q, pool, other, lens, up(c.group_rows), up(c.shared)), want)
    lens = up(np.array([600, 10 ** 9, 2 ** 31 - 1], np.int32))
    step("lengths past the table")
    assert same_bytes(grouped(d, q, pool, table, lens, up(c.group_rows), up(c.shared)), plain(d, q, pool, table, lens))


RAGGED = [
    ("two groups", [1024, 512], [[1025 + 3 * i for i in range(33)], [513 + i for i in range(41)]]),
    ("groups of all sizes", [768, 0, 512, 256, 1536], [[770] * 35, [300, 20], [513 + i for i in range(70)], [900, 257, 300], [1537 + 5 * i for i in range(64)]]),
    ("rows that end inside", [1280], [[1280] + [1 + 31 * i for i in range(60)]]),
]


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (9, 3), (8, 2), (5, 1), (16, 2), (16, 1)])
@pytest.mark.parametrize("what,common,lengths", RAGGED, ids=[s[0] for s in RAGGED])
def test_groups_of_many_rows(d, what, common, lengths, Hq, Hkv):
    """Runs of chunks that begin and end anywhere in a group; pages given up in some of them, tokens that are not finite in others."""
    c = SharedCache(720 + Hq, Hkv, common, lengths)
    rng = np.random.default_rng(Hq)
    for g, n in enumerate(common):
        b, e = c.group_rows[g], c.group_rows[g + 1]
        away = rng.choice(n // PAGE, n // PAGE // 4, replace=False) if n else []
        c.table[b:e, away] = -1
    c.table[c.group_rows[0]:c.group_rows[1], 4:8] = -1
    last = c.group_rows[-2]
    if common[-1] >= 512 and len(common) > 2:
        parts(c.pool)[3][c.table[last][c.table[last] >= 0][3], 0, 9] = np.inf  # all rows of the last group see it
    bits = ds.normal_bf16(721 + Hq, (len(c.lengths), Hq, D), 1.5)
    bits[7, Hq - 1, 3] = 0xFF80
    bits[11] = ds.f32_to_bf16_bits(ds.bf16_bits_to_f32(bits[11]) * np.float32(2.0 ** 36))
    q, pool, table, lens = up_bf16(bits), up(c.pool), up(c.table), up(np.asarray(c.lengths, np.int32))
    rows, shared = up(c.group_rows), up(c.shared)
    step(f"{what}, {Hq}/{Hkv} heads")
    want = plain(d, q, pool, table, lens)
    assert same_bytes(grouped(d, q, pool, table, lens, rows, shared), want)
    out, weights = weighed(d, q, pool, table, lens, None, rows, shared)
    alone, others = weighed(d, q, pool, table, lens, None)
    assert same_bytes(out, want) and same_bytes(alone, want) and torch.equal(weights, others)
    assert torch.isfinite(weights).all() and not weights[table < 0].any()
    perm = torch.randperm(len(c.lengths), device=DEV)  # the slots in another order, named by the rows
    inverse = torch.argsort(perm)
    slots = inverse.to(torch.int32)
    out, weights = weighed(d, q, pool, table[perm].contiguous(), lens, None, rows, shared, slots)
    assert same_bytes(out, want) and torch.equal(weights, others[perm])


# rows' own chunks, cut into runs: of one group, of more rows and groups than a wave has lanes, rows without tokens, and groups that fill the chip
BEHIND = [
    ("one group", [512], [[600 + 397 * i for i in range(15)] + [0, 512]]),
    ("no group shares anything", [0, 192], [[900 + 90 * i for i in range(12)], [200, 2000, 192, 3000]]),
    ("forty rows", [512, 1024], [[513 + 97 * i for i in range(25)] + [0, 511, 3], [1025 + 61 * i for i in range(12)]]),
    ("forty rows of a chunk or two", [512], [[513 + 7 * i for i in range(36)] + [0, 511, 3, 900]]),
    ("many groups", [256 * (g % 4) for g in range(100)], [[256 * (g % 4) + 1 + 31 * g % 1500, 256 * (g % 4) + 2 * g] for g in range(100)]),
    ("long and short behind groups of every size", [256 * (g % 3) for g in range(70)], [[1000 + 40 * g, 530 + g, 777][:1 + g % 3] for g in range(70)]),
]


@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (8, 1), (6, 2), (16, 8)])
@pytest.mark.parametrize("what,common,lengths", BEHIND, ids=[s[0] for s in BEHIND])
def test_rows_with_much_behind_what_they_share(d, what, common, lengths, Hq, Hkv):
    c = SharedCache(800 + Hq, Hkv, common, lengths)
    _, q, pool, table, lens = fill(c, 801 + Hq, Hq)
    step(f"{what}, {Hq}/{Hkv} heads")
    want = plain(d, q, pool, table, lens)
    assert same_bytes(grouped(d, q, pool, table, lens, up(c.group_rows), up(c.shared)), want)
    out, weights = weighed(d, q, pool, table, lens, None, up(c.group_rows), up(c.shared))
    _, others = weighed(d, q, pool, table, lens, None)
    assert same_bytes(out, want) and torch.equal(weights, others)


def test_missing_pages_and_slots_that_are_none(d):
    """Pages given up weigh nothing, whole chunks of them too; rows without any page, slot or token give zeros and add nothing."""
    c = SharedCache(800, 2, [1024], [[1100, 1200, 1300, 1024]])
    c.table[:, [1, 4, 5, 6, 7, 13]] = -1   # a page, a whole chunk, and one of the shared ones' last chunk
    c.table[3] = -1
    gone = np.repeat(c.table < 0, PAGE, 1)
    bits, q, pool, table, lens = fill(c, 801, 8)
    step("missing pages")
    want = plain(d, q, pool, table, lens)
    rows, shared = up(np.array([0, 3, 4], np.int32)), up(np.array([1024, 0], np.int32))
    out, weights = weighed(d, q, pool, table, lens, None, rows, shared)
    assert same_bytes(out, want) and same_bytes(grouped(d, q, pool, table, lens, rows, shared), want)
    assert not out[3].any() and not weights[3].any()
    ref, tol = page_weights(c, bits, c.lengths, np.arange(4), *c.table.shape, 0.0, gone=gone)
    got = weights.cpu().numpy()
    assert (np.abs(got - ref) <= tol).all() and not got[c.table < 0].any()
    slots = up(np.array([0, -1, 4, 2], np.int32))
    step("slots that are none")
    out, weights = weighed(d, q, pool, table, lens, None, slots=slots)
    assert same_bytes(out, plain(d, q, pool, table, lens, slots)) and not out[1].any() and not out[2].any()
    assert not weights[1].any() and not weights[3].any() and weights[0].any() and weights[2].any()


def test_rows_and_tokens_that_are_not_finite(d):
    """A query or a token that is not finite makes NaN of the rows that see it, and of no weight; large scores keep their weights."""
    c = SharedCache(900, 2, [512], [[600, 700, 800, 520]])
    bits, q, pool, table, lens = fill(c, 901, 8)
    bits[1, 3, 5] = 0x7F80
    bits[2] = ds.f32_to_bf16_bits(ds.bf16_bits_to_f32(bits[2]) * np.float32(2.0 ** 40))
    q = up_bf16(bits)
    p, t = divmod(750, PAGE)
    parts(c.pool)[2][c.table[2, p], 0, t] = np.nan  # a token of row 2 alone
    pool = up(c.pool)
    step("not finite")
    want = plain(d, q, pool, table, lens)
    out, weights = weighed(d, q, pool, table, lens, None, up(c.group_rows), up(c.shared))
    assert same_bytes(out, want)
    assert torch.isnan(out[1, 3].float()).all() and torch.isnan(out[2, :4].float()).all() and not torch.isnan(out[0].float()).any()
    sums = weights.double().sum(1).cpu().numpy()
    assert np.isfinite(sums).all() and np.abs(sums - [8, 7, 4, 8]).max() < 8 * 1e-5  # the heads that are finite


def test_weights_in_place_and_from_step_to_step(d):
    c = SharedCache(1000, 2, [512], [[600, 700]])
    _, q, pool, table, lens = fill(c, 1001, 8)
    _, once = weighed(d, q, pool, table, lens, None)
    ws = space(d.det_attn_decode_kv8_weights_workspace_bytes(2, 8, 2, D, table.shape[1]))
    weights, out = torch.zeros(table.shape, device=DEV), torch.empty_like(q)
    step("in place")
    for _ in range(3):
        d.det_attn_decode_kv8_weights(q, pool, table, lens, None, None, None, weights, weights, out, ws, SCALE)
    assert torch.equal(weights, once + once + once)


def test_a_cache_past_32_bit_offsets(d):
    """Pages behind the fourth gigabyte of a pool, and the workspace's too."""
    P, Hkv, Hq = 40000, 8, 32
    pool = torch.zeros((P, Hkv, 16896), dtype=torch.uint8, device=DEV)  # 5.4 GB
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    n = 24
    codes = torch.randint(-127, 128, (n, Hkv, 16384), dtype=torch.int8, device=DEV, generator=g)
    at = torch.arange(P - n, P, device=DEV)
    pool[at, :, :16384] = codes.view(torch.uint8)
    pool.view(torch.float32)[at, :, 4096:] = 0.01
    table = torch.full((4, n), -1, dtype=torch.int32, device=DEV)
    table[:, :20] = at[:20].to(torch.int32)
    table[:, 20] = at[20:24].to(torch.int32)
    q = torch.randn((4, Hq, D), device=DEV, generator=g).to(torch.bfloat16)
    lens = torch.full((4,), 20 * PAGE + 40, dtype=torch.int32, device=DEV)
    low = pool[at].contiguous()
    step("far pages")
    rows, shared = up(np.array([0, 4], np.int32)), up(np.array([20 * PAGE], np.int32))
    out = grouped(d, q, pool, table, lens, rows, shared)
    near = torch.where(table >= 0, table - (P - n), -1)
    assert same_bytes(out, grouped(d, q, low, near, lens, rows, shared)) and same_bytes(out, plain(d, q, low, near, lens))


def test_streams_and_graphs(d):
    """Captured and replayed with eager work between, on a stream of its own, beside a second graph with its own workspace."""
    c = SharedCache(1100, 2, [768], [[800, 900, 1000, 770]])
    _, q0, pool, table, lens = fill(c, 1101, 8)
    rows, shared = up(c.group_rows), up(c.shared)
    want, weights_want = weighed(d, q0, pool, table, lens, None, rows, shared)
    q, side = torch.zeros_like(q0), torch.cuda.Stream()
    calls = []
    for _ in range(2):
        out, weights = torch.empty_like(q0), torch.empty(table.shape, device=DEV)
        ws = space(d.det_attn_decode_kv8_weights_workspace_bytes(4, 8, 2, D, table.shape[1]))
        graph = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                d.det_attn_decode_kv8_weights(q, pool, table, lens, None, rows, shared, None, weights, out, ws, SCALE)
        calls.append((graph, out, weights, ws))  # the graph's workspace lives as long as the graph
    torch.cuda.synchronize()
    for i in range(4):
        step(f"replay {i}")
        q.copy_(q0 if i % 2 == 0 else -q0)
        other = None
        if i % 2:
            other = weighed(d, q, pool, table, lens, None, rows, shared)
        for graph, out, weights, _ in calls:
            out.zero_()
            weights.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, out, weights, _ in calls:
            assert same_bytes(out, want if other is None else other[0]) and torch.equal(weights, weights_want if other is None else other[1])
    step("a stream of its own")
    with torch.cuda.stream(side):
        out = torch.empty_like(q0)
        ws = space(d.det_attn_decode_kv8_shared_workspace_bytes(4, 8, 2, D, table.shape[1]))
    side.synchronize()
    d.det_attn_decode_kv8_shared(q0, pool, table, lens, None, rows, shared, out, ws, SCALE, stream=side)
    side.synchronize()
    assert same_bytes(out, want)


# ---------------------------------------------------------------- the pages that go

def picked(weights, table, n_pages, lengths, keep, first, recent):
    """Which pages go, by a sort of each slot's candidates."""
    dropped = np.zeros(weights.shape, np.uint8)
    for s in range(len(lengths)):
        pages = min(max(0, -(-int(lengths[s]) // PAGE)), weights.shape[1])
        there = [i for i in range(pages) if 0 <= table[s, i] < n_pages]
        order = sorted((-np.inf if np.isnan(weights[s, i]) else weights[s, i], 0 if np.isnan(weights[s, i]) else 1, i) for i in there
                       if first <= i < pages - recent)
        order.sort(key=lambda x: (x[1] != 0, x[0], x[2]))
        for _, _, i in order[:max(0, len(there) - max(0, int(keep[s])))]:
            dropped[s, i] = 1
    return dropped


def run_pick(d, weights, table, n_pages, lengths, keep, first, recent):
    dropped = torch.full(table.shape, 7, dtype=torch.uint8, device=DEV)
    d.det_kv8_pick_pages(up(weights), up(table), n_pages, up(lengths), up(keep), first, recent, dropped)
    return dropped.cpu().numpy()


@pytest.mark.parametrize("width", [1, 2, 7, 64, 255, 256, 257, 700, 5000])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
def test_the_pages_of_least_weight_go(d, width, kind):
    rng = np.random.default_rng(width)
    S, P = 9, 50
    weights = rng.exponential(3.0, (S, width)).astype(np.float32)
    if kind == "ties":
        weights = np.floor(weights)
    elif kind == "equal":
        weights[:] = 2.5
    elif kind == "odd":
        weights -= 2
        some = rng.random((S, width))
        weights[some < 0.05] = np.nan
        weights[(some > 0.1) & (some < 0.15)] = np.inf
        weights[(some > 0.2) & (some < 0.25)] = -np.inf
        weights[(some > 0.3) & (some < 0.4)] = 0.0
        weights[(some > 0.4) & (some < 0.5)] = -0.0
        weights[(some > 0.5) & (some < 0.55)] = np.float32(1e-42)
    table = rng.integers(-1, P + 1, (S, width)).astype(np.int32)  # P is none
    lengths = np.array([0, -5, 1, 64, 65, width * PAGE, width * PAGE - 63, 2 ** 31 - 1, max(1, width * PAGE // 2)], np.int32)
    for keep, first, recent in [(0, 0, 0), (1, 1, 1), (width // 2, 1, 4), (width // 3, 0, 2), (width, 2, 0), (-3, 3, 3), (0, 2 ** 31 - 1, 2 ** 31 - 1)]:
        step(f"{width} pages, {kind}, keep {keep}, first {first}, recent {recent}")
        keeps = (keep + np.arange(S) % 3).astype(np.int32)
        got = run_pick(d, weights, table, P, lengths, keeps, first, recent)
        assert np.array_equal(got, picked(weights, table, P, lengths, keeps, first, recent))
