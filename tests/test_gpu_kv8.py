"""The 8-bit paged cache: append, read, copies and attention against references in numpy (the quantizer's bytes exactly, attention in
fp64), at the sizes, masks and orders where they can go wrong."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, bits_to_f64, down_bf16, step, up, up_bf16
from kv8_ref import D, PAGE, RECORD, SCALE, Cache, attend, parts, quantize, store

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    import paper_2602_00182_amd as d
    return d


def attn(d, q, pool, table, lens, slots, scale=SCALE, stream=None, ws=None, out=None):
    R, Hq, _ = q.shape
    if ws is None:
        ws = torch.empty(d.det_attn_decode_kv8_workspace_bytes(R, Hq, pool.shape[1], D, table.shape[1]), dtype=torch.uint8, device=DEV)
        ws.fill_(0xFF)
    out = torch.full_like(q, float("nan")) if out is None else out
    d.det_attn_decode_kv8(q, pool, table, lens, slots, out, ws, scale, stream)
    return out


def run_attn(d, cache, q, lens, slots, scale=SCALE):
    out = attn(d, up_bf16(q), up(cache.pool), up(cache.table), up(np.asarray(lens, np.int32)),
               None if slots is None else up(np.asarray(slots, np.int32)), scale)
    torch.cuda.synchronize()
    return down_bf16(out)


# ---------------------------------------------------------------- append and read

@pytest.mark.parametrize("R,Hq,Hkv", [(1, 1, 1), (3, 5, 1), (17, 32, 8), (2, 48, 8), (70, 4, 4), (130, 16, 2)])
def test_append_writes_the_quantizers_bytes_and_nothing_else(d, R, Hq, Hkv):
    rng = np.random.default_rng(R * 100 + Hq)
    S, P, pages = 4, 24, 6
    table = rng.permutation(P).reshape(S, pages).astype(np.int32)
    spots = rng.permutation(S * pages * PAGE)[:R]
    slots, pos = (spots // (pages * PAGE)).astype(np.int32), (spots % (pages * PAGE)).astype(np.int32)
    n = (Hq + 2 * Hkv) * D
    wide = ds.normal_bf16(7000 + R, (R, n + 24))
    wide[0, :D] = 0                     # a zero head
    wide[R // 2, Hq * D:Hq * D + 2 * D] = ds.f32_to_bf16_bits(np.float32(1e-39) * np.arange(2 * D, dtype=np.float32))  # subnormal keys or a value head
    wide[R - 1, (Hq + Hkv) * D:(Hq + Hkv + 1) * D] = 0
    cos, sin = ds.rope_tables(pages * PAGE, D)
    pool0 = rng.integers(0, 256, (P, Hkv, RECORD), dtype=np.uint8)
    dev = up_bf16(wide)
    pool, q = up(pool0.copy()), torch.full((R, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    step(f"append {R} rows, {Hq}/{Hkv} heads")
    d.det_kv8_rope_append(dev[:, :n], q, pool, up(table), up(pos), up(slots), up(cos), up(sin))
    torch.cuda.synchronize()
    heads = up_bf16(np.ascontiguousarray(wide[:, :n]).reshape(R, Hq + 2 * Hkv, D))
    turned = torch.empty_like(heads[:, :Hq + Hkv].contiguous())
    d.det_rope(heads[:, :Hq + Hkv].contiguous(), turned, up(pos), up(cos), up(sin))
    turned = down_bf16(turned)
    assert np.array_equal(down_bf16(q), turned[:, :Hq])
    kc, kd = quantize(turned[:, Hq:])
    vc, vd = quantize(wide[:, :n].reshape(R, Hq + 2 * Hkv, D)[:, Hq + Hkv:])
    want = pool0.copy()
    for r in range(R):
        for g in range(Hkv):
            store(want, table[slots[r], pos[r] // PAGE], g, pos[r] % PAGE, kc[r, g], kd[r, g], vc[r, g], vd[r, g])
    assert np.array_equal(pool.cpu().numpy(), want)
    # and read back
    k, v = (torch.full((R, Hkv, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    step("read them back")
    d.det_kv8_read(pool, up(table), up(pos), up(slots), k, v)
    torch.cuda.synchronize()
    assert np.array_equal(down_bf16(k), ds.f32_to_bf16_bits(kc.astype(np.float32) * kd[..., None]))
    assert np.array_equal(down_bf16(v), ds.f32_to_bf16_bits(vc.astype(np.float32) * vd[..., None]))


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_append_of_many_rows_in_runs_and_in_no_order(d, seed):
    """Some hundred rows: runs of neighbouring positions that begin anywhere, single rows, rows without a page, every one where it belongs."""
    rng = np.random.default_rng(seed)
    Hq, Hkv, S, pages = 3, 1, 9, 5
    P = S * pages + 2
    table = rng.permutation(P)[:S * pages].reshape(S, pages).astype(np.int32)
    table[3, 1] = -1
    spots = []
    for s in range(S):
        at = int(rng.integers(0, 30))
        while at < pages * PAGE:
            run = int(rng.choice([1, 2, 5, 16, 33, 70]))
            spots.append([(s, p) for p in range(at, min(at + run, pages * PAGE))])
            at += run + int(rng.integers(0, 40))
    spots = [x for i in rng.permutation(len(spots)) for x in (spots[i] if rng.integers(2) else spots[i][::-1])]
    spots.insert(100, (2, -1))
    spots.insert(101, (S, 3))
    slots, pos = (np.array([x[i] for x in spots], dtype=np.int32) for i in (0, 1))
    R = len(spots)
    x = ds.normal_bf16(7050 + seed, (R, (Hq + 2 * Hkv) * D))
    cos, sin = ds.rope_tables(pages * PAGE, D)
    pool0 = rng.integers(0, 256, (P, Hkv, RECORD), dtype=np.uint8)
    pool, q = up(pool0.copy()), torch.empty((R, Hq, D), dtype=torch.bfloat16, device=DEV)
    step(f"{R} rows in runs")
    d.det_kv8_rope_append(up_bf16(x), q, pool, up(table), up(pos), up(slots), up(cos), up(sin))
    torch.cuda.synchronize()
    heads = up_bf16(np.ascontiguousarray(x.reshape(R, Hq + 2 * Hkv, D)[:, :Hq + Hkv]))
    turned = torch.empty_like(heads)
    d.det_rope(heads, turned, up(pos), up(cos), up(sin))
    turned = down_bf16(turned)
    assert np.array_equal(down_bf16(q), turned[:, :Hq])
    kc, kd = quantize(turned[:, Hq:])
    vc, vd = quantize(x.reshape(R, Hq + 2 * Hkv, D)[:, Hq + Hkv:])
    want = pool0.copy()
    for r in range(R):
        if 0 <= slots[r] < S and pos[r] >= 0 and table[slots[r], pos[r] // PAGE] >= 0:
            store(want, table[slots[r], pos[r] // PAGE], 0, pos[r] % PAGE, kc[r, 0], kd[r, 0], vc[r, 0], vd[r, 0])
    assert np.array_equal(pool.cpu().numpy(), want)


def test_append_of_rows_without_a_place_and_rows_that_are_not_finite(d):
    Hq, Hkv, P = 2, 1, 3
    table = np.array([[2, -1], [0, 7]], dtype=np.int32)  # page 7 does not exist
    slots = np.array([0, 0, 1, 2, -1, 0, 0, 1, 1], dtype=np.int32)
    pos = np.array([5, 64, 64, 0, 0, 128, -1, 3, 4], dtype=np.int32)
    R = len(pos)
    x = ds.normal_bf16(71, (R, (Hq + 2 * Hkv) * D))
    x[7, Hq * D + 3] = 0x7F80            # an infinite key: rotation spreads it to its pair
    x[8, (Hq + Hkv) * D + 100] = 0x7FC0  # a NaN among a value row
    cos, sin = ds.rope_tables(200, D)
    pool0 = np.full((P, Hkv, RECORD), 0xAB, dtype=np.uint8)
    pool, q = up(pool0.copy()), torch.empty((R, Hq, D), dtype=torch.bfloat16, device=DEV)
    step("rows without a page")
    d.det_kv8_rope_append(up_bf16(x), q, pool, up(table), up(pos), up(slots), up(cos), up(sin))
    torch.cuda.synchronize()
    got = pool.cpu().numpy()
    heads = up_bf16(x.reshape(R, Hq + 2 * Hkv, D)[:, :Hq + Hkv])
    turned = torch.empty_like(heads)
    d.det_rope(heads, turned, up(pos), up(cos), up(sin))
    kc, kd = quantize(down_bf16(turned)[:, Hq:])
    vc, vd = quantize(x.reshape(R, Hq + 2 * Hkv, D)[:, Hq + Hkv:])
    want = pool0.copy()
    for r, page in ((0, 2), (7, 0), (8, 0)):
        store(want, page, 0, pos[r] % PAGE, kc[r, 0], kd[r, 0], vc[r, 0], vd[r, 0])
    assert np.isnan(kd[7]).all() and np.isnan(vd[8]).all() and not kc[7].any() and not vc[8].any()
    same = got == want
    scales = slice(2 * PAGE * D, RECORD)
    assert same[..., :2 * PAGE * D].all()
    assert np.array_equal(got[..., scales].copy().view(np.float32), want[..., scales].copy().view(np.float32), equal_nan=True)
    k, v = (torch.full((R, Hkv, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    d.det_kv8_read(pool, up(table), up(pos), up(slots), k, v)
    torch.cuda.synchronize()
    for r in (1, 2, 3, 4, 5, 6):
        assert not k[r].any() and not v[r].any()
    assert torch.isnan(k[7]).all() and torch.isnan(v[8]).all()


def test_append_token_by_token_is_append_at_once(d):
    Hq, Hkv, T = 4, 2, 150
    x = up_bf16(ds.normal_bf16(73, (T, (Hq + 2 * Hkv) * D)))
    cos, sin = (up(t) for t in ds.rope_tables(T, D))
    table = up(np.array([[3, 0, 2]], dtype=np.int32))
    pos = up(np.arange(T, dtype=np.int32))
    slots = torch.zeros(T, dtype=torch.int32, device=DEV)
    pools = [torch.zeros((4, Hkv, RECORD), dtype=torch.uint8, device=DEV) for _ in range(2)]
    q = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV)
    step("150 rows at once and one by one")
    d.det_kv8_rope_append(x, q, pools[0], table, pos, slots, cos, sin)
    for t in range(T):
        d.det_kv8_rope_append(x[t:t + 1], q[t:t + 1], pools[1], table, pos[t:t + 1], None, cos, sin)
    torch.cuda.synchronize()
    assert torch.equal(pools[0], pools[1])


# ---------------------------------------------------------------- attention

LENGTHS = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 770, 1025]


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (2, 1), (6, 2), (8, 2), (5, 1), (14, 2), (8, 1), (32, 8), (16, 1)])
def test_single_tokens_at_every_kind_of_length(d, Hq, Hkv):
    cache = Cache(7100 + Hq, LENGTHS, Hkv)
    q = ds.normal_bf16(7200 + Hq, (len(LENGTHS), Hq, D), 2.0)
    step(f"{len(LENGTHS)} lengths, {Hq}/{Hkv} heads")
    got = run_attn(d, cache, q, LENGTHS, None)
    ref, tol = attend(cache, q, LENGTHS, range(len(LENGTHS)))
    assert (np.abs(bits_to_f64(got) - ref) <= tol).all()


def test_rows_that_see_nothing_give_zeros(d):
    cache = Cache(7300, [300, 40, 64, 0], 2)
    table = cache.table.copy()
    table[1] = -1                                   # a sequence without pages
    table[2, 0] = cache.pool.shape[0]               # a page that does not exist
    lens = np.array([0, 40, 64, 64, 5, -3, 300], dtype=np.int32)
    slots = np.array([0, 1, 2, 3, 9, 0, -1], dtype=np.int32)
    q = ds.normal_bf16(7301, (len(lens), 4, D))
    step("rows without tokens")
    out = attn(d, up_bf16(q), up(cache.pool), up(table), up(lens), up(slots))
    torch.cuda.synchronize()
    assert not out.float().any()


def test_missing_pages_are_left_out_and_lengths_are_cut_to_the_table(d):
    lengths = [700, 513, 130]
    cache = Cache(7310, lengths, 2, extra_pages=0)
    gone = np.zeros((3, 704), dtype=bool)
    gone[0, 64:128] = gone[0, 256:576] = gone[1, :64] = gone[1, 512:576] = True
    table = cache.table.copy()
    table[0, 1] = table[0, 4:9] = table[1, 0] = -5
    table[1, 8] = 10 ** 6
    q = ds.normal_bf16(7311, (3, 8, D), 2.0)
    step("missing pages")
    lens = up(np.array(lengths, dtype=np.int32))
    out = down_bf16(attn(d, up_bf16(q), up(cache.pool), up(table), lens, None))
    ref, tol = attend(cache, q, lengths, range(3), gone=gone)
    assert (np.abs(bits_to_f64(out) - ref) <= tol).all()
    # a full table: tokens past it are not there
    lengths = [128, 128]
    cache = Cache(7312, lengths, 1, extra_pages=0)
    q = ds.normal_bf16(7313, (2, 2, D))
    got = run_attn(d, cache, q, [128, 2 ** 31 - 1], None)
    ref, tol = attend(cache, q, lengths, range(2))
    assert (np.abs(bits_to_f64(got) - ref) <= tol).all()


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 2), (16, 2), (16, 1)])
def test_rows_that_share_slots_in_any_order(d, Hq, Hkv):
    lengths = [400, 90, 257]
    cache = Cache(7320 + Hq, lengths, Hkv)
    rng = np.random.default_rng(Hq)
    rows = [(s, n) for s, L in enumerate(lengths) for n in rng.integers(0, L + 1, 15)] + [(0, 400), (0, 400), (2, 256)]
    rows = [rows[i] for i in rng.permutation(len(rows))]
    slots, lens = np.array([r[0] for r in rows], np.int32), np.array([r[1] for r in rows], np.int32)
    q = ds.normal_bf16(7330 + Hq, (len(rows), Hq, D), 1.5)
    step(f"{len(rows)} rows of three slots, {Hq}/{Hkv} heads")
    got = run_attn(d, cache, q, lens, slots)
    ref, tol = attend(cache, q, lens, slots)
    assert (np.abs(bits_to_f64(got) - ref) <= tol).all()
    # a row alone, in other pages, with a longer table: the same bytes
    pool, table = up(cache.pool), cache.table
    moved = torch.empty((table.size * 2 + 5,) + cache.pool.shape[1:], dtype=torch.uint8, device=DEV).fill_(0x7F)
    other = np.full((5, table.shape[1] + 9), -1, dtype=np.int32)
    for s in range(3):
        for i, page in enumerate(table[s]):
            if page >= 0:
                other[s + 1, i] = 2 * (s * table.shape[1] + i) + 3
                moved[other[s + 1, i]] = pool[page]
    for r in list(range(0, len(rows), 7)) + [len(rows) - 1]:
        one = attn(d, up_bf16(q[r:r + 1]), moved, up(other), up(lens[r:r + 1]), up(slots[r:r + 1] + 1))
        assert np.array_equal(down_bf16(one)[0], got[r]), rows[r]


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (32, 8), (16, 16), (8, 1), (15, 5)])
def test_prompt_rows_are_the_tokens_decoded_one_by_one(d, Hq, Hkv):
    """Many rows of a prompt in one call against calls of one row: the same bytes whatever form the sizes select."""
    lengths = [1203, 700, 389]
    cache = Cache(7340, lengths, Hkv)
    slots = np.repeat(np.arange(3), lengths).astype(np.int32)
    lens = np.concatenate([np.arange(1, n + 1) for n in lengths]).astype(np.int32)
    q = ds.normal_bf16(7341, (len(lens), Hq, D), 1.5)
    step(f"{len(lens)} prompt rows")
    pool, table, qd = up(cache.pool), up(cache.table), up_bf16(q)
    got = down_bf16(attn(d, qd, pool, table, up(lens), up(slots)))
    pick = list(range(0, len(lens), 173)) + [1202, 1203, 2291]
    ref, tol = attend(cache, q[pick], lens[pick], slots[pick])
    assert (np.abs(bits_to_f64(got[pick]) - ref) <= tol).all()
    for r in pick:
        one = attn(d, qd[r:r + 1], pool, table, up(lens[r:r + 1]), up(slots[r:r + 1]))
        assert np.array_equal(down_bf16(one)[0], got[r]), r
    # 5 consecutive rows (drafts), and 40
    for a, b in ((1000, 1005), (1180, 1220)):
        some = attn(d, qd[a:b].contiguous(), pool, table, up(lens[a:b]), up(slots[a:b]))
        assert np.array_equal(down_bf16(some), got[a:b])


def test_many_rows_of_many_slots_in_no_order(d):
    """As many rows as a prompt has, but every one of some forty sequences, interleaved; a stretch of one slot and of two among them."""
    rng = np.random.default_rng(7345)
    lengths = [int(n) for n in rng.integers(1, 700, 40)]
    Hq, Hkv = 32, 8
    cache = Cache(7345, lengths, Hkv)
    slots = rng.integers(0, 40, 1400).astype(np.int32)
    slots[200:300], slots[600:700] = 7, rng.choice([3, 5], 100)
    lens = np.array([rng.integers(0, lengths[s] + 1) for s in slots], dtype=np.int32)
    q = ds.normal_bf16(7346, (1400, Hq, D), 1.5)
    step("1400 rows of 40 slots")
    pool, table, qd = up(cache.pool), up(cache.table), up_bf16(q)
    got = down_bf16(attn(d, qd, pool, table, up(lens), up(slots)))
    pick = list(range(0, 1400, 97)) + [200, 260, 640, 1399]
    ref, tol = attend(cache, q[pick], lens[pick], slots[pick])
    assert (np.abs(bits_to_f64(got[pick]) - ref) <= tol).all()
    for r in pick:
        one = attn(d, qd[r:r + 1], pool, table, up(lens[r:r + 1]), up(slots[r:r + 1]))
        assert np.array_equal(down_bf16(one)[0], got[r]), r


@pytest.mark.parametrize("R,Hq,Hkv,named", [(600, 32, 8, False), (600, 64, 8, False), (1700, 8, 8, True)])
def test_workgroups_that_take_several_chunks(d, R, Hq, Hkv, named):
    """So many rows that a workgroup goes on from chunk to chunk, in a table much wider than the sequences are long; slots that share pages."""
    lengths = [4000, 40, 2900, 700]
    cache = Cache(7347, lengths, Hkv)
    rng = np.random.default_rng(R + Hq)
    slots = np.sort(rng.integers(0, 4, R)).astype(np.int32) if named else (np.arange(R) % 4).astype(np.int32)
    lens = np.array([rng.integers(0, lengths[s] + 1) for s in slots], dtype=np.int32)
    wide = np.full((4 if named else R, 500), -1, dtype=np.int32)
    for s in range(wide.shape[0]):
        wide[s, :cache.table.shape[1]] = cache.table[s % 4]
    q = ds.normal_bf16(7348, (R, Hq, D), 1.5)
    step(f"{R} rows, {Hq}/{Hkv} heads, a table of 500 pages")
    pool, qd = up(cache.pool), up_bf16(q)
    got = down_bf16(attn(d, qd, pool, up(wide), up(lens), up(slots) if named else None))
    pick = list(range(0, R, 61)) + [R - 1]
    ref, tol = attend(cache, q[pick], lens[pick], slots[pick])
    assert (np.abs(bits_to_f64(got[pick]) - ref) <= tol).all()
    for r in pick:
        one = attn(d, qd[r:r + 1], pool, up(cache.table), up(lens[r:r + 1]), up(slots[r:r + 1]))
        assert np.array_equal(down_bf16(one)[0], got[r]), r


def test_extreme_scores_and_values(d):
    """One weight that is all (scores in the hundreds), equal scores, values of very different sizes, zero queries and zero keys."""
    def edit(k, v):
        k[1, :, :, :] = k[1, :, :1, :]                         # all keys of slot 1 alike
        k[2, :, 10] = 0                                        # a zero key
        v[2, :, ::7] = ds.f32_to_bf16_bits(ds.bf16_bits_to_f32(v[2, :, ::7]) * np.float32(2.0 ** 40))
        v[3] = ds.f32_to_bf16_bits(ds.bf16_bits_to_f32(v[3]) * np.float32(2.0 ** -60))
        v[4, :, 5:] = 0
    lengths = [600, 300, 555, 200, 310]
    cache = Cache(7350, lengths, 2, edit=edit)
    q = ds.normal_bf16(7351, (5, 4, D))
    q[0] = ds.f32_to_bf16_bits(ds.bf16_bits_to_f32(q[0]) * np.float32(60.0))
    q[3, 1] = 0
    q[3, 2] = ds.f32_to_bf16_bits(ds.bf16_bits_to_f32(q[3, 2]) * np.float32(2.0 ** -70))
    q[3, 3, 7] = ds.f32_to_bf16_bits(np.float32([300.0]))[0]
    step("extreme scores")
    got = run_attn(d, cache, q, lengths, None)
    ref, tol = attend(cache, q, lengths, range(5))
    assert (np.abs(bits_to_f64(got) - ref) <= tol).all()


def test_rows_that_are_not_finite_reach_only_those_that_see_them(d):
    def edit(k, v):
        k[0, 0, 100, 3] = 0x7FC0     # slot 0: a NaN key at token 100 of KV head 0
        v[1, 1, 70, 9] = 0x7F80      # slot 1: an infinite value at token 70 of KV head 1
    cache = Cache(7360, [300, 300], 2, edit=edit)
    lens = np.array([100, 101, 300, 70, 71, 300, 64], dtype=np.int32)
    slots = np.array([0, 0, 0, 1, 1, 1, 0], dtype=np.int32)
    q = ds.normal_bf16(7361, (7, 4, D))
    q[6, 2, 0] = 0xFF80               # an infinite query: its own head only
    step("rows that are not finite")
    got = bits_to_f64(run_attn(d, cache, q, lens, slots))
    bad = np.zeros((7, 4), dtype=bool)
    bad[1, :2] = bad[2, :2] = bad[4, 2:] = bad[5, 2:] = bad[6, 2] = True
    assert np.isnan(got[bad]).all()
    q2 = q.copy()
    q2[6, 2, 0] = 0
    clean = Cache(7360, [300, 300], 2)
    clean.v[1, 1, 70] = 0
    ref, tol = attend(clean, q2, lens, slots)
    assert (np.abs(got - ref) <= tol)[~bad].all()


def test_a_long_cache_past_32_bit_offsets(d):
    """A sequence of 9000 tokens whose pages lie past 4 GiB of the pool, beside pages of the same numbers modulo 2^32 bytes."""
    Hkv, Hq, n = 8, 32, 9000
    cache = Cache(7370, [n], Hkv, spare=0, extra_pages=0)
    P = 2 ** 33 // (Hkv * RECORD) + 200
    pool = torch.zeros((P, Hkv, RECORD), dtype=torch.uint8, device=DEV)
    far = np.linspace(2 ** 32 // (Hkv * RECORD) + 1, P - 1, cache.table.shape[1]).astype(np.int32)
    src = up(cache.pool)
    pool[up(far).long()] = src[up(cache.table[0]).long()]
    q = ds.normal_bf16(7371, (2, Hq, D), 2.0)
    lens = np.array([n, n - 1], dtype=np.int32)
    step("pages past 4 GiB")
    out = down_bf16(attn(d, up_bf16(q), pool, up(far[None]), up(lens), up(np.zeros(2, np.int32))))
    ref, tol = attend(cache, q, lens, [0, 0])
    assert (np.abs(bits_to_f64(out) - ref) <= tol).all()
    # appended there, and copied there
    cos, sin = (up(t) for t in ds.rope_tables(n + 1, D))
    x = up_bf16(ds.normal_bf16(7372, (1, (Hq + 2 * Hkv) * D)))
    qb = torch.empty((1, Hq, D), dtype=torch.bfloat16, device=DEV)
    at = up(np.array([n], dtype=np.int32))
    k, v, k2, v2 = (torch.empty((1, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(4))
    near = torch.zeros((2, Hkv, RECORD), dtype=torch.uint8, device=DEV)
    d.det_kv8_rope_append(x, qb, pool, up(far[None]), at, None, cos, sin)
    d.det_kv8_read(pool, up(far[None]), at, None, k, v)
    d.det_kv8_rope_append(x, qb, near, up(np.full((1, far.size), 1, np.int32)), at, None, cos, sin)
    d.det_kv8_read(near, up(np.full((1, far.size), 1, np.int32)), at, None, k2, v2)
    d.det_kv8_copy_pages(pool[None], up(far[-1:]), up(np.array([2 ** 32 // (Hkv * RECORD)], np.int32)))
    torch.cuda.synchronize()
    assert torch.equal(k, k2) and torch.equal(v, v2) and k.float().any()
    assert torch.equal(pool[2 ** 32 // (Hkv * RECORD)], pool[int(far[-1])])


def test_streams_and_graphs(d):
    """Two calls at once on two streams, each with its workspace; one captured call replayed with eager work between; the eager bytes each time."""
    lengths, Hq, Hkv = [777, 64, 1030], 8, 2
    cache = Cache(7380, lengths, Hkv)
    pool, table = up(cache.pool), up(cache.table)
    lens = up(np.array(lengths, np.int32))
    qs = [up_bf16(ds.normal_bf16(7381 + i, (3, Hq, D))) for i in range(2)]
    want = [attn(d, q, pool, table, lens, None) for q in qs]
    torch.cuda.synchronize()
    step("two streams")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    size = d.det_attn_decode_kv8_workspace_bytes(3, Hq, Hkv, D, table.shape[1])
    wss, outs = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in qs], [torch.empty_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(5):
        for q, s, w, o in zip(qs, streams, wss, outs):
            attn(d, q, pool, table, lens, None, stream=s, ws=w, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    step("graph")
    x = up_bf16(ds.normal_bf16(7390, (3, (Hq + 2 * Hkv) * D)))
    cos, sin = (up(t) for t in ds.rope_tables(2048, D))
    q, out = torch.empty((3, Hq, D), dtype=torch.bfloat16, device=DEV), torch.empty((3, Hq, D), dtype=torch.bfloat16, device=DEV)
    at = lens - 1
    k, v = (torch.empty((3, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    src, dst = up(np.array([int(cache.table[0, 0])], np.int32)), up(np.array([cache.pool.shape[0]], np.int32))
    big = torch.cat([pool, torch.zeros_like(pool[:1])])

    def work():
        d.det_kv8_rope_append(x, q, big, table, at, None, cos, sin)
        d.det_attn_decode_kv8(q, big, table, lens, None, out, wss[0], SCALE)
        d.det_kv8_read(big, table, at, None, k, v)
        d.det_kv8_copy_pages(big[None], src, dst)

    work()
    torch.cuda.synchronize()
    eager = [t.clone() for t in (out, k, v, big)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            work()
    for _ in range(4):
        for t in (out, k, v, q):
            t.fill_(float("nan"))
        big[-1] = 0
        wss[0].fill_(0xEE)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, k, v, big), eager))
        assert torch.equal(attn(d, qs[0], pool, table, lens, None), want[0])


# ---------------------------------------------------------------- copies

@pytest.mark.parametrize("layers,P,Hkv,n", [(1, 3, 1, 1), (2, 40, 3, 11), (5, 300, 8, 120)])
def test_copies_move_pages_and_leave_the_others(d, layers, P, Hkv, n):
    rng = np.random.default_rng(n)
    pool = rng.integers(0, 256, (layers, P, Hkv, RECORD), dtype=np.uint8)
    order = rng.permutation(P)
    src, dst = order[:n].astype(np.int32), order[n:2 * n].astype(np.int32)
    src[n // 2:] = src[0]                      # one page forked several times
    pairs_src = np.concatenate([src, [0, -1, P, int(order[-1])]]).astype(np.int32)
    pairs_dst = np.concatenate([dst, [P, int(order[-1]), int(order[-1]), int(order[-1])]]).astype(np.int32)
    if 2 * n == P:
        pairs_src, pairs_dst = src, dst
    dev = up(pool)
    step(f"copy {n} pages of {layers} layers")
    d.det_kv8_copy_pages(dev, up(pairs_src), up(pairs_dst))
    torch.cuda.synchronize()
    pool[:, dst] = pool[:, src]
    assert np.array_equal(dev.cpu().numpy(), pool)
