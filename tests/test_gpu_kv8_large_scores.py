"""Attention over the 8-bit cache with scores of any size that fp32 holds, in every form."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, bits_to_f64, down_bf16, step, up, up_bf16
from kv8_ref import D, SCALE, Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    import paper_2602_00182_amd as d
    return d


@pytest.mark.parametrize("R,Hq,Hkv,named,mixed", [(6, 4, 2, False, False), (6, 16, 2, False, False), (6, 4, 2, True, False), (500, 32, 8, True, False),
                                                  (500, 32, 8, True, True)])  # mixed: tiles that walk alone
@pytest.mark.parametrize("exponent", [20, 24, 30, 36, 60, 100])
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_of_large_scores_takes_all(d, R, Hq, Hkv, named, mixed, exponent, sign):
    """Scores of about 2^exponent; the largest stands out by far more than a score's rounding (checked here: three fp32 roundings, each 2^-24 of the sum
    of magnitudes, and the query's 2^-22), so its token has the weight 1 and the others 0.  Then the result is the token's value: e <= 1 has two
    roundings of 2^-24 beside its quotient's, the weight as an integer of 22 bits half a step of at most 2^-21, and bf16 rounds by 2^-8.  With sign -1 all
    keys point away from the query: every score is below zero."""
    lengths = [300, 64, 700, 257, 513, 130]
    G = Hq // Hkv

    def edit(k, v):
        x = np.abs(ds.bf16_bits_to_f32(k)) + np.float32(0.5)
        k[:] = ds.f32_to_bf16_bits(x * np.float32(sign * 2.0 ** (exponent // 2)))
    cache = Cache(7800 + exponent, lengths, Hkv, edit=edit)
    rng = np.random.default_rng(exponent)
    if not named:
        slots = np.arange(R)
    else:
        slots = rng.integers(0, len(lengths), R)
        if not mixed:
            slots.sort()
    slots = slots.astype(np.int32)
    lens = np.array([lengths[s] if i % 3 else rng.integers(1, lengths[s] + 1) for i, s in enumerate(slots)], dtype=np.int32)
    q = ds.f32_to_bf16_bits((np.abs(ds.bf16_bits_to_f32(ds.normal_bf16(7801, (R, Hq, D)))) + np.float32(0.5)) * np.float32(2.0 ** (exponent - exponent // 2 - 4)))
    ref, size, clear = np.zeros((R, Hq, D)), np.zeros((R, Hq)), np.zeros((R, Hq), dtype=bool)
    qf = ds.bf16_bits_to_f32(q).astype(np.float64)
    for r in range(R):
        s, n = slots[r], lens[r]
        for h in range(Hq):
            g = h // G
            kc, kd = cache.k[s, g, :n].astype(np.float64), cache.kd[s, g, :n].astype(np.float64)
            x = (kc @ qf[r, h]) * kd * SCALE
            top = int(x.argmax())
            gap = x[top] - np.partition(x, -2)[-2] if n > 1 else np.inf
            clear[r, h] = gap > 200 + 2.0 ** -20 * (np.abs(kc) @ np.abs(qf[r, h]) * kd * SCALE).max()
            ref[r, h] = cache.v[s, g, top].astype(np.float64) * float(cache.vd[s, g, top])
            size[r, h] = abs(x[top])
    assert clear.mean() > (0.9 if exponent > 24 else 0.5) and np.median(size) > 2.0 ** (exponent - 4)
    ws = torch.empty(d.det_attn_decode_kv8_workspace_bytes(R, Hq, Hkv, D, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
    out = torch.full((R, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    step(f"scores of 2^{exponent}, sign {sign}, {R} rows, {Hq}/{Hkv} heads, named {named}, mixed {mixed}")
    dev = [up_bf16(q), up(cache.pool), up(cache.table), up(lens), up(slots)]
    d.det_attn_decode_kv8(*dev[:4], dev[4] if named else None, out, ws, SCALE)
    torch.cuda.synchronize()
    got = bits_to_f64(down_bf16(out))
    assert (np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -20) * np.abs(ref))[clear].all()
    assert np.isfinite(got).all()
    for r in range(0, R, max(1, R // 6)):  # a row alone
        one = torch.empty_like(out[:1])
        d.det_attn_decode_kv8(dev[0][r:r + 1], dev[1], dev[2], dev[3][r:r + 1], dev[4][r:r + 1], one, ws, SCALE)
        assert torch.equal(one[0], out[r])
