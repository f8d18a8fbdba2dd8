"""References of the 8-bit cache's tests: the layout of a record, the quantizer in fp32 and attention in fp64, without the library."""
import math

import numpy as np

import detsynth as ds

PAGE, RECORD, D = 64, 16896, 128
SCALE = float(np.float32(1.0 / math.sqrt(128.0)))


def quantize(bits):
    """bf16 rows [..., 128] -> (codes int8, scales fp32) by the written rule, every step an IEEE fp32 operation."""
    x = ds.bf16_bits_to_f32(bits)
    with np.errstate(all="ignore"):
        amax = np.max(np.abs(x), axis=-1)
        d = np.where(np.isfinite(x).all(-1), amax / np.float32(127), np.float32(np.nan)).astype(np.float32)
        c = np.rint(x / np.where(d > 0, d, np.float32(1))[..., None])
    c = np.where((d > 0)[..., None], np.clip(c, -127, 127), 0)
    return c.astype(np.int8), d


def parts(pool):
    """Views of a pool [..., RECORD] of bytes: K codes [..., 64, 128], V codes [..., 4, 128, 16], K and V scales [..., 64]."""
    codes = pool.view(np.int8)
    scales = pool.view(np.float32)
    lead = pool.shape[:-1]
    k, v = codes[..., :PAGE * D].reshape(*lead, PAGE, D), codes[..., PAGE * D:2 * PAGE * D].reshape(*lead, 4, D, 16)
    at = 2 * PAGE * D // 4
    return k, v, scales[..., at:at + PAGE], scales[..., at + PAGE:at + 2 * PAGE]


def store(pool, page, kvh, t, kc, kd, vc, vd):
    """Token t of a page: writes into pool [P, Hkv, RECORD]."""
    rec = pool[page, kvh]
    rec[t * D:(t + 1) * D] = kc.view(np.uint8)
    at = PAGE * D + (t // 16) * (16 * D) + t % 16
    rec[at:at + 16 * D:16] = vc.view(np.uint8)
    f = rec.view(np.float32)
    f[2 * PAGE * D // 4 + t] = kd
    f[2 * PAGE * D // 4 + PAGE + t] = vd


class Cache:
    """Sequences of random tokens, quantized, in pages in no order; bytes that no token owns hold rubbish (NaN scales among it)."""

    def __init__(self, seed, lengths, Hkv, spare=3, std=1.0, extra_pages=1, edit=None):
        self.lengths, self.Hkv = list(lengths), Hkv
        S, longest = len(self.lengths), max(max(lengths), 1)
        k = ds.normal_bf16(seed, (S, Hkv, longest, D), std)
        v = ds.normal_bf16(seed + 1, (S, Hkv, longest, D), std)
        if edit is not None:
            edit(k, v)
        self.k, self.kd = quantize(k)
        self.v, self.vd = quantize(v)
        counts = [-(-n // PAGE) for n in self.lengths]
        rng = np.random.default_rng(seed)
        P = sum(counts) + spare
        order = rng.permutation(P)
        self.table = np.full((S, max(max(counts), 1) + extra_pages), -1, dtype=np.int32)
        pool = rng.integers(0, 256, (P, Hkv, RECORD), dtype=np.uint8)
        pool.view(np.float32)[..., 2 * PAGE * D // 4:] = np.nan
        kp, vp, ks, vs = parts(pool)
        at = 0
        for s, n in enumerate(self.lengths):
            pages = order[at:at + counts[s]]
            at += counts[s]
            self.table[s, :counts[s]] = pages
            for i, page in enumerate(pages):
                m = min(PAGE, n - i * PAGE)
                rows = slice(i * PAGE, i * PAGE + m)
                kp[page, :, :m] = self.k[s, :, rows]
                full = np.zeros((Hkv, PAGE, D), dtype=np.int8)
                full[:, :m] = self.v[s, :, rows]
                keep = np.arange(PAGE).reshape(4, 1, 16) < m
                vp[page] = np.where(keep, full.reshape(Hkv, 4, 16, D).transpose(0, 1, 3, 2), vp[page])
                ks[page, :, :m] = self.kd[s, :, rows]
                vs[page, :, :m] = self.vd[s, :, rows]
        self.pool = pool


def attend(cache, q_bits, lens, slots, scale=SCALE, gone=None):
    """fp64 attention of rows q [R, Hq, 128] and how far a result may be from it, elementwise.

    gone [S, tokens] bool: tokens whose page is missing.  The allowance, with p, v the exact weights and values:
      half a step of bf16 of the result;
      the score: q as integers of step 2^(E-22), off by half a step an element, times the codes and d^K; three fp32 roundings of it (the two
      digit sums joined, the factor, the scale), each 2^-24 of the magnitudes that enter, and the rounding of scale * log2 e; the exponential one unit in
      the last place.  A score's error x moves a weight by the factor exp(x), and the normalized weight by twice that;
      the weights as integers: half a step of 2^(E-22) of the chunk's largest, at most 2^-22 of the row's largest weight a token;
      fp32 sums over the chunk and over the chunks: 2^-24 each for about 10 + chunks additions."""
    R, Hq, _ = q_bits.shape
    q = ds.bf16_bits_to_f32(q_bits).astype(np.float64)
    G = Hq // cache.Hkv
    ref, tol = np.zeros((R, Hq, D)), np.zeros((R, Hq, D))
    for r in range(R):
        n, s = int(lens[r]), int(slots[r])
        keep = np.arange(n)
        if gone is not None:
            keep = keep[~gone[s, :n]]
        if len(keep) == 0:
            continue
        for g in range(cache.Hkv):
            kc, vc = cache.k[s, g, keep].astype(np.float64), cache.v[s, g, keep].astype(np.float64)
            kd, vd = cache.kd[s, g, keep].astype(np.float64), cache.vd[s, g, keep].astype(np.float64)
            for h in range(g * G, (g + 1) * G):
                x = (kc @ q[r, h]) * kd * scale
                mags = (np.abs(kc) @ np.abs(q[r, h])) * kd * scale
                top = np.abs(q[r, h]).max()
                step = 2.0 ** (math.frexp(top)[1] - 22) if top > 0 else 0.0
                err = 0.5 * step * np.abs(kc).sum(1) * kd * scale + 4 * 2.0 ** -24 * mags
                w = np.exp(x - x.max())
                p = w / w.sum()
                rel = 2 * (err.max() + 2.0 ** -23) + (12 + n / 256) * 2.0 ** -23
                o, oabs = p @ (vc * vd[:, None]), p @ (np.abs(vc) * vd[:, None])
                ref[r, h] = o
                tol[r, h] = 2.0 ** -8 * np.abs(o) + rel * oabs + 2.0 ** -22 * (p * vd).max() * np.abs(vc).sum(0)
    return ref, tol
