"""References of the shared prefixes' and page weights' tests: a cache whose sequences hold their first tokens in the same pages, and the pages' weights in
fp64 (both on kv8_ref)."""
import math

import numpy as np

import detsynth as ds
from kv8_ref import PAGE, SCALE, Cache


class SharedCache(Cache):
    """Groups of sequences: group g has rows[g] of them, of lengths[g][i] tokens, and their first common[g] (whole pages) lie in the pages of its first."""

    def __init__(self, seed, Hkv, common, lengths, **more):
        super().__init__(seed, [n for of in lengths for n in of], Hkv, **more)
        self.group_rows = np.cumsum([0] + [len(of) for of in lengths]).astype(np.int32)
        self.shared = np.asarray(common, dtype=np.int32)
        for g, n in enumerate(common):
            b, e = self.group_rows[g], self.group_rows[g + 1]
            assert n % PAGE == 0 and all(x >= n or r > b for r, x in enumerate(self.lengths[b:e], int(b))) and self.lengths[b] >= n
            for r in range(b + 1, e):
                self.table[r, :n // PAGE] = self.table[b, :n // PAGE]
                for x in (self.k, self.v, self.kd, self.vd):
                    x[r, :, :n] = x[b, :, :n]


def page_weights(cache, q_bits, lens, slots, n_slots, max_pages, before, scale=SCALE, gone=None):
    """fp64 weights [n_slots, max_pages] that rows q add to `before`, and how far a result may be from them.

    The allowance of one p is attend's: `rel` of its size.  Sums over a page's 64 tokens (lane sums and four rotations: 2 + 4 additions), the product with
    the row's factor and the factor itself (three roundings with the reciprocal), then R Hq additions in four parts: 2^-24 each of what has been added
    up; and one onto `before`."""
    R, Hq, _ = q_bits.shape
    q = ds.bf16_bits_to_f32(q_bits).astype(np.float64)
    G = Hq // cache.Hkv
    ref, tol = np.zeros((n_slots, max_pages)), np.zeros((n_slots, max_pages))
    for r in range(R):
        n, s = min(int(lens[r]), max_pages * PAGE), int(slots[r])
        if not 0 <= s < n_slots:
            continue
        keep = np.arange(max(n, 0))
        if gone is not None:
            keep = keep[~gone[s, :n]]
        if len(keep) == 0:
            continue
        for h in range(Hq):
            g = h // G
            kc, kd = cache.k[s, g, keep].astype(np.float64), cache.kd[s, g, keep].astype(np.float64)
            x = (kc @ q[r, h]) * kd * scale
            mags = (np.abs(kc) @ np.abs(q[r, h])) * kd * scale
            top = np.abs(q[r, h]).max()
            each = 2.0 ** (math.frexp(top)[1] - 22) if top > 0 else 0.0
            err = 0.5 * each * np.abs(kc).sum(1) * kd * scale + 4 * 2.0 ** -24 * mags
            w = np.exp(x - x.max())
            p = w / w.sum()
            rel = 2 * (err.max() + 2.0 ** -23) + (12 + n / 256) * 2.0 ** -23 + 9 * 2.0 ** -24
            np.add.at(ref[s], keep // PAGE, p)
            np.add.at(tol[s], keep // PAGE, rel * p)
    return before + ref, tol + (R * Hq / 4 + 4) * 2.0 ** -24 * ref + 2.0 ** -24 * (before + ref)
