"""How far attention over a latent cache may be off, element by element, from the numbers of the row itself; and caches whose values tell every key, or every
tile of keys, from the others."""
from __future__ import annotations

import numpy as np

from target_harness import HALF, U, stored

TILE = 32                              # keys that the bf16 kernels take at a time
GRAN = 64                              # entries of a granule of the work split
FEW, SOME = 160, 512                   # granules (of a sequence's blocks of rows) from which a workgroup takes 32 rows, and all that it can


def granules(lengths, rows, dtype):
    """Granules of a call as its choice of rows counts them; lengths: entries of the sequences, the block's included."""
    most = 16 if rows <= 16 else 32 if rows <= 32 else 64 if rows <= 64 or dtype == "f32" else 128
    return sum(-(-int(n) // GRAN) for n in lengths) * -(-rows // most)


def one_part(lengths, rows, dtype):
    """Whether probabilities are multiplied in one bf16 part."""
    return dtype == "bf16" and rows > 64 and granules(lengths, rows, dtype) >= SOME


def place(lat, b, n):
    """Where the first n entries of a sequence lie."""
    p = np.arange(n)
    return (np.full(n, b), p) if lat.table is None else (lat.table[b, p // lat.page], p % lat.page)


def entries(lat, b, n):
    return lat.c[place(lat, b, n)].astype(np.float64)


def visible(L, n_q, words):
    """[n_q, L + n_q]"""
    see = np.ones((n_q, L + n_q), bool)
    for i in range(n_q):
        word = int(words[i]) if words is not None else (2 << i) - 1
        see[i, L:] = [word >> j & 1 for j in range(n_q)]
    return see


def attend(q, k, r, see, scale):
    """q [R, w], k [n, w], see [R, n]: outputs [R, r], probabilities, scores, in 64 bits; rows that see nothing are zero."""
    s = np.where(see, scale * (np.asarray(q, np.float64) @ k.T), -np.inf)
    top = np.where(see.any(1), s.max(1), 0.0)[:, None]
    p = np.exp(s - top)
    total = p.sum(1, keepdims=True)
    p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
    return p @ k[:, :r], p, s


def row_bounds(q, k, r, see, scale, dtype, single):
    """(outputs in 64 bits, how far off each element may be).

    A score is a sum of w products in w / per steps of `per` of them (32; fp32: 4): (per + w / per + 6) U of the sum of |q_c k_c|, times the scale.  Scale, reference and their
    distance: 4 U (|s| + |s - max|); the exponential and the merges' weights 2^-22 each.  A probability p then is p e^(+-x), which moves an output by sum p (e^x - 1)
    (|v| + |out|) at most, the normaliser being made of the same numbers.  Probabilities of two bf16 parts are off by 2^-16, of one by half a step, 2^-8.  Sums over n
    keys take n / per steps and the merges of rings and segments: (n / per + per + 40) U of sum p |v|, and of |out| for the normaliser.  The result's rounding is half a step."""
    w, n, per = k.shape[1], k.shape[0], 32 if dtype == "bf16" else 4
    out, p, s = attend(q, k, r, see, scale)
    off = scale * (per + w / per + 6) * U * (np.abs(np.asarray(q, np.float64)) @ np.abs(k).T)
    live = np.where(see, s, 0.0)
    top = np.where(see.any(1), s.max(1), 0.0)[:, None]
    off += 4 * U * (np.abs(live) + np.abs(np.where(see, s - top, 0.0))) + 2.0 ** -21
    off += 0.0 if dtype == "f32" else 2.0 ** -8 if single else 2.0 ** -16
    moved = p * np.expm1(off)
    share = 1.0 / np.maximum(1.0 - moved.sum(1, keepdims=True), 1e-3)
    v = np.abs(k[:, :r])
    weighed = p @ v
    bound = share * (moved @ v + moved.sum(1, keepdims=True) * np.abs(out)) + (n / per + per + 40) * U * (weighed + np.abs(out))
    return out, bound + (HALF["bf16"] if dtype == "bf16" else U) * np.abs(out)


def worst_share(lat, q, L, got, mask, scale, dtype, sequences=None):
    """The largest |got - reference| / bound, the norm of the difference over that of the reference, and that of the reference's own rounding to the type."""
    B, n_q, Hq, w = q.shape
    single = one_part(np.asarray(L) + n_q, n_q * Hq, dtype)
    worst, diff, rounding, norm = 0.0, 0.0, 0.0, 0.0
    for b in range(B) if sequences is None else sequences:
        n = int(L[b]) + n_q
        see = visible(int(L[b]), n_q, None if mask is None else mask[b]).repeat(Hq, 0)
        ref, bound = row_bounds(q[b].reshape(n_q * Hq, w), entries(lat, b, n), lat.r, see, scale, dtype, single)
        err = np.abs(got[b].reshape(n_q * Hq, lat.r) - ref)
        assert np.isfinite(err).all()
        worst = max(worst, float(np.max(np.divide(err, bound, out=np.where(err > 0, np.inf, 0.0), where=bound > 0))))
        diff, norm = diff + float((err ** 2).sum()), norm + float((ref ** 2).sum())
        rounding += float(((stored(ref, dtype) - ref) ** 2).sum())
    return worst, (diff / norm) ** 0.5, (rounding / norm) ** 0.5


def telling_values(lat, rng, L, n_q, per):
    """Latents of which column (p // per) mod r alone is not zero, rotated parts as they are: with per = 1 a column belongs to every r-th key, with TILE to every r-th tile, so that
    one lost, doubled or taken from elsewhere changes some column by a large part of it, and one weighed with another key's score by some of it."""
    lat.c[..., :lat.r] = 0
    for b in range(len(L)):
        n = int(L[b]) + n_q
        lat.c[place(lat, b, n) + (np.arange(n) // per % lat.r,)] = rng.choice([1.0, 1.25, 1.5, 1.75], n)
