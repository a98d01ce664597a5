"""How far attention over the 8-bit cache may be off, element by element, from the numbers of the row itself; and caches whose values
tell every tile of keys, or every key, from the others."""
from __future__ import annotations

import numpy as np

from oracle import specexit_oracle as O

TILE = 32               # keys that the kernels take at a time


def unit_rows(cache, b, g, n):
    """K and V of the first n entries of a sequence's KV head, [n, d] each."""
    p = np.arange(n)
    at = (b, g, p) if cache.table is None else (cache.table[b, p // cache.page], g, p % cache.page)
    return O.dequant_rows(cache.k[at], cache.ks[at]), O.dequant_rows(cache.v[at], cache.vs[at])


def visible(L, n_q, mask_row):
    """[n_q, L + n_q] of truth values."""
    words = mask_row if mask_row is not None else [(2 << i) - 1 for i in range(n_q)]
    see = np.ones((n_q, L + n_q), bool)
    for i, w in enumerate(words):
        see[i, L:] = [int(w) >> j & 1 for j in range(n_q)]
    return see


def attend(q, k, v, see, scale):
    """q [R, d], see [R, n] -> outputs [R, d], probabilities [R, n], scores; in 64 bits, rows that see nothing are zero."""
    s = np.where(see, scale * (np.asarray(q, np.float64) @ k.T), -np.inf)
    top = np.where(see.any(1), s.max(1), 0.0)
    p = np.exp(s - top[:, None])
    total = p.sum(1, keepdims=True)
    p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
    return p @ v, p, s


def row_bounds(q, k, v, see, scale, dtype):
    """(outputs in 64 bits, how far off each element may be) of R rows of one unit.

    A score is off by (e = 2^-23, products |q_c k_c| of the d columns, all times `scale`)
      bf16: what the instruction drops, e of the largest product for each of the d, of both parts of the queries, the lesser of which is a
            sixteenth: 17/16 d e max; what the two parts do not hold of an element below 2^-13 of the row's largest m, at most m / 224 / 2^14; two
            roundings of the sum: 2 e sum
      fp32: e of the largest product for each of the d, of parts that are 1, 2^-8, 2^-16: 1.01 d e max; four roundings of sums of three parts: 4 e sum
    and, in both, by its product with the scale and the difference to the row's reference, 2 e (|s| + |s - max|), and the exponential's and
    the merge's roundings, 4 e.  A probability p then is p e^(+-x), which moves an output by sum p (e^x - 1) (|v| + |out|) at most.  Sums over
    n keys are made of n / 32 steps (three of fp32) of 32 products, each off by e / 2: (3 n / 32 + 96) e / 2 of sum p |v|.  Roundings of half a step:
    bf16 probabilities and outputs 2^-8 each; fp32 probabilities 2^-24, outputs (a division) 2^-23."""
    e = 2.0 ** -23
    q = np.asarray(q, np.float64)
    out, p, s = attend(q, k, v, see, scale)
    aq, ak = np.abs(q), np.abs(k)
    d, n = k.shape[1], k.shape[0]
    total = aq @ ak.T
    largest = np.stack([(ak * r).max(1) for r in aq])
    m = aq.max(1, keepdims=True)
    if dtype == "bf16":
        lost = np.where((aq > 0) & (aq < m * 2.0 ** -13), m / 224 * 2.0 ** -14, 0.0)
        off = scale * (17 / 16 * d * e * largest + lost @ ak.T + 2 * e * total)
    else:
        off = scale * (1.01 * d * e * largest + 4 * e * total)
    live = np.where(see, s, 0.0)
    top = np.where(see.any(1), np.where(see, s, -np.inf).max(1), 0.0)[:, None]
    off = off + 2 * e * (np.abs(live) + np.abs(np.where(see, s - top, 0.0))) + 4 * e
    moved = p * np.expm1(off)
    share = 1.0 / np.maximum(1.0 - moved.sum(1, keepdims=True), 1e-3)
    weighed = p @ np.abs(v)
    bound = share * (moved @ np.abs(v) + moved.sum(1, keepdims=True) * np.abs(out))
    bound += (3 * n / 32 + 96) * e / 2 * (weighed + np.abs(out))
    bound += 2.0 ** -8 * (weighed + np.abs(out)) if dtype == "bf16" else 2.0 ** -24 * weighed + e * np.abs(out)
    return out, bound


def worst_share(cache, q, L, got, mask=None, scale=None, dtype="bf16", sequences=None):
    """The largest |got - reference| / bound, and the largest bound over the outputs' root mean square."""
    B, n_q, Hq, d = q.shape
    G = Hq // cache.Hkv
    scale = d ** -0.5 if scale is None else scale
    worst, size, square, count = 0.0, 0.0, 0.0, 0
    for b in range(B) if sequences is None else sequences:
        n = int(L[b]) + n_q
        see = visible(int(L[b]), n_q, None if mask is None else mask[b]).repeat(G, 0)
        for g in range(cache.Hkv):
            k, v = unit_rows(cache, b, g, n)
            rows = q[b, :, g * G:(g + 1) * G].reshape(n_q * G, d)
            ref, bound = row_bounds(rows, k, v, see, scale, dtype)
            err = np.abs(got[b, :, g * G:(g + 1) * G].reshape(n_q * G, d) - ref)
            assert not np.isnan(err).any()
            worst = max(worst, float(np.max(np.divide(err, bound, out=np.where(err > 0, np.inf, 0.0), where=bound > 0))))
            size, square, count = max(size, float(bound.max())), square + float((ref ** 2).sum()), count + ref.size
    return worst, size / max((square / count) ** 0.5, 1e-300)


def signed_values(cache, rng, per):
    """V codes of which column (p // per) mod d alone is not zero in a row: with per = TILE a column belongs to the keys of every d-th tile, with 1
    to every d-th key, so that a tile or key lost, doubled or taken from elsewhere changes some column by a large part of it."""
    cache.v[:] = 0
    cache.vs[:] = rng.integers(126, 129, cache.vs.shape)
    for b in range(cache.B):
        n = cache.k.shape[2] if cache.table is None else cache.table.shape[1] * cache.page
        for p in range(n):
            if cache.table is None or p // cache.page < cache.table.shape[1]:
                at, heads, j = cache.at(b, p)
                cache.v[at, :, j, p // per % cache.d] = rng.integers(0x38, 0x40, cache.Hkv)
