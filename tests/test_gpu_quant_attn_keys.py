"""GPU: attention over the 8-bit cache, every key and tile of keys of it: values that tell them apart (quant_bound.py), the bound of the row itself."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O
from workloads import gen

from quant_bound import TILE, attend, signed_values, unit_rows, visible, worst_share
from quant_harness import Cache, attn, queries, tree_masks

pytestmark = pytest.mark.gpu


def check(cache, q, L, mask=None, scale=None, dtype="bf16", sequences=None):
    got = attn(cache, q, L, mask, scale, dtype)
    worst, size = worst_share(cache, q, L, got, mask, scale, dtype, sequences)
    print("worst share of the bound %.3f, largest bound %.1e of the outputs" % (worst, size), flush=True)
    assert worst <= 1.0
    return got


# every count of 16-row tiles, both widths and types; flat scores, so that every key has a share that shows
@pytest.mark.parametrize("per", [TILE, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(1, 1), (4, 7), (8, 5), (8, 8), (8, 9), (6, 16), (7, 15), (2, 64)])
def test_every_key_counts(dtype, d, G, n_q, per):
    rng = np.random.default_rng(G * 100 + n_q + per)
    L = np.array([d + 77, 700, 31])
    cache = Cache(rng, 3, 2, d, L + n_q, 16 if per == TILE else None, spread=0.0)
    signed_values(cache, rng, per)
    check(cache, queries(rng, 3, n_q, 2 * G, d, dtype), L, None, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16, 48, 112])
def test_lengths_and_trees(dtype, page):
    rng = np.random.default_rng(52)
    L = np.array([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 121, 500])
    n_q = 7
    cache = Cache(rng, len(L), 2, 128, L + n_q, page, spread=0.0)
    signed_values(cache, rng, 1)
    check(cache, queries(rng, len(L), n_q, 8, 128, dtype), L, tree_masks(rng, len(L), n_q), dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,top,page", [(1, 9000, 16), (1, 9000, None), (5, 3000, 48), (70, 400, 16), (130, 60, 16)])
def test_every_tile_of_every_share(dtype, d, B, top, page):
    """One long unit over all compute units, shares with the end of one unit and the start of the next, more sequences than a wave has lanes."""
    rng = np.random.default_rng(B + d)
    L = rng.integers(max(0, top - 700), top, B)
    n_q = 3
    cache = Cache(rng, B, 2, d, L + n_q, page, spread=0.0)
    signed_values(cache, rng, TILE)
    check(cache, queries(rng, B, n_q, 8, d, dtype), L, dtype=dtype, sequences=None if B < 10 else sorted(rng.choice(B, 24, replace=False).tolist()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_ordinary_rows_within_their_own_bound(dtype, d):
    """Rows of magnitudes of their own, as keys and values have them, peaked and flat."""
    rng = np.random.default_rng(53)
    L = np.array([300, 37, 1100])
    n_q = 5
    cache = Cache(rng, 3, 2, d, L + n_q, 16)
    q = queries(rng, 3, n_q, 8, d, dtype)
    for e in (-3, 0, 2):
        check(cache, np.ldexp(q, e).astype(np.float32), L, dtype=dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_the_lesser_part_of_bf16_queries(d):
    """Lesser parts that all point one way: 6 % of every score."""
    rng = np.random.default_rng(54)
    n_q, n = 3, 64
    cache = Cache(rng, 1, 1, d, [n], None)
    codes, s = O.quant_rows(np.repeat(np.linspace(-2.0, 2.0, n)[:, None], d, 1))
    cache.k[0, 0, :n], cache.ks[0, 0, :n] = codes, s
    signed_values(cache, rng, 1)
    q = np.full((1, n_q, 4, d), 1.0625, np.float32) * np.array([1.0, -1.0, 0.5], np.float32)[None, :, None, None]
    check(cache, q, np.array([n - n_q]), scale=2.0 / d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [-115, -117, -118, -120])
def test_the_smallest_queries(d, e):
    """Rows whose scale byte leaves none for the lesser part, with a scale that makes their scores count."""
    rng = np.random.default_rng(55)
    L = np.array([90])
    cache = Cache(rng, 1, 2, d, L + 4, None, spread=0.0)
    signed_values(cache, rng, 1)
    q = gen.round_to_bf16(np.ldexp(queries(rng, 1, 4, 8, d, "bf16"), e).astype(np.float32))
    check(cache, q, L, scale=np.ldexp(d ** -0.5, -e))
    # and lesser parts that all point one way
    q = np.full((1, 4, 8, d), np.ldexp(1.0625, e), np.float32) * np.where(np.arange(8) % 2, 1.0, -1.0).astype(np.float32)[None, None, :, None]
    codes, s = O.quant_rows(np.repeat(np.linspace(-2.0, 2.0, 94)[:, None], d, 1))
    cache.k[0, :, :94], cache.ks[0, :, :94] = codes, s
    check(cache, q, L, scale=np.ldexp(2.0 / d, -e))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [6, 12, 14, 15, 17])
def test_a_large_query_channel_that_no_key_has(d, r):
    """Keys with a zero where the query's largest value is, 2^r times the others: the scores are what the others make them.  Up to 2^12 nothing is
    lost, beyond it 2^-21 of the large value at most for each of the others."""
    rng = np.random.default_rng(56)
    L = np.array([130])
    cache = Cache(rng, 1, 2, d, L + 3, None, spread=0.0)
    cache.k[..., 5] = 0
    signed_values(cache, rng, 1)
    q = rng.uniform(1.0, 2.0, (1, 3, 8, d)) * rng.choice([-1.0, 1.0], (1, 3, 8, d))
    q[..., 5] = np.ldexp(1.0, r)
    check(cache, gen.round_to_bf16(q.astype(np.float32)), L, scale=0.5 * d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(4, 1), (4, 7), (8, 8), (8, 9), (8, 16)])
def test_a_rows_largest_probability_is_not_rounded(d, G, n_q):
    """One key with a value, a few nats above those before it in its ring: its probability is the reference, 1 in bf16, and the result off by the
    rounding of the output alone, half a step, and by what a score and the sums are off (2^-14 of the result at most: scores of 4 and less, d 2^-23 of
    their largest product for each of two parts, 4000 numbers added in fp32)."""
    rng = np.random.default_rng(57)
    B, Hkv = 8, 4
    L = np.full(B, 4000)
    cache = Cache(rng, B, Hkv, d, L + n_q, None, spread=0.0)
    u = rng.choice([-1.0, 1.0], d)
    q = gen.round_to_bf16((u * rng.uniform(1.0, 1.5, (B, n_q, Hkv * G, 1))).astype(np.float32))
    cache.ks -= 2                                              # scores of the other keys: a quarter of a nat
    cache.v[:] = 0
    for b in range(B):
        p = int(rng.integers(200, 3900))
        codes, s = O.quant_rows(u * rng.uniform(2.0, 3.0, (Hkv, 1)) * d ** -0.5)
        cache.k[b, :, p], cache.ks[b, :, p] = codes, s
        cache.v[b, :, p], cache.vs[b, :, p] = rng.integers(0x38, 0x40, (Hkv, d)), 139
    got = attn(cache, q, L)
    for b in range(B):
        see = visible(int(L[b]), n_q, None).repeat(G, 0)
        for g in range(Hkv):
            k, v = unit_rows(cache, b, g, int(L[b]) + n_q)
            ref = attend(q[b, :, g * G:(g + 1) * G].reshape(n_q * G, d), k, v, see, d ** -0.5)[0]
            half = np.exp2(np.floor(np.log2(ref)) - 8)
            err = np.abs(got[b, :, g * G:(g + 1) * G].reshape(n_q * G, d) - ref)
            assert (err <= half + 2.0 ** -14 * ref).all(), (b, g, float((err / half).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_that_are_not_finite(dtype, d):
    """A query with an infinity or a NaN has scores that are none: its row is NaN, and no other is touched."""
    rng = np.random.default_rng(58)
    L = np.array([300, 20])
    cache = Cache(rng, 2, 2, d, L + 4, 16)
    q = queries(rng, 2, 4, 8, d, dtype)
    clean = attn(cache, q, L, dtype=dtype)
    q[0, 0, 0, 3], q[0, 1, 1, 5], q[1, 2, 2, 7] = np.inf, -np.inf, np.nan
    q[1, 3, 3] = np.inf
    bad = ~np.isfinite(q).all(-1)
    got = attn(cache, q, L, dtype=dtype)
    assert np.isnan(got[bad]).all()
    np.testing.assert_array_equal(got[~bad], clean[~bad])
