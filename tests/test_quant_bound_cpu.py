"""The bound that the tests of the 8-bit cache's attention use lets arithmetic of the kernels' kind pass and none of the faults planted here (no GPU)."""
import numpy as np
import pytest

from oracle import specexit_oracle as O
from workloads import gen

from quant_bound import TILE, attend, row_bounds, signed_values, unit_rows, visible, worst_share
from quant_harness import Cache, queries, tree_masks


def like_the_kernel(q, k, v, see, scale, dtype):
    """The outputs with the kernels' roundings: queries in two parts of four bits, probabilities in bf16 (fp32 ones as they are), the result's type."""
    if dtype == "bf16":
        q = sum(two_parts(q))
    s = np.where(see, (scale * (q @ k.T)).astype(np.float32).astype(np.float64), -np.inf)
    p = np.exp(s - s.max(1, keepdims=True))
    w = gen.round_to_bf16(p.astype(np.float32)).astype(np.float64) if dtype == "bf16" else p.astype(np.float32)
    out = ((w @ v) / p.sum(1, keepdims=True)).astype(np.float32)
    return gen.round_to_bf16(out) if dtype == "bf16" else out


def two_parts(q):
    c, s = O.quant_rows(q)
    first = O.dequant_rows(c, s)
    unit = np.ldexp(1.0, s.astype(int) - 127)[..., None]
    rest = (np.asarray(q, np.float64) - first) * 16 / unit
    grid = np.concatenate([-O.E4M3[126::-1], O.E4M3[1:127]])
    return first, grid[np.abs(rest[..., None] - grid).argmin(-1)] / 16 * unit


def case(seed, n, rows, d, dtype, per, spread=0.0):
    rng = np.random.default_rng(seed)
    cache = Cache(rng, 1, 1, d, [n], None, spread=spread)
    signed_values(cache, rng, per)
    k, v = unit_rows(cache, 0, 0, n)
    q = queries(rng, 1, 1, rows, d, dtype)[0, 0]
    return rng, q, k, v, np.ones((rows, n), bool), d ** -0.5


def share(bad, ref, bound):
    err = np.abs(bad - ref)                    # (a column without keys is 0, and so is its bound)
    return float(np.max(np.divide(err, bound, out=np.where(err > 0, np.inf, 0.0), where=bound > 0)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,n", [(64, 700), (128, 300), (128, 9000)])
def test_the_kernels_arithmetic_passes(dtype, d, n):
    for per in (TILE, 1):
        _, q, k, v, see, scale = case(1, n, 5, d, dtype, per)
        ref, bound = row_bounds(q, k, v, see, scale, dtype)
        assert share(like_the_kernel(q, k, v, see, scale, dtype), ref, bound) <= 1.0
        # and the bound says something: of fp32 results 1e-4 of their size at most (sums of 9000 entries are 2 (3 9000 / 32 + 96) 2^-24 = 1.1e-4 of it
        # by themselves), of bf16 ones two per cent
        assert (bound <= (2e-2 if dtype == "bf16" else 1e-4 if n < 1000 else 2e-4) * np.abs(ref).max()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,n", [(64, 1040), (128, 333), (128, 9000)])
def test_no_tile_can_be_lost_or_taken_twice(dtype, d, n):
    _, q, k, v, see, scale = case(2, n, 3, d, dtype, TILE)
    ref, bound = row_bounds(q, k, v, see, scale, dtype)
    w = np.exp(scale * (q.astype(np.float64) @ k.T))
    for t in range((n + TILE - 1) // TILE):
        a = slice(t * TILE, min(n, (t + 1) * TILE))
        part, mass = w[:, a] @ v[a], w[:, a].sum(1, keepdims=True)
        for sign in (-1.0, 1.0):
            bad = (w @ v + sign * part) / (w.sum(1, keepdims=True) + sign * mass)
            assert share(bad, ref, bound) > 1.0, (t, sign)
        other = slice((t * TILE + 5 * TILE) % (n - TILE), (t * TILE + 5 * TILE) % (n - TILE) + a.stop - a.start)
        bad = (w @ v - part + w[:, other] @ v[other]) / (w.sum(1, keepdims=True) - mass + w[:, other].sum(1, keepdims=True))
        assert share(bad, ref, bound) > 1.0, t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,n", [(64, 60), (128, 700)])
def test_no_key_can_be_lost(dtype, d, n):
    _, q, k, v, see, scale = case(3, n, 4, d, dtype, 1)
    ref, bound = row_bounds(q, k, v, see, scale, dtype)
    for j in range(n):
        fewer = see.copy()
        fewer[:, j] = False
        assert share(attend(q, k, v, fewer, scale)[0], ref, bound) > 1.0, j


@pytest.mark.parametrize("d", [64, 128])
def test_fp32_operands_cannot_be_rounded_to_bf16(d):
    _, q, k, v, see, scale = case(4, 500, 4, d, "f32", 1)
    ref, bound = row_bounds(q, k, v, see, scale, "f32")
    assert share(attend(gen.round_to_bf16(q), k, v, see, scale)[0], ref, bound) > 20.0
    assert share(gen.round_to_bf16(ref.astype(np.float32)), ref, bound) > 20.0
    s = scale * (q.astype(np.float64) @ k.T)
    p = np.exp(s - s.max(1, keepdims=True))
    assert share(gen.round_to_bf16(p.astype(np.float32)) @ v / p.sum(1, keepdims=True), ref, bound) > 20.0


@pytest.mark.parametrize("d", [64, 128])
def test_the_lesser_part_of_bf16_queries_counts(d):
    q, k, v, scale = aligned(d)
    see = np.ones((q.shape[0], k.shape[0]), bool)
    ref, bound = row_bounds(q, k, v, see, scale, "bf16")
    first, second = two_parts(q)
    np.testing.assert_array_equal(first + second, q)
    assert share(like_the_kernel(q, k, v, see, scale, "bf16"), ref, bound) <= 1.0
    assert share(attend(first, k, v, see, scale)[0], ref, bound) > 4.0
    for wrong in (0.5, 2.0):
        assert share(attend(first + wrong * second, k, v, see, scale)[0], ref, bound) > 2.0


def aligned(d):
    """Queries whose lesser parts all point one way, keys that are alike in all columns: the lesser part is 6 % of every score."""
    q = np.full((3, d), 1.0625) * np.array([[1.0], [-1.0], [0.5]])
    m = np.linspace(-2.0, 2.0, 64)
    codes, s = O.quant_rows(np.repeat(m[:, None], d, 1))
    v = np.zeros((64, d))
    v[np.arange(64), np.arange(64) % d] = 1.0
    return q, O.dequant_rows(codes, s), v, 2.0 / d


def test_the_reference_is_the_oracles():
    rng = np.random.default_rng(7)
    L, n_q = np.array([0, 33, 100]), 5
    for page in (None, 16, 48):
        cache = Cache(rng, 3, 2, 64, L + n_q, page)
        q = queries(rng, 3, n_q, 6, 64, "f32")
        for mask in (None, tree_masks(rng, 3, n_q)):
            k, v = cache.values()
            ref = O.verify_attn(q, k, v, L, mask, None, cache.table, page or 16)
            assert worst_share(cache, q, L, ref, mask, None, "f32")[0] < 1e-6


@pytest.mark.parametrize("d", [64, 128])
def test_what_the_two_parts_of_a_query_hold(d):
    """Exact from 2^-13 of the row's largest magnitude on; below, off by 2^-21 of it at most, and that is met."""
    rng = np.random.default_rng(8)
    q = rng.uniform(1.0, 2.0, (400, d)) * np.exp2(-rng.integers(0, 30, (400, d)))
    q[:, 3] = rng.uniform(1.0, 2.0, 400)
    q = gen.round_to_bf16(q.astype(np.float32)).astype(np.float64)
    m = q.max(1, keepdims=True)
    off = np.abs(sum(two_parts(q)) - q)
    assert (off[q >= m * 2.0 ** -13] == 0).all()
    assert (off <= m / 224 * 2.0 ** -14).all() and (off <= m * 2.0 ** -21).all()
    assert (off > m * 2.0 ** -23).any()
