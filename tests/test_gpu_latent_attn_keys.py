"""GPU: latent attention, every key and tile of keys of it: values that tell them apart and the bound of the row itself (latent_bound.py); the digits that
probabilities, entries and sums keep; references that a segment's scores leave behind, at every width."""
import numpy as np
import pytest

from latent_bound import FEW, GRAN, SOME, TILE, attend, entries, granules, one_part, place, row_bounds, telling_values, visible, worst_share
from target_harness import run_latent_attn, stored
from test_gpu_latent_attn import case

pytestmark = pytest.mark.gpu


def check(lat, q, L, mask, scale, dtype, sequences=None):
    B, n_q, Hq, _ = q.shape
    got = run_latent_attn(lat.gpu()[0], B, n_q, Hq, lat.r, q, L, mask, scale, dtype)
    worst, err, rounding = worst_share(lat, q, L, got, mask, scale, dtype, sequences)
    print("worst share of the bound %.3f, error %.2e, a rounding %.2e" % (worst, err, rounding), flush=True)
    assert worst <= 1.0
    return got, err, rounding


def telling(seed, B, n_q, Hq, r, L, dtype, page, per, tree=False):
    """Scores within about one of each other, so that every key has a share that shows."""
    rng = np.random.default_rng(seed)
    lat, q, L, mask, _ = case(seed, B, n_q, Hq, r, L, dtype, page, tree)
    telling_values(lat, rng, L, n_q, per)
    return lat, q, L, mask, 0.05


ROWS = [(1, 1), (1, 16), (4, 8), (3, 11), (4, 16), (5, 13), (7, 16), (8, 16), (2, 70), (9, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [128, 256, 512])
@pytest.mark.parametrize("rows", range(len(ROWS)))
def test_every_key_counts(dtype, r, rows):
    """Few granules: rings of one and of two waves."""
    n_q, Hq = ROWS[rows]
    lat, q, L, mask, scale = telling(rows, 5, n_q, Hq, r, [0, 1, 31, 65, 700], dtype, [None, 16, 48][rows % 3], 1, tree=n_q > 2 and rows % 2 == 0)
    check(lat, q, L, mask, scale, dtype)


# rows, contexts: more granules than FEW and than SOME, one long sequence and several, some of them with hardly anything
LONG = [((1, 20), [11000]), ((4, 8), [6000, 0, 5000]), ((3, 11), [33500]), ((4, 16), [12000, 70, 21000]), ((5, 13), [33000]), ((7, 16), [20000, 13500]), ((8, 16), [33001, 31]),
        ((9, 16), [17000]), ((9, 33), [11100, 200])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,page", [(128, 64), (512, None), (512, 64)])
@pytest.mark.parametrize("shape", range(len(LONG)))
def test_every_tile_of_long_contexts(dtype, r, page, shape):
    (n_q, Hq), L = LONG[shape]
    lat, q, L, mask, scale = telling(40 + shape, len(L), n_q, Hq, r, L, dtype, page, TILE, tree=n_q > 4)
    assert granules(L + n_q, n_q * Hq, dtype) >= (FEW if n_q * Hq <= 32 else SOME)
    check(lat, q, L, mask, scale, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,Hq,r,page", [(1, 20, 128, 16), (4, 16, 256, 48), (7, 16, 512, 16), (8, 16, 128, None), (9, 15, 256, 32)])
def test_every_tile_of_many_sequences(dtype, n_q, Hq, r, page):
    """More sequences than a wave has lanes, shares that end one unit and begin the next."""
    L = [0, 1, 2, 31, 33, 64, 127] + [400 + 37 * b % 361 for b in range(64)]
    lat, q, L, mask, scale = telling(60 + Hq, len(L), n_q, Hq, r, L, dtype, page, 1, tree=n_q == 7)
    assert granules(L + n_q, n_q * Hq, dtype) >= SOME
    check(lat, q, L, mask, scale, dtype, sequences=[0, 1, 3, 6, 7, 20, 41, 63, 64, 65, 70])


@pytest.mark.parametrize("Hq", [32, 64, 128])
@pytest.mark.parametrize("gran", [FEW - 1, FEW, FEW + 1, SOME - 1, SOME, SOME + 1])
def test_every_tile_where_the_rows_of_a_block_change(Hq, gran):
    """One sequence whose last granule is full, one short of that, or a single entry."""
    for extra in (0, -1, 1 - GRAN):
        lat, q, L, mask, scale = telling(gran, 1, 1, Hq, 128, [GRAN * gran + extra - 1], "bf16", 64, TILE)
        assert granules(L + 1, Hq, "bf16") == gran and one_part(L + 1, Hq, "bf16") == (Hq > 64 and gran >= SOME)
        check(lat, q, L, mask, scale, "bf16")


# rows and contexts below and above the lengths where the rows of a block change
DIGITS = [((1, 3), [9000]), ((1, 16), [700, 3000]), ((2, 16), [900, 12000]), ((4, 16), [3000]), ((4, 16), [40000]), ((7, 16), [4096]), ((8, 16), [20000]), ((1, 128), [32000]), ((8, 16), [500, 33000])]


@pytest.mark.parametrize("r", [128, 512])
@pytest.mark.parametrize("shape", range(len(DIGITS)))
def test_fp32_entries_and_probabilities_keep_their_digits(r, shape):
    """Roundings of 32 bits do not all point one way.  Of a score of w = r + 64 products, w / 4 steps of four: sqrt(w / 4 + 10) U of what it comes to on its way, three at most here; the
    exponential 2^-22; sums over 64 to 40000 keys, sqrt(n / 4 + 100) U: 7e-6 together at most.  Probabilities, queries or entries of 16 bits (2^-16) would be some 10^-5 each, of 8 bits 10^-3."""
    (n_q, Hq), L = DIGITS[shape]
    lat, q, L, mask, scale = case(80 + shape, len(L), n_q, Hq, r, L, "f32", 64 if shape % 2 else None)
    _, err, _ = check(lat, q, L, mask, 0.05, "f32")
    assert err <= 7e-6


@pytest.mark.parametrize("r", [128, 512])
@pytest.mark.parametrize("shape", range(len(DIGITS)))
def test_bf16_probabilities_have_two_parts_where_they_should(r, shape):
    """With two parts what is left of the error is the result's rounding to bf16.  One part is off by as much once more, independently (probabilities of a row are rounded like
    results): at most sqrt(2) times that."""
    (n_q, Hq), L = DIGITS[shape]
    lat, q, L, mask, scale = case(80 + shape, len(L), n_q, Hq, r, L, "bf16", 64 if shape % 2 else None)
    single = one_part(L + n_q, n_q * Hq, "bf16")
    assert single == (shape == 8)                 # (500 + 1 granules and less in front of it: 32001 entries; 8 + 516 there)
    _, err, rounding = check(lat, q, L, mask, 0.05, "bf16")
    assert err < (1.05 * 2 ** 0.5 if single else 1.05) * rounding


def segments(n, rows):
    """Key ranges of the workgroups of one sequence of n entries, one block of rows, 256 workgroups at least on the card; two granules of nothing in front."""
    T = -(-n // GRAN) + 2
    most = -(-T // 256)
    W = -(-T // most)
    cut = [(max(w * T // W - 2, 0) * GRAN, min(n, ((w + 1) * T // W - 2) * GRAN)) for w in range(W)]
    return [(a, z) for a, z in cut if z > a]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,page", [(128, None), (256, 64), (512, None), (512, 64)])
@pytest.mark.parametrize("n_q,Hq", [(4, 16), (8, 16)])
@pytest.mark.parametrize("height", [40.0, 150.0])
def test_references_left_behind(dtype, r, page, n_q, Hq, height):
    """Scores that rise and fall over 256 entries by up to 120 binary digits: further, within a segment, than the reference of its first tile reaches (60), or, with a height of 40, not as far."""
    lat, q, L, mask, scale = case(r, 1, n_q, Hq, r, [64 * 600 + 5], dtype, page)
    q = q * np.float32(0.25)
    q[..., r] = 8.0
    n = int(L[0]) + n_q
    lat.c[place(lat, 0, n) + (r,)] = stored(height * (np.arange(n) % 256) / 256, "bf16")
    _, _, s = attend(q.reshape(n_q * Hq, -1), entries(lat, 0, n), r, visible(int(L[0]), n_q, None).repeat(Hq, 0), scale / np.log(2.0))
    rise = max(float((s[:, a:z].max(1) - s[:, a:min(a + TILE, z)].max(1)).max()) for a, z in segments(n, n_q * Hq))
    assert rise > 70 if height > 100 else 8 < rise < 50
    check(lat, q, L, mask, scale, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,page", [(128, None), (256, 64), (512, None), (512, 64)])
@pytest.mark.parametrize("n_q,Hq", [(4, 16), (8, 16)])
def test_hidden_and_visible_values_that_are_not_finite_behind_long_contexts(dtype, r, page, n_q, Hq):
    """What no row sees may be anything; a NaN that some rows see reaches those; an infinite key is a NaN or the whole probability: NaN either way, since it is the value as well."""
    lat, q, L, _, scale = case(r + 1, 3, n_q, Hq, r, [12000, 33000, 300], dtype, page)
    words = [(1 << i) | 1 for i in range(n_q)]
    words[2] = 5 | 1 << (n_q - 1)                 # the row that sees the block's last entry, beside its own
    words[n_q - 1] = 1
    mask = np.tile(np.array(words, np.uint64), (3, 1))
    clean = lat.c.copy()
    hidden = 1                                    # entry 1 of the block is row 1's own: taken out of its word here
    mask[:, 1] = 1
    for b, value in enumerate((np.nan, np.inf, -np.inf)):
        lat.c[lat.at(b, int(L[b]) + hidden)] = value
    lat.c[lat.at(0, int(L[0]) + n_q - 1)][7] = np.nan
    lat.c[lat.at(2, 17)][r + 5] = np.inf
    got = run_latent_attn(lat.gpu()[0], 3, n_q, Hq, r, q, L, mask, scale, dtype)
    assert np.isnan(got[0, 2]).all()
    # an infinite score: NaN (its own weight is infinity over infinity), or nothing at all where it is minus infinity
    sign = np.sign(q[2, ..., r + 5])
    assert np.isnan(got[2][sign > 0]).all()
    seen = visible(300, n_q, mask[2]).repeat(Hq, 0)
    lat.c = clean
    seen[:, 17] = False
    ref, _, _ = attend(q[2].reshape(n_q * Hq, -1), entries(lat, 2, 300 + n_q), r, seen, scale)
    ref = ref.reshape(n_q, Hq, r)
    assert np.abs(got[2] - ref)[sign < 0].max() < (2e-2 if dtype == "bf16" else 1e-4)
    got[0, 2] = 0
    for b, rows in ((0, [i for i in range(n_q) if i != 2]), (1, list(range(n_q)))):
        keep = np.zeros(n_q, bool)
        keep[rows] = True
        ref, bound = _bounds(lat, q, L, mask, scale, dtype, b)
        assert (np.abs(got[b] - ref) <= bound)[keep].all()


def _bounds(lat, q, L, mask, scale, dtype, b):
    B, n_q, Hq, w = q.shape
    n = int(L[b]) + n_q
    see = visible(int(L[b]), n_q, mask[b]).repeat(Hq, 0)
    ref, bound = row_bounds(q[b].reshape(n_q * Hq, w), entries(lat, b, n), lat.r, see, scale, dtype, one_part(np.asarray(L) + n_q, n_q * Hq, dtype))
    return ref.reshape(n_q, Hq, -1), bound.reshape(n_q, Hq, -1)
