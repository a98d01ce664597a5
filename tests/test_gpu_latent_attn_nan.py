"""GPU: scores of a latent cache that are no number reach every row that sees them, whatever the rest of the row weighs."""
import numpy as np
import pytest

from target_harness import run_latent_attn
from test_gpu_latent_attn import case

pytestmark = pytest.mark.gpu

# rows of a sequence and entries of the contexts: blocks of 16 rows with four rings of keys, of 32 with two, of 64, and of up to 128
SHAPES = [(3, 4, [300, 700]), (4, 16, [300, 9000]), (8, 16, [300, 5000]), (2, 20, [300, 11000]), (4, 16, [300, 33000]), (8, 16, [300, 33000]), (1, 72, [300, 33000])]


def put(lat, b, entries, column, value):
    for p in entries:
        lat.c[lat.at(b, p)][column] = value


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 64])
@pytest.mark.parametrize("every", [1, 4])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_segment_without_a_number(dtype, page, every, shape):
    """64 entries with a NaN in each, or in one of the four that a lane has of sixteen: the maximum of their scores then knows no number."""
    n_q, Hq, L = SHAPES[shape]
    lat, q, L, _, scale = case(shape, 2, n_q, Hq, 128, L, dtype, page)
    put(lat, 1, range(0, 64, every), 3, np.nan)
    got = run_latent_attn(lat.gpu()[0], 2, n_q, Hq, 128, q, L, None, scale, dtype)
    assert np.isnan(got[1]).all() and np.isfinite(got[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [128, 512])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_nan_among_entries_that_weigh_nothing(dtype, r, shape):
    """448 entries whose scores are 800 binary digits below the others', more than a weight's exponent has, one of them a NaN in its rotated part."""
    n_q, Hq, L = SHAPES[shape]
    lat, q, L, _, scale = case(shape, 2, n_q, Hq, r, L, dtype)
    q[..., r] = 8.0
    for b in range(2):
        put(lat, b, range(int(L[b]) + n_q), r, 0.0)
    put(lat, 1, range(448), r, -1000.0)                   # 0.07 * 8 * 1000 / ln 2
    put(lat, 1, [5], r + 1, np.nan)
    got = run_latent_attn(lat.gpu()[0], 2, n_q, Hq, r, q, L, None, scale, dtype)
    assert np.isnan(got[1]).all() and np.isfinite(got[0]).all()
