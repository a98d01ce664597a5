"""The bound that the tests of the latent attention's keys use lets arithmetic of the kernels' kind pass and none of the faults planted here (no GPU)."""
import numpy as np
import pytest

from latent_bound import TILE, attend, granules, one_part, row_bounds, telling_values
from target_harness import Latent, stored
from workloads import gen


def case(seed, n, rows, r, dtype, per):
    rng = np.random.default_rng(seed)
    lat = Latent(rng, 1, r, [n], dtype)
    if per:
        telling_values(lat, rng, [n - 1], 1, per)
    return rng, stored(rng.standard_normal((rows, r + 64)), dtype), lat.c[0].astype(np.float64), np.ones((rows, n), bool), 0.05


def like_the_kernel(q, k, r, scale, dtype, single):
    """The outputs with the kernels' roundings, one after the other."""
    s = (np.asarray(q, np.float64) @ k.T).astype(np.float32) * np.float32(scale)
    p = np.exp((s - s.max(1, keepdims=True)).astype(np.float64)).astype(np.float32)
    if dtype == "bf16":
        hi = gen.round_to_bf16(p)
        p = hi if single else hi + gen.round_to_bf16(p - hi)
    out = (p.astype(np.float64) @ k[:, :r] / p.astype(np.float64).sum(1, keepdims=True)).astype(np.float32)
    return gen.round_to_bf16(out) if dtype == "bf16" else out


def share(bad, ref, bound):
    err = np.abs(bad - ref)
    return float(np.max(np.divide(err, bound, out=np.where(err > 0, np.inf, 0.0), where=bound > 0)))


KINDS = [("f32", False), ("bf16", False), ("bf16", True)]


@pytest.mark.parametrize("dtype,single", KINDS)
@pytest.mark.parametrize("r,n,per", [(128, 9, 1), (512, 703, 1), (128, 33000, TILE), (512, 9000, None)])
def test_the_kernels_arithmetic_passes(dtype, single, r, n, per):
    _, q, k, see, scale = case(1, n, 5, r, dtype, per)
    ref, bound = row_bounds(q, k, r, see, scale, dtype, single)
    assert share(like_the_kernel(q, k, r, scale, dtype, single), ref, bound) <= 1.0


@pytest.mark.parametrize("dtype,single", KINDS)
@pytest.mark.parametrize("r,n,per", [(128, 703, 1), (512, 703, 1), (128, 33000, TILE), (512, 33000, TILE), (128, 64 * 513, TILE)])
def test_nothing_can_be_lost_taken_twice_or_taken_from_elsewhere(dtype, single, r, n, per):
    """A key or sixteen of them (half of a bf16 tile, a tile of fp32), anywhere, of one row."""
    rng, q, k, see, scale = case(2, n, 1, r, dtype, per)
    ref, bound = row_bounds(q, k, r, see, scale, dtype, single)
    _, p, _ = attend(q, k, r, see, scale)
    size = 1 if per == 1 else 16
    for t in sorted({0, n // size - 1, *rng.integers(0, n // size, 12).tolist()}):
        keys = slice(t * size, (t + 1) * size)
        for weight in (0.0, 2.0):
            w = p.copy()
            w[:, keys] *= weight
            assert share(w @ k[:, :r] / w.sum(1, keepdims=True), ref, bound) > 1.0, (t, weight)
        v = k[:, :r].copy()
        other = (np.arange(keys.start, keys.stop) + 3 * TILE) % n
        v[keys] = v[other]
        assert share(p @ v, ref, bound) > 1.0, t


@pytest.mark.parametrize("r", [128, 512])
def test_fewer_digits_show_in_the_norm(r):
    """What the test of the fp32 digits allows, 7e-6, is less than any part of 16 bits would cost; and one bf16 part of the probabilities costs more than a twentieth of the results' rounding."""
    _, q, k, see, scale = case(3, 9000, 8, r, "f32", None)
    ref, p, s = attend(q, k, r, see, scale)
    norm = lambda x: np.linalg.norm(x - ref) / np.linalg.norm(ref)
    assert norm(like_the_kernel(q, k, r, scale, "f32", False)) < 7e-6
    half = lambda x: gen.round_to_bf16(x.astype(np.float32)).astype(np.float64)
    two = lambda x: half(x) + half(x - half(x))
    cut = lambda f: [f(p) @ k[:, :r] / f(p).sum(1, keepdims=True), attend(f(q.astype(np.float64)), k, r, see, scale)[0], attend(q, f(k), r, see, scale)[0]]
    # roundings to bf16 are 1.6e-3 of a value on average.  Of queries and entries they go into the outputs whole; of n probabilities by sqrt(sum p^2), 0.0105 and more with 9000, of values of
    # one, where outputs are some 0.05 (the queries times the scale): 3.4e-4 of them
    assert min(map(norm, cut(half))) > 3.4e-4
    assert norm(two(p) @ k[:, :r] / two(p).sum(1, keepdims=True)) < 7e-6          # (16 bits of a probability are off by 2^-18 on average, too little to show here)
    _, q, k, see, scale = case(3, 4100, 8, r, "bf16", None)
    ref, _, _ = attend(q, k, r, see, scale)
    rounding = norm(stored(ref, "bf16"))
    assert norm(like_the_kernel(q, k, r, scale, "bf16", False)) < 1.05 * rounding < norm(like_the_kernel(q, k, r, scale, "bf16", True))


def test_which_calls_take_one_part():
    for rows, gran, single in ((64, 5000, False), (65, 511, False), (65, 512, True), (128, 512, True), (129, 255, False), (129, 256, True)):
        assert one_part([gran * 64], rows, "bf16") == single and not one_part([gran * 64], rows, "f32")
        assert granules([gran * 64 - 63, 1], rows, "bf16") == (gran + 1) * -(-rows // (128 if rows > 64 else 64))
