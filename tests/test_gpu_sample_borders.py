"""GPU: sampled tokens of rows with many tokens about a border, which are selected from without a list, and of numbers next to a border."""
import numpy as np
import pytest

from workloads import gen

import harness as H
from test_gpu_sample import check, head_like, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("above", [9.0, 10.0, 11.0])
@pytest.mark.parametrize("sd", [0.3, 0.5])
def test_a_flat_row_with_one_token_far_above(sd, above):
    """One token makes the bins of the whole row wide, and thousands of the others share the border's."""
    rng = np.random.default_rng(61)
    V = 151936
    x = (rng.standard_normal((5, V)) * sd).astype(np.float32)
    x[np.arange(5), [0, 70000, V - 1, 512, 511]] = above
    check(x, rng.random(5).astype(np.float32), top_p=[0.9, 0.5, 0.99, 0.3, 1.0], top_k=[0, 0, 0, 1000, 1024])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_widest_vocabulary_with_plain_deviations(dtype):
    rng = np.random.default_rng(62)
    V = H.sx().SAMPLE_MAX_V
    x = (rng.standard_normal((4, V)) * np.array([[0.9], [1.0], [1.1], [2.0]])).astype(np.float32)
    check(x, rng.random(4).astype(np.float32), dtype, top_p=[0.9, 0.8, 0.95, 0.9])


def test_nuclei_of_nearly_everything():
    """top-p about and beyond 0.99998, where the border's margin is more than the rest of the row."""
    rng = np.random.default_rng(63)
    p = [0.999, 0.9999, 0.99997, 0.99998, 0.99999, 0.999999, 1.0 - 2.0 ** -24]
    x = head_like(rng, len(p), 40003)
    check(x, np.float32([0.1, 0.5, 0.9, 0.99999, 0.3, 0.7, 0.999]), top_p=p)
    check(x, rng.random(len(p)).astype(np.float32), top_p=p, min_p=[1e-6] * len(p), temperature=[1.4] * len(p))


def neighbours(x):
    """The two fp32 numbers about a real one, the first not above it."""
    lo = np.float32(x)
    lo = lo if float(lo) <= x else np.nextafter(lo, np.float32(-1))
    return lo, np.nextafter(lo, np.float32(2))


# what the header says a border is met to: a weight's rounding, half of 2^-45, for each of V tokens, and 2^-52 of the logit over the temperature
def off(V, far=64.0):
    return V * 2.0 ** -46 + 2.0 ** -52 * far


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 5003, 40003])
def test_draws_next_to_a_border_of_two_tokens(dtype, V):
    """u on both sides of the sums of a row's weights, one step of fp32 apart: the token on either side."""
    rng = np.random.default_rng(64)
    x = head_like(rng, 1, V)[0]
    if dtype == "bf16":
        x = gen.round_to_bf16(x)
    w = np.exp((x.astype(np.float64) - float(x.max())) / 0.75)
    upto = np.cumsum(w.astype(np.longdouble)) / w.astype(np.longdouble).sum()
    big = np.flatnonzero(w / w.sum() > 2.0 ** -20)[:-1]
    u, want, clear = [], [], []
    for i in rng.choice(big, 40):
        for v in neighbours(float(upto[i])):           # (the step of u may pass further tokens of little weight)
            u.append(v)
            want.append(int(np.searchsorted(upto, np.longdouble(v), side="right")))
            clear.append(float(np.abs(upto - np.longdouble(v)).min()) > off(V) + 1e-12)
    token, _ = run(np.repeat(x[None], len(u), 0), u, dtype, temperature=[0.75] * len(u))
    clear = np.array(clear)
    assert clear.sum() > 60
    np.testing.assert_array_equal(token[clear], np.array(want)[clear])


@pytest.mark.parametrize("V", [700, 5003, 40003])
def test_nuclei_next_to_a_border(V):
    """top-p on both sides of the sum of the best n tokens: with the last of them the next one's, or without it."""
    rng = np.random.default_rng(65)
    x = head_like(rng, 1, V)[0]
    w = np.exp((x.astype(np.float64) - float(x.max())) / 0.75)
    order = np.lexsort((np.arange(V), -x))
    upto = np.cumsum(w[order].astype(np.longdouble)) / w.astype(np.longdouble).sum()
    p, rows = [], []
    for n in rng.choice(np.arange(1, 120), 30, replace=False):
        for v in neighbours(float(upto[n - 1])):
            if abs(float(v) - float(upto[n - 1])) > off(V) + 1e-12:
                p.append(v)
                rows.append(int(n) + (float(v) > float(upto[n - 1])))
    assert len(p) > 45
    token, prob = run(np.repeat(x[None], len(p), 0), [0.0] * len(p), temperature=[0.75] * len(p), top_p=p)
    for r, n in enumerate(rows):
        kept = np.sort(order[:n])
        assert token[r] == kept[0]
        share = w[kept[0]] / w[kept].sum()
        # (the n-th token's weight is 1e-5 of the sum at least: a token more or less shows in the share)
        assert w[order[n - 1]] / w[kept].sum() > 1e-5
        assert abs(prob[r] - share) <= 2.0 ** -24 * share + off(V) * share + 1e-12


@pytest.mark.parametrize("steps", [32.5, 33.49, 40.5])
def test_draws_in_a_long_tail(steps):
    """151935 tokens of `steps` times 2^-45 each in front of the best one: a draw among them is within V 2^-46 of the sum of where it belongs."""
    V = 151936
    l = np.float32(np.log(steps) - 45 * np.log(2.0))
    x = np.full((1, V), l, np.float32)
    x[0, -1] = 0.0
    w = np.exp(float(l))
    total = (V - 1) * w + 1.0
    u = np.float32(np.linspace(0.01, 0.99, 50) * (V - 1) * w / total)
    token, _ = run(np.repeat(x, 50, 0), u)
    # (33.49 steps are rounded to 33, and the tail's sum ends at 33 / 33.49 = 0.985 of its own: the last draw, at 0.99, may be the best token)
    for t, v in zip(token.astype(np.int64), u.astype(np.float64)):
        assert t * w / total - off(V) <= v <= (t + 1) * w / total + off(V)
    # beyond the tail and what its sum may be off by, the best token
    assert run(x, [np.float32((V - 1) * w / total + 2 * off(V))])[0][0] == V - 1
