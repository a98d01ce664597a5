"""GPU: sampled tokens of rows with many tokens about a border, which are selected from without a list, and of numbers next to a border."""
import numpy as np
import pytest

import harness as H
from test_gpu_sample import check, head_like

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
