"""The oracle's 8-bit rows and sampled tokens, pinned by library conversions, closed forms and brute force (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O


def test_e4m3_values_are_the_library_types():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(O.E4M3, t)


def test_codes_are_the_library_conversions_of_the_scaled_rows():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((300, 64)) * np.exp(4 * rng.standard_normal((300, 1)))).astype(np.float32)
    codes, s = O.quant_rows(x)
    y = torch.from_numpy(x).double() * torch.from_numpy(np.ldexp(1.0, 127 - s.astype(int))).unsqueeze(1)
    np.testing.assert_array_equal(codes, y.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    scale = np.ldexp(1.0, s.astype(int) - 127)
    amax = np.abs(x).max(1)
    assert (amax <= 448 * scale).all() and (amax > 224 * scale).all()      # the least power of two


def test_rows_at_the_edges():
    x = np.zeros((6, 64))
    x[1, 3] = 448.0
    x[2, 3] = np.nextafter(np.float32(448.0), np.float32(1e9))
    x[3, 3], x[3, 4], x[3, 5] = np.inf, -np.inf, np.nan
    x[4, 0] = 1e-42
    x[5, 0], x[5, 1] = 3e38, -3e38
    codes, s = O.quant_rows(x)
    assert s.tolist() == [1, 127, 128, 1, 1, 127 + 120]
    assert codes[1, 3] == 126 and codes[2, 3] == 118                       # 448, and 448.00003 / 2 rounded to 224
    assert codes[3, 3:6].tolist() == [127, 255, 127] and codes[0].max() == 0
    assert np.abs(O.dequant_rows(codes, s)[5, :2]).max() <= 3.4e38


@pytest.mark.parametrize("seed", range(4))
def test_a_draw_inverts_the_cumulative_sum(seed):
    rng = np.random.default_rng(seed)
    l = rng.standard_normal(50) * 2
    p = np.exp(l) / np.exp(l).sum()
    hit = np.zeros(50)
    us = (np.arange(4000) + 0.5) / 4000
    for u in us:
        t, prob, _ = O.sample(l, u)
        assert abs(prob - p[t]) < 1e-12
        hit[t] += 1
    assert np.abs(hit / 4000 - p).max() <= 1.0 / 4000 + 1e-9


def test_filters_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.1, 0.2, 0.2]))
    kept = lambda **kw: O.sample(l, 0.0, **kw)[2].tolist()
    assert kept() == [0, 1, 2, 3, 4]
    assert kept(top_k=2) == [1, 3]                         # ties: the lower index
    assert kept(top_k=5) == kept(top_k=0) == kept(top_k=-1) == [0, 1, 2, 3, 4]
    assert kept(top_p=0.39) == [1] and kept(top_p=0.45) == [1, 3] and kept(top_p=0.0) == [1]
    assert kept(min_p=0.4) == [1, 3, 4] and kept(min_p=5.0) == [1]
    assert kept(top_k=3, top_p=0.55) == [1, 3]             # of the three best's 0.8: 0.44
    assert kept(temperature=0.0) == [1] and O.sample(l, 0.99, temperature=0.0)[:2] == (1, 1.0)
    assert O.sample(np.full(4, -np.inf), 0.5)[:2] == (-1, 0.0)
    assert O.sample([-np.inf, 1.0, np.nan, -np.inf], 0.999)[:2] == (1, 1.0)
    assert O.sample([1.0, np.inf, 2.0, np.inf], 0.6)[:2] == (3, 0.5)
