"""GPU: log probabilities of given tokens, entropy and best alternatives against the oracle."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O

import harness as H
from target_harness import DT, U, i32, logprob_bound

pytestmark = pytest.mark.gpu


def run(x, V, tokens, n_top, temperature=None, per=1, dtype="f32", flags=0, entropy=True):
    """x: torch [M, >= V] on the GPU"""
    lib, guard = H.sx(), H.Guarded()
    M, n_tok = x.shape[0], tokens.shape[1]
    lp, ent = guard.empty((M, n_tok), torch.float32), guard.empty(M, torch.float32)
    top, tlp = guard.empty((M, n_top), torch.int32), guard.empty((M, n_top), torch.float32)
    code = lib.dtype_code(DT[dtype])
    ws = guard.empty(lib.specexit_token_logprobs_workspace_bytes(code, M, V, n_top), torch.uint8)
    lib.specexit_token_logprobs(code, M, V, x, ent if entropy else None, i32(tokens) if n_tok else None, lp if n_tok else None, top if n_top else None,
                                tlp if n_top else None, None if temperature is None else torch.tensor(temperature, dtype=torch.float32, device="cuda"),
                                per, ws, flags=flags)
    guard.check()
    return H.host(lp), H.host(ent), top.cpu().numpy(), H.host(tlp)


def check(x, V, tokens, n_top, temperature=None, per=1, dtype="f32", got=None):
    got = run(x, V, tokens, n_top, temperature, per, dtype) if got is None else got
    l = x[:, :V].float().cpu().numpy()
    for r in range(len(l)):
        T = 1.0 if temperature is None else float(np.float32(temperature[r // per]))
        T = min(max(T, 2.0 ** -10), 2.0 ** 96)
        lp, ent, top, tlp = O.token_logprobs(l[r], tokens[r], n_top, T)
        assert np.array_equal(got[2][r], top), r
        row = np.where(np.isnan(l[r]), -np.inf, l[r]).astype(np.float64)
        with np.errstate(invalid="ignore"):
            y = np.where(row == row.max(), 0.0, (row - row.max()) / T)
        p = np.exp(y - np.log(np.exp(y).sum()))
        weight = float((p * np.where(p > 0, np.abs(y), 0)).sum())
        second = float((p * np.where(p > 0, y * y, 0)).sum())
        for a, b, yy in ((got[0][r], lp, y[tokens[r]]), (got[3][r], tlp, y[np.maximum(top, 0)])):
            with np.errstate(over="ignore"):
                b = b.astype(np.float32).astype(np.float64)        # (what lies below the type's range is -infinity in it)
            fin = np.isfinite(b)
            assert np.array_equal(a[~fin], b[~fin]), r
            assert (np.abs(a - b)[fin] <= logprob_bound(yy, b, weight)[fin]).all(), (r, float((np.abs(a - b) - logprob_bound(yy, b, weight))[fin].max()))
        # entropy: the logarithms' sum as above, and the mean distance, whose weights are off by 2^-22 of their distance and whose sum passes 128 steps
        assert abs(got[1][r] - ent) <= 2.0 ** -22 * (ent + 2 * weight + second + 2) + 128 * U * (1 + weight), (r, got[1][r], ent)


def rows(seed, M, ld, dtype, V):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, ld), generator=g) * 2.2
    for r in range(M):
        k = 3 + 7 * (r % 5)
        x[r, torch.randint(0, V, (k,), generator=g)] += torch.linspace(14, 2, k)
    return x.cuda().to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,ld,n_tok,n_top", [(1, 1, 1, 1, 1), (3, 2, 5, 2, 32), (2, 31, 31, 1, 5), (5, 1000, 1003, 3, 20), (4, 2049, 2051, 1, 32),
                                                (7, 8193, 8193, 64, 1), (2, 50257, 50260, 0, 5), (9, 128259, 128262, 2, 0), (3, 262144, 262144, 1, 32),
                                                (70, 65536, 65537, 1, 20)])
def test_rows(dtype, M, V, ld, n_tok, n_top):
    x = rows(V, M, ld, dtype, V)
    rng = np.random.default_rng(V)
    tokens = rng.integers(0, V, (M, n_tok))
    check(x, V, tokens, n_top, dtype=dtype)
    per = 2 if M > 1 else 1
    heat = rng.uniform(0.3, 2.0, -(-M // per))
    check(x, V, tokens, n_top, heat, per, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_slice_that_starts_anywhere(dtype):
    x = rows(4, 6, 3001, dtype, 2990)
    for first in range(1, 9):
        view = x[1:, first:]
        tokens = np.full((5, 1), 17)
        check(view, 2980, tokens, 7, dtype=dtype, got=run(view, 2980, tokens, 7, dtype=dtype))


@pytest.mark.parametrize("V,M", [(9000, 3), (9000, 200), (30000, 2)])
def test_ties_and_orders_that_defeat_the_bound(V, M):
    """All equal; ascending; descending; blocks of a few values: ties go to the lowest index, and lists that overflow are searched."""
    up = torch.arange(V, dtype=torch.float32) / 1000
    kinds = [torch.zeros(V), up, up.flip(0), torch.arange(V).remainder(3).float(), (torch.arange(V) // 700).float(), -up.clone()]
    x = torch.stack([kinds[r % len(kinds)] for r in range(max(M, len(kinds)))]).cuda()
    for n_top in (1, 6, 32):
        check(x, V, np.zeros((len(x), 1), int), n_top)
    y = x.to(torch.bfloat16)
    check(y, V, np.zeros((len(y), 1), int), 20, dtype="bf16")


@pytest.mark.parametrize("V", [40, 20000])
def test_infinities_nan_and_rows_that_allow_little(V):
    x = torch.randn((8, V), generator=torch.Generator().manual_seed(3))
    x[0, :] = -np.inf
    x[1, :] = -np.inf
    x[1, 7] = 2.0
    x[2, 3:] = np.nan
    x[3, 5] = np.inf
    x[4, [1, 8, 30]] = np.inf
    x[5, ::2] = -np.inf
    x[6, :] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    x[7, 9] = 3e38
    x[7, 10] = -3e38
    tokens = np.tile([5, 7, 8, 0], (8, 1))
    check(x.cuda(), V, tokens, 32)
    check(x.cuda(), V, tokens, 32, [0.5] * 8)
    check(x.cuda(), V, tokens, 32, [0.0] * 8)                  # forced to 2^-10


def test_tokens_outside_the_vocabulary():
    lib = H.sx()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = rows(1, 2, 100, "f32", 100)
    lib.specexit_set_dev_status(word)
    try:
        got = run(x, 100, np.array([[3, -1], [4, 5]]), 2, flags=lib.FLAG_VALIDATE)
        assert int(word.item()) == lib.STATUS_OK and np.isnan(got[0][0, 1]) and np.isfinite(got[0][[0, 1, 1], [0, 0, 1]]).all()
        got = run(x, 100, np.array([[3, 100], [-2, 5]]), 0, flags=lib.FLAG_VALIDATE)
        assert int(word.item()) == lib.STATUS_BAD_TOKEN and np.isnan(got[0][0, 1]) and np.isnan(got[0][1, 0]) and np.isfinite(got[0][0, 0])
    finally:
        lib.specexit_set_dev_status(None)


def test_a_sure_token_keeps_its_digits():
    """ln p of a token with nearly all of the probability is - the sum of the others, to its own digits."""
    x = torch.zeros((2, 5000))
    x[0, 77], x[1, 4999] = 30.0, 40.0
    got = run(x.cuda(), 5000, np.array([[77], [4999]]), 1)
    for r, gap in ((0, 30.0), (1, 40.0)):
        rest = 4999 * np.exp(-gap)
        assert abs(got[0][r, 0] / -rest - 1) < 1e-4 and abs(got[1][r] / (rest * (1 + gap)) - 1) < 1e-4


def test_the_sampled_token_has_its_probability():
    """Beside specexit_sample: with nothing filtered its share of a drawn token is the exponential of the log probability."""
    lib = H.sx()
    M, V = 12, 4096
    x = rows(9, M, V, "f32", V)
    heat = torch.tensor([0.7, 1.0, 1.4], device="cuda")
    u = torch.linspace(0.01, 0.99, M, device="cuda")
    token, prob = torch.empty(M, dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
    lib.specexit_sample(lib.F32, M, V, x, u, token, prob, heat, rows_per_seq=4, workspace=H.workspace(lib.specexit_sample_workspace_bytes(lib.F32, M, V)))
    lp = torch.empty((M, 1), device="cuda")
    lib.specexit_token_logprobs(lib.F32, M, V, x, token=token.view(M, 1), logprob=lp, temperature=heat, rows_per_seq=4,
                                workspace=H.workspace(lib.specexit_token_logprobs_workspace_bytes(lib.F32, M, V)))
    assert torch.allclose(torch.exp(lp[:, 0]), prob, rtol=1e-4, atol=1e-8)
