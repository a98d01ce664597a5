"""The oracle's rotations, latent cache and log probabilities against closed forms and library routines (CPU)."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O


def test_rotation_is_the_draft_layers_rotation_and_a_complex_product():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4, 3, 16))
    pos = np.array([0, 1, 77, 5000])
    f = O.rope_frequencies(16, 1e6)
    got = O.rope_heads(x, pos, f)
    for t in range(4):
        for h in range(3):
            assert np.allclose(got[t, h], O.rope_rotate_half(x[t, h], int(pos[t]), 1e6), atol=1e-12)
    got = O.rope_heads(x, pos, f, interleaved=True, amplitude=1.5)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * 1.5 * np.exp(1j * pos[:, None, None] * f.astype(float))
    assert np.allclose(got[..., 0::2], z.real) and np.allclose(got[..., 1::2], z.imag)


def test_rotation_leaves_the_rest_and_scores_depend_on_distance_only():
    rng = np.random.default_rng(1)
    f = O.rope_frequencies(8, 1e4)
    q, k = rng.standard_normal((2, 1, 1, 32))
    assert np.array_equal(O.rope_heads(q, [9], f)[..., 8:], q[..., 8:])
    dot = lambda a, b: float((O.rope_heads(q, [a], f) * O.rope_heads(k, [b], f)).sum())
    assert abs(dot(5, 2) - dot(1005, 1002)) < 1e-11
    assert np.array_equal(O.rope_heads(q, [0], f), q)


def test_scaled_frequencies():
    f = O.rope_frequencies(128, 5e5).astype(float)
    assert np.allclose(f, 5e5 ** (-np.arange(64) / 64))
    assert np.allclose(O.rope_frequencies(128, 5e5, O.LINEAR, 4.0).astype(float), f / 4)
    turns = 8192 * f / (2 * np.pi)
    g = O.rope_frequencies(128, 5e5, O.BANDS, 8.0, 1.0, 4.0, 8192).astype(float)
    assert np.allclose(g[turns > 4], f[turns > 4]) and np.allclose(g[turns < 1], f[turns < 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 8).all()
    g = O.rope_frequencies(64, 1e4, O.RAMP, 40.0, 1.0, 32.0, 4096).astype(float)
    f = O.rope_frequencies(64, 1e4).astype(float)
    # 64 ln(4096 / 64 pi) / 2 ln 10^4 = 10.47 -> 10, 64 ln(4096 / 2 pi) / 2 ln 10^4 = 22.51 -> 23
    assert np.allclose(g[:11], f[:11]) and np.allclose(g[23:], f[23:] / 40) and np.allclose(g[16], f[16] * (7 / 13 + 6 / 13 / 40))


def test_latent_rows():
    rng = np.random.default_rng(2)
    x, gain = rng.standard_normal((3, 16)), rng.standard_normal(8)
    f = O.rope_frequencies(8, 1e4)
    got = O.latent_rows(x, gain, 1e-6, [0, 3, 9], f)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x[:, :8]), (8,), torch.from_numpy(gain), 1e-6).numpy()
    assert np.allclose(got[:, :8], want)
    assert np.array_equal(O.latent_rows(x, None, 1e-6, [0, 3, 9], f)[:, :8], x[:, :8])


@pytest.mark.parametrize("paged", [False, True])
def test_latent_attention_is_attention_with_shared_keys_and_values(paged):
    rng = np.random.default_rng(3)
    B, n_q, H, r, w = 2, 3, 4, 8, 12
    L = np.array([5, 30])
    pool = rng.standard_normal((8, 16, w)) if paged else rng.standard_normal((B, 48, w))
    table = np.array([[3, 0, 0], [1, 6, 2]], np.int32) if paged else None
    q = rng.standard_normal((B, n_q, H, w))
    got = O.latent_attn(q, pool, r, L, None, 0.3, table, 16)
    wide = np.concatenate([pool[..., :r], np.zeros(pool.shape[:-1] + (w - r,))], -1)
    k, v = (pool[:, None], wide[:, None])
    want = O.verify_attn(q, k, v, L, None, 0.3, table, 16)
    assert np.allclose(got, want[..., :r])
    # expanded: keys and values of every head from the latent, as a model defines them
    up_k, up_v = rng.standard_normal((H, 6, r)), rng.standard_normal((H, 5, r))
    q_nope, q_pe = rng.standard_normal((B, n_q, H, 6)), rng.standard_normal((B, n_q, H, w - r))
    absorbed = np.concatenate([np.einsum("bihn,hnr->bihr", q_nope, up_k), q_pe], -1)
    out = np.einsum("bihr,hvr->bihv", O.latent_attn(absorbed, pool, r, L, None, 0.3, table, 16), up_v)
    for b in range(B):
        rows = np.concatenate([pool[p] for p in table[b]])[:L[b] + n_q] if paged else pool[b, :L[b] + n_q]
        for h in range(H):
            keys, vals = np.concatenate([rows[:, :r] @ up_k[h].T, rows[:, r:]], 1), rows[:, :r] @ up_v[h].T
            qq = np.concatenate([q_nope[b, :, h], q_pe[b, :, h]], 1)
            m = np.tril(np.ones((n_q, L[b] + n_q), bool), L[b])
            want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (qq, keys, vals)), torch.from_numpy(m), scale=0.3)
            assert np.allclose(out[b, :, h], want[0].numpy())


def test_latent_attention_of_a_row_that_sees_nothing():
    c = np.ones((1, 16, 12))
    out = O.latent_attn(np.ones((1, 2, 1, 12)), c, 8, [0], np.array([[0, 2]], np.uint64), 1.0)
    assert (out[0, 0] == 0).all() and (out[0, 1] == 1).all()


def test_log_probabilities():
    rng = np.random.default_rng(4)
    l = rng.standard_normal(50) * 3
    lp, ent, top, top_lp = O.token_logprobs(l, [3, 49], 4, 0.7)
    want = torch.log_softmax(torch.from_numpy(l) / 0.7, 0)
    assert np.allclose(lp, want[[3, 49]].numpy()) and np.isclose(ent, torch.distributions.Categorical(logits=want).entropy().item())
    assert np.array_equal(top, torch.topk(want, 4).indices.numpy()) and np.allclose(top_lp, torch.topk(want, 4).values.numpy())
    lp, ent, top, _ = O.token_logprobs(np.zeros(8), [0, 7], 3)
    assert np.allclose(lp, -np.log(8)) and np.isclose(ent, np.log(8)) and top.tolist() == [0, 1, 2]
    lp, ent, top, tl = O.token_logprobs([-np.inf, 2.0, np.nan], [0, 1, 2], 3)
    assert lp.tolist() == [-np.inf, 0.0, -np.inf] and ent == 0 and top.tolist() == [1, -1, -1] and tl[1] == -np.inf
    lp, ent, top, _ = O.token_logprobs([1.0, np.inf, np.inf], [0, 1], 3)
    assert lp[0] == -np.inf and np.isclose(lp[1], -np.log(2)) and np.isclose(ent, np.log(2)) and top.tolist() == [1, 2, 0]
    lp, ent, top, _ = O.token_logprobs([-np.inf] * 3, [1], 2)
    assert lp[0] == -np.inf and ent == 0 and top.tolist() == [-1, -1]
