"""GPU: latent attention where there is work for large blocks of rows, and at the lengths where the rows of a block change."""
import numpy as np
import pytest
import torch

import harness as H
from target_harness import dev, i32, run_latent_attn, stored
from test_gpu_latent_attn import case, check

pytestmark = pytest.mark.gpu

# a few granules of 64 entries each for many sequences, some with next to nothing: 600 granules and more
MANY = [0, 1, 2, 31, 33, 64, 127] + [400 + (37 * b) % 361 for b in range(64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,Hq,r,page", [(1, 20, 128, 16), (1, 33, 256, None), (3, 16, 128, 48), (4, 16, 512, 64), (5, 13, 128, None), (7, 16, 256, 32),
                                           (8, 16, 512, 64), (9, 15, 128, 16), (2, 70, 512, None)])
def test_many_granules(dtype, n_q, Hq, r, page):
    B = len(MANY)
    lat, q, L, mask, scale = case(n_q * Hq, B, n_q, Hq, r, MANY, dtype, page, tree=n_q > 2)
    got = run_latent_attn(lat.gpu()[0], B, n_q, Hq, r, q, L, mask, scale, dtype)
    check(lat, q, L, mask, scale, dtype, got)


@pytest.mark.parametrize("Hq", [32, 64, 128])
@pytest.mark.parametrize("granules", [159, 160, 161, 511, 512, 513])
def test_where_the_rows_of_a_block_change(Hq, granules):
    """One sequence whose last granule is full, one short of that, or a single entry."""
    for extra in (0, -1, -63):
        n = 64 * granules + extra
        lat, q, L, mask, scale = case(granules, 1, 1, Hq, 128, [n - 1], "bf16", 64)
        got = run_latent_attn(lat.gpu()[0], 1, 1, Hq, 128, q, L, mask, scale, "bf16")
        check(lat, q, L, mask, scale, "bf16", got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q", [4, 8])
def test_sharp_and_rising_scores(dtype, n_q):
    """References that the rows' later scores leave far behind, in some segments and not in others."""
    rng = np.random.default_rng(2)
    B, r = 48, 128
    lat, q, L, mask, scale = case(7, B, n_q, 16, r, [700 + b for b in range(B)], dtype, sharp=4.0)
    d = rng.standard_normal(r + 64)
    q = stored(q + 2.0 * d, dtype)
    for b in range(0, B, 2):
        lat.c[b] = stored(lat.c[b] + np.arange(lat.c.shape[1])[:, None] / 300.0 * d, dtype)
    got = run_latent_attn(lat.gpu()[0], B, n_q, 16, r, q, L, mask, scale, dtype)
    check(lat, q, L, mask, scale, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [16, 40])
def test_hidden_entries_empty_rows_and_what_is_not_finite(dtype, Hq):
    n_q, r, B = 3, 128, len(MANY)
    lat, q, L, _, scale = case(19, B, n_q, Hq, r, MANY, dtype, 16)
    mask = np.tile(np.array([1, 3, 7], np.uint64), (B, 1))
    mask[0] = [0, 2, 0]                           # no context: rows 0 and 2 see nothing
    mask[1] = [1, 0, 4]
    mask[10] = [1, 0, 5]                          # nothing of the block, the context all the same
    clean = lat.c.copy()
    for b, node, value in ((0, 0, np.nan), (0, 2, np.inf), (1, 1, -np.inf), (10, 1, np.nan)):      # entries that no row of theirs sees
        lat.c[lat.at(b, int(L[b]) + node)] = value
    lat.c[lat.at(12, int(L[12]) + 2)][5] = np.nan            # seen by row 2 of sequence 12 only
    lat.c[lat.at(20, 3)][r + 2] = np.inf                     # a key part of the context: scores of all rows of sequence 20 are infinite
    got = run_latent_attn(lat.gpu()[0], B, n_q, Hq, r, q, L, mask, scale, dtype)
    lat.c = clean
    assert (got[0, 0] == 0).all() and (got[0, 2] == 0).all()
    assert np.isnan(got[12, 2]).all()
    fine = np.ones((B, n_q), bool)
    fine[12, 2] = False
    fine[20] = False
    check(lat, q, L, mask, scale, dtype, got, rows=np.nonzero(fine))


def test_one_graph_for_lengths_that_change():
    """A captured call replayed after its lengths grew, so that it takes blocks of 16, 32 and 128 rows in turn, with eager work between."""
    lib = H.sx()
    B, n_q, Hq, r = 4, 8, 16, 256
    most = [9000, 7000, 8500, 9100]
    lat, q, L, mask, scale = case(23, B, n_q, Hq, r, most, "bf16", 64, tree=True)
    view, _, _ = lat.gpu()
    qd, Ld, md = dev(q, "bf16"), i32(L), H.dev(mask)
    out = torch.zeros((B, n_q, Hq, r), dtype=torch.bfloat16, device="cuda")
    again = torch.zeros_like(out)
    bytes_ = lib.specexit_latent_verify_attn_workspace_bytes(view, B, n_q, Hq)
    ws, ws2 = H.workspace(bytes_), H.workspace(bytes_)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    lib.specexit_graph_begin(stream)
    lib.specexit_latent_verify_attn(view, B, n_q, Hq, qd, Ld, md, scale, out, ws, stream=stream)
    graph = lib.specexit_graph_end(stream)
    try:
        for lengths in ([100, 7, 0, 64], most, [5000, 3000, 4000, 2000], [100, 7, 0, 64], most):
            Ld.copy_(i32(lengths))
            out.fill_(7.0)
            torch.cuda.synchronize()
            lib.specexit_graph_launch(graph, stream)
            torch.cuda.synchronize()
            lib.specexit_latent_verify_attn(view, B, n_q, Hq, qd, Ld, md, scale, again, ws2)
            torch.cuda.synchronize()
            assert torch.equal(out, again)
            # (the block's entries are at the lengths of now)
            check(lat, q, np.asarray(lengths), mask, scale, "bf16", H.host(out))
    finally:
        lib.specexit_graph_destroy(graph)
