"""GPU: verification attention over a latent cache against the oracle."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O

import harness as H
from target_harness import DT, Latent, dev, i32, latent_attn_bound, run_latent_attn, stored, tree_masks

pytestmark = pytest.mark.gpu


def check(lat, q, L, mask, scale, dtype, got, rows=None):
    ref = O.latent_attn(q, lat.c, lat.r, L, mask, scale, lat.table, lat.page or 16)
    weighed = O.latent_attn(q, lat.c, lat.r, L, mask, scale, lat.table, lat.page or 16, absolute=True)
    over = np.abs(got - ref) / latent_attn_bound(ref, weighed, q, lat.c, lat.r, int(max(L)) + q.shape[1], scale, dtype)
    over = over if rows is None else over[rows]
    assert np.isfinite(over).all() and over.max() <= 1.0, float(over.max())


def case(seed, B, n_q, Hq, r, L, dtype, page=None, tree=False, scale=0.07, sharp=1.0):
    rng = np.random.default_rng(seed)
    L = np.asarray(L)
    lat = Latent(rng, B, r, L + n_q, dtype, page)
    q = stored(rng.standard_normal((B, n_q, Hq, r + 64)) * sharp, dtype)
    mask = tree_masks(rng, B, n_q)[0] if tree else None
    return lat, q, L, mask, scale


# rows of a sequence: 1 .. 16, 17 .. 32, 33 .. 64, 65 .. 128 and several blocks; contexts from nothing on, ends within tiles and pages
SHAPES = [(1, 1, 1, [0]), (2, 1, 16, [0, 1]), (3, 5, 3, [31, 32, 33]), (2, 7, 4, [63, 200]), (3, 3, 8, [15, 64, 1029]), (2, 4, 16, [100, 7]),
          (2, 5, 16, [17, 300]), (1, 1, 128, [513]), (3, 2, 64, [0, 47, 128]), (2, 16, 16, [90, 31]), (1, 9, 33, [260]), (1, 64, 5, [10])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [128, 256, 512])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_shapes(dtype, r, shape):
    B, n_q, Hq, L = SHAPES[shape]
    page = [None, 16, 48, 64][(shape + r // 128) % 4]
    lat, q, L, mask, scale = case(shape, B, n_q, Hq, r, L, dtype, page, tree=shape % 2 == 1)
    got = run_latent_attn(lat.gpu()[0], B, n_q, Hq, r, q, L, mask, scale, dtype)
    check(lat, q, L, mask, scale, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [3, 24, 48, 100])
@pytest.mark.parametrize("page", [None, 32])
def test_long_and_unequal_contexts(dtype, Hq, page):
    """Many workgroups a sequence, page ids in several batches of 64, one long context among short ones."""
    lat, q, L, mask, scale = case(Hq, 3, 1, Hq, 512, [9000 + Hq, 5, 1500], dtype, page)
    got = run_latent_attn(lat.gpu()[0], 3, 1, Hq, 512, q, L, mask, scale, dtype)
    check(lat, q, L, mask, scale, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_segments_longer_than_a_batch_of_page_ids(dtype):
    lat, q, L, mask, scale = case(3, 40, 1, 16, 128, [4000 + 61 * b for b in range(40)], dtype, 16)
    got = run_latent_attn(lat.gpu()[0], 40, 1, 16, 128, q, L, mask, scale, dtype)
    check(lat, q, L, mask, scale, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,n_q", [(2, 4), (16, 4), (16, 8)])
def test_sharp_and_rising_scores(dtype, Hq, n_q):
    """Scores that reach hundreds, and rise along the context, so that the reference moves with every tile."""
    rng = np.random.default_rng(1)
    lat, q, L, mask, scale = case(6, 2, n_q, Hq, 256, [700, 333], dtype, sharp=4.0)
    d = rng.standard_normal(320)
    q = stored(q + 2.0 * d, dtype)
    for b in range(2):
        ramp = np.arange(lat.c.shape[1])[:, None] / 300.0
        lat.c[b] = stored(lat.c[b] + ramp * d, dtype)
    got = run_latent_attn(lat.gpu()[0], 2, n_q, Hq, 256, q, L, mask, scale, dtype)
    check(lat, q, L, mask, scale, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [4, 20, 40])
def test_hidden_entries_may_hold_anything_and_empty_rows_are_zero(dtype, Hq):
    n_q, r = 3, 256
    lat, q, L, _, scale = case(9, 4, n_q, Hq, r, [0, 0, 50, 61], dtype, 16)
    mask = np.array([[0, 2, 0], [1, 0, 4], [1, 0, 5], [1, 3, 0]], np.uint64)
    clean = lat.c.copy()
    for b, node, value in ((0, 0, np.nan), (0, 2, np.inf), (1, 1, -np.inf), (2, 1, np.nan), (3, 2, np.inf)):      # entries that no row of theirs sees
        lat.c[lat.at(b, int(L[b]) + node)] = value
    got = run_latent_attn(lat.gpu()[0], 4, n_q, Hq, r, q, L, mask, scale, dtype)
    lat.c = clean
    check(lat, q, L, mask, scale, dtype, got)
    for b, i in ((0, 0), (0, 2), (1, 1)):
        assert (got[b, i] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_reaches_the_rows_that_see_it_only(dtype):
    n_q, r, Hq = 3, 128, 20
    lat, q, L, _, scale = case(10, 2, n_q, Hq, r, [90, 40], dtype)
    mask = np.array([[1, 2, 5], [1, 3, 7]], np.uint64)
    clean = lat.c.copy()
    lat.c[0, 91, 5] = np.nan              # seen by row 1 of sequence 0 only
    lat.c[1, 3, r + 2] = np.nan           # a key part of the context: scores of all rows of sequence 1
    got = run_latent_attn(lat.gpu()[0], 2, n_q, Hq, r, q, L, mask, scale, dtype)
    assert np.isnan(got[0, 1]).all() and np.isnan(got[1]).all()          # (the entry is key as well)
    lat.c = clean
    check(lat, q, L, mask, scale, dtype, got, rows=(0, [0, 2]))


def test_bad_lengths_and_pages_are_contained_and_reported():
    lib = H.sx()
    lat, q, L, _, scale = case(11, 3, 2, 16, 512, [40, 100, 200], "bf16", 16)
    view, c, table = lat.gpu()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.specexit_set_dev_status(word)
    try:
        for lengths, pages, code, whole in (([40, 100, 200], {}, lib.STATUS_OK, [0, 1, 2]), ([40, 10 ** 7, -3], {}, lib.STATUS_BAD_LENGTH, [0]),
                                            ([40, 100, 200], {(1, 2): 1 << 30, (1, 3): -7}, lib.STATUS_BAD_PAGE, [0, 2])):
            bad = lat.table.copy()
            for at, v in pages.items():
                bad[at] = v
            table.copy_(i32(bad))
            print("latent attention with lengths", lengths, "pages", pages, flush=True)
            got = run_latent_attn(view, 3, 2, 16, 512, q, lengths, None, scale, "bf16", flags=lib.FLAG_VALIDATE)
            assert int(word.item()) == code
            word.zero_()
            check(lat, q, L, None, scale, "bf16", got, rows=whole)
    finally:
        lib.specexit_set_dev_status(None)


def test_other_streams_and_the_same_call_twice():
    """Calls of two streams with workspaces of their own, and a second call of the same bits."""
    lib = H.sx()
    lat, q, L, mask, scale = case(12, 4, 4, 32, 512, [900, 30, 2000, 511], "bf16", 64, tree=True)
    view, _, _ = lat.gpu()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    qd, Ld, md = dev(q, "bf16"), i32(L), H.dev(mask)
    outs = [torch.zeros((4, 4, 32, 512), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    ws = [H.workspace(lib.specexit_latent_verify_attn_workspace_bytes(view, 4, 4, 32)) for _ in range(3)]
    torch.cuda.synchronize()
    for out, w, s in zip(outs, ws, (a, b, a)):
        lib.specexit_latent_verify_attn(view, 4, 4, 32, qd, Ld, md, scale, out, w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    check(lat, q, L, mask, scale, "bf16", H.host(outs[0]))
