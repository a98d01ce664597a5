"""GPU: attention over the 8-bit cache against the oracle."""
import numpy as np
import pytest
import torch

from workloads import gen

import harness as H
from quant_harness import Cache, attn, check_attn, queries, tree_masks

pytestmark = pytest.mark.gpu


# every count of 16-row tiles (1 to 8), both widths and types, odd row counts
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(1, 1), (4, 4), (4, 7), (8, 4), (5, 9), (4, 16), (8, 9), (6, 16), (7, 15), (8, 16), (2, 64)])
def test_row_counts(dtype, d, G, n_q):
    rng = np.random.default_rng(G * 100 + n_q)
    L = np.array([300, 37])
    cache = Cache(rng, 2, 2, d, L + n_q, 16)
    q = queries(rng, 2, n_q, 2 * G, d, dtype)
    print("worst share of the bound", check_attn(cache, q, L, None, dtype=dtype), flush=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16, 32, 48, 112])
@pytest.mark.parametrize("tree", [False, True])
def test_ragged_lengths(dtype, page, tree):
    rng = np.random.default_rng(11)
    L = np.array([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 121, 500, 1023])
    n_q = 7
    cache = Cache(rng, len(L), 2, 128, L + n_q, page)
    q = queries(rng, len(L), n_q, 8, 128, dtype)
    check_attn(cache, q, L, tree_masks(rng, len(L), n_q) if tree else None, dtype=dtype)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,top", [(1, 9000), (70, 400), (130, 60), (5, 3000)])
def test_work_splits(d, B, top):
    """One long unit over all compute units, more sequences than a wave has lanes, units that start and end inside a share."""
    rng = np.random.default_rng(B)
    L = rng.integers(max(0, top - 700), top, B)
    n_q = 5
    cache = Cache(rng, B, 2, d, L + n_q, 16)
    q = queries(rng, B, n_q, 8, d, "bf16")
    only = None if B < 10 else [(int(b), int(i), int(h)) for b, i, h in zip(rng.integers(0, B, 60), rng.integers(0, n_q, 60), rng.integers(0, 8, 60))]
    check_attn(cache, q, L, None, only=only)


def test_the_widest_block():
    rng = np.random.default_rng(4)
    L = np.array([700, 64])
    cache = Cache(rng, 2, 1, 128, L + 64, None)
    q = queries(rng, 2, 64, 2, 128, "bf16")
    check_attn(cache, q, L, tree_masks(rng, 2, 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing_are_zero(dtype, d):
    rng = np.random.default_rng(5)
    L = np.array([0, 40, 0])
    n_q = 4
    cache = Cache(rng, 3, 2, d, L + n_q, 16)
    q = queries(rng, 3, n_q, 4, d, dtype)
    mask = np.array([[0, 1, 2, 0], [0, 0, 0, 15], [0, 0, 0, 0]], np.uint64)
    got = attn(cache, q, L, mask, dtype=dtype)
    empty = [(0, 0), (0, 3), (2, 0), (2, 1), (2, 2), (2, 3)]
    for b, i in empty:
        assert (got[b, i] == 0).all()
    only = [(b, i, h) for b in range(3) for i in range(n_q) for h in range(4) if (b, i) not in empty]
    check_attn(cache, q, L, mask, dtype=dtype, got=got, only=only)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16])
def test_entries_that_a_row_does_not_see_may_hold_anything(dtype, page):
    rng = np.random.default_rng(6)
    L = np.array([50, 90, 8])
    n_q, d = 6, 128
    cache = Cache(rng, 3, 2, d, L + n_q, page)
    q = queries(rng, 3, n_q, 8, d, dtype)
    mask = tree_masks(rng, 3, n_q)
    clean = attn(cache, q, L, mask, dtype=dtype)
    # entry 4 of every block: NaN codes and a scale byte that no row has, seen only by the rows whose bit 4 is set
    for b in range(3):
        at = cache.at(b, L[b] + 4)
        cache.k[at], cache.v[at] = 0x7F, 0xFF
        cache.ks[at], cache.vs[at] = 255, 255
    got = attn(cache, q, L, mask, dtype=dtype)
    sees = (mask >> np.uint64(4) & np.uint64(1)).astype(bool)
    assert np.isnan(got[sees]).all()
    assert np.isfinite(got[~sees]).all()
    k, v = cache.values()
    only = [(b, i, h) for b in range(3) for i in range(n_q) for h in range(8) if not sees[b, i]]
    # (the row is taken again key by key: fp32 sums, the output's rounding)
    sel = tuple(np.array(only).T)
    assert np.abs(got[sel] - clean[sel]).max() <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * np.abs(clean[sel]).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_of_any_size(dtype):
    """Magnitudes from 2^-100 to 2^100 times a usual one (with the scale to match), a row of zeros, a row with one large value."""
    rng = np.random.default_rng(8)
    L = np.array([200])
    n_q, d = 5, 128
    cache = Cache(rng, 1, 1, d, L + n_q, 16)
    q = queries(rng, 1, n_q, 4, d, dtype)
    q[0, 1, 2] = 0.0
    q[0, 2, 1] *= 2.0 ** -20
    q[0, 2, 1, 17] = 3.0
    for e in (-100, 0, 100):
        check_attn(cache, np.ldexp(q, e).astype(np.float32), L, None, scale=2.0 ** -e * d ** -0.5, dtype=dtype)


def test_keys_of_any_size():
    """Scale bytes over the whole range that bf16 rows have: large values of keys that count little, small ones of those that count."""
    rng = np.random.default_rng(9)
    L = np.array([300])
    n_q, d = 3, 64
    cache = Cache(rng, 1, 1, d, L + n_q, None, spread=0.0)
    q = queries(rng, 1, n_q, 4, d, "bf16")
    cache.vs[:] = rng.integers(90, 150, cache.vs.shape)
    cache.ks[:, :, :100] = 60
    check_attn(cache, q, L, None)


def test_peaked_and_growing_scores():
    """Scores that grow along the cache (the softmax reference moves at every tile) and one key that takes all."""
    rng = np.random.default_rng(10)
    L = np.array([1500])
    n_q, d = 2, 128
    cache = Cache(rng, 1, 2, d, L + n_q, None, spread=0.0)
    cache.ks[:] = (cache.ks.astype(int) + np.arange(cache.ks.shape[2]) // 400).astype(np.uint8)
    q = queries(rng, 1, n_q, 8, d, "bf16") * 4
    check_attn(cache, q, L, None)


def test_unaligned_queries_and_output():
    lib, rng = H.sx(), np.random.default_rng(12)
    L = np.array([100, 30])
    n_q, d = 3, 128
    cache = Cache(rng, 2, 2, d, L + n_q, 16)
    q = queries(rng, 2, n_q, 4, d, "bf16")
    view, t = cache.gpu()
    buf = torch.zeros(q.size + 1, dtype=torch.bfloat16, device="cuda")
    qd = buf[1:].view(q.shape)
    qd.copy_(torch.from_numpy(q))
    out = torch.zeros(q.size + 1, dtype=torch.bfloat16, device="cuda")[1:].view(q.shape)
    ws = H.workspace(lib.specexit_quant_verify_attn_workspace_bytes(view, lib.BF16, 2, n_q, 4))
    lib.specexit_quant_verify_attn(view, lib.BF16, 2, n_q, 4, qd, torch.from_numpy(L.astype(np.int32)).cuda(), None, d ** -0.5, out, ws)
    torch.cuda.synchronize()
    check_attn(cache, q, L, None, got=out.float().cpu().numpy())


@pytest.mark.parametrize("page", [None, 16])
def test_a_cache_past_32_bits(page):
    """Entries more than 4 GiB behind the pool's start."""
    lib, rng = H.sx(), np.random.default_rng(13)
    n_q, d, Hkv = 4, 128, 8
    L = np.array([100, 130])
    small = Cache(rng, 2, Hkv, d, L + n_q, page)
    q = queries(rng, 2, n_q, 16, d, "bf16")
    view, t = small.gpu()
    if page is None:
        l_max = 2_400_000
        big = [torch.zeros((2, Hkv, l_max, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
        big += [torch.ones((2, Hkv, l_max), dtype=torch.uint8, device="cuda") for _ in range(2)]
        n = t[0].shape[2]
        for a, s in zip(big, t):
            a[:, :, :n] = s
        table = None
    else:
        far = 300_000
        pages = t[0].shape[0]
        big = [torch.zeros((far + pages, Hkv, page, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
        big += [torch.ones((far + pages, Hkv, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
        for a, s in zip(big, t):
            a[far:] = s
        table = t[4] + far
    assert big[0].numel() > 1 << 32
    bv = lib.quant_kv_view(*big, table)
    check_attn(small, q, L, None, got=attn(small, q, L, view=(bv, big)))
    # and rows written there
    x = torch.randn((2, n_q, Hkv, d), device="cuda").bfloat16()
    pos = torch.from_numpy(L.astype(np.int32)).cuda()
    for v in (view, bv):
        lib.specexit_quant_kv_write(v, lib.BF16, 2, n_q, x, x, pos)
    torch.cuda.synchronize()
    for a, s in zip(big, t):
        assert torch.equal(a[:, :, :n] if page is None else a[far:], s)


def test_bad_pages_and_lengths_are_contained_and_reported():
    lib, rng = H.sx(), np.random.default_rng(14)
    L = np.array([200, 300, 250])
    n_q, d = 5, 128
    cache = Cache(rng, 3, 2, d, L + n_q, 16)
    q = queries(rng, 3, n_q, 8, d, "bf16")
    good = attn(cache, q, L)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.specexit_set_dev_status(word)
    try:
        view, t = cache.gpu()
        bad = cache.table.copy()
        bad[1, 2], bad[1, 5] = 1 << 30, -7
        t[4].copy_(torch.from_numpy(bad))
        out = attn(cache, q, L, flags=lib.FLAG_VALIDATE, view=(view, t))
        assert int(word.item()) == lib.STATUS_BAD_PAGE
        np.testing.assert_array_equal(out[[0, 2]], good[[0, 2]])
        assert np.isfinite(out).all()
        word.zero_()
        out = attn(cache, q, np.array([-5, 300, 10_000_000]), flags=lib.FLAG_VALIDATE)
        assert int(word.item()) == lib.STATUS_BAD_LENGTH
        assert np.isfinite(out).all()
        word.zero_()
        attn(cache, q, np.array([-5, 300, 10_000_000]))
        assert int(word.item()) == 0
    finally:
        lib.specexit_set_dev_status(None)


def test_other_stream_and_replays():
    """A call on a stream of its own, captured and replayed with other work between the replays: the eager result every time."""
    lib, rng = H.sx(), np.random.default_rng(15)
    L = np.array([700, 90, 2000])
    n_q, d = 7, 128
    cache = Cache(rng, 3, 2, d, L + n_q, 16)
    view, t = cache.gpu()
    qd = torch.from_numpy(queries(rng, 3, n_q, 8, d, "bf16")).cuda().bfloat16()
    ctx = torch.from_numpy(L.astype(np.int32)).cuda()
    ws = H.workspace(lib.specexit_quant_verify_attn_workspace_bytes(view, lib.BF16, 3, n_q, 8))
    x = torch.randn((3, n_q, 2, d), device="cuda").bfloat16()
    outs = [torch.empty_like(qd) for _ in range(2)]
    def calls(out, stream):
        lib.specexit_quant_kv_write(view, lib.BF16, 3, n_q, x, x, ctx, stream=stream)
        lib.specexit_quant_verify_attn(view, lib.BF16, 3, n_q, 8, qd, ctx, None, d ** -0.5, out, ws, stream=stream)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        calls(outs[0], st)
        torch.cuda.synchronize()
        lib.specexit_graph_begin(st)
        calls(outs[1], st)
        graph = lib.specexit_graph_end(st)
        try:
            for rep in range(3):
                outs[1].zero_()
                ws.fill_(255)
                lib.specexit_graph_launch(graph, st)
                torch.cuda.synchronize()
                assert torch.equal(outs[0], outs[1]), rep
                (torch.randn(1 << 16, device="cuda") * 2).sum().item()
        finally:
            lib.specexit_graph_destroy(graph)


def test_same_bits_every_time():
    rng = np.random.default_rng(16)
    L = rng.integers(0, 3000, 9)
    cache = Cache(rng, 9, 2, 128, L + 9, 16)
    q = queries(rng, 9, 9, 16, 128, "bf16")
    first = attn(cache, q, L)
    for _ in range(3):
        np.testing.assert_array_equal(attn(cache, q, L), first)
