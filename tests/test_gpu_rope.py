"""GPU: rotary positions and the write of a block's rows into the plain and the latent cache, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O

import harness as H
from target_harness import DT, HALF, U, Latent, Rope, dev, depths, i32, stored, tree_masks

pytestmark = pytest.mark.gpu

SCALED = [dict(), dict(scaling=1, factor=4.0), dict(scaling=2, factor=8.0, high=4.0, orig_len=8192, theta=5e5),
          dict(scaling=3, factor=32.0, amplitude=1.3466, theta=1e4)]


def check(got, ref, bound, what):
    over = np.abs(got - ref) / np.maximum(bound, 1e-30)
    assert np.isfinite(got).all() and over.max(initial=0.0) <= 1.0, (what, float(over.max()))


@pytest.mark.parametrize("scaling", range(4))
def test_table(scaling):
    r = Rope(128, **SCALED[scaling])
    _, turns = r.gpu()
    got = turns.cpu().numpy().view(np.uint64).astype(O.LONG)
    want = r.f / (2 * O.LONG(np.pi) + O.LONG(2.4492935982947064e-16)) * O.LONG(2.0) ** 64
    # 64-bit arithmetic: a power (exponent times logarithm: 14 units at theta 1e6), and four operations; then cut to a whole number, of which the
    # slowest pairs have few: 10^-6 / 2 pi turns are 2.9e12, a unit 3.4e-13 of them
    assert (np.abs(got - want) < 1 + 32 * 2.0 ** -53 * want).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (64, 26), (64, 64), (16, 16), (48, 16), (512, 256), (192, 2), (80, 80)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows(dtype, d, rot, interleaved):
    lib, rng = H.sx(), np.random.default_rng(d + rot)
    r = Rope(rot, interleaved=interleaved, **SCALED[rot // 2 % 4])
    desc, turns = r.gpu()
    B, T, heads = 3, 5, 7
    pos, count = np.array([0, 40000, 123456]), np.array([5, 0, 3])
    x = stored(rng.standard_normal((B, T, heads, d)) * 3, dtype)
    ref = r.heads(x, pos[:, None] + np.arange(T))
    xd = dev(x, dtype)
    guard = H.Guarded()
    out = guard.empty(x.shape, DT[dtype])
    out.fill_(-9.0)
    lib.specexit_rope(lib.dtype_code(DT[dtype]), desc, turns, B, T, heads, d, xd, out, i32(pos), None, i32(count))
    guard.check()
    got = H.host(out)
    for b in range(B):
        check(got[b, :count[b]], ref[b, :count[b]], r.bound(x, ref, dtype)[b, :count[b]], b)
        assert (got[b, count[b]:] == -9).all()
    assert np.array_equal(got[0, ..., rot:], x[0, ..., rot:].astype(np.float32))
    # in place, within a wider row, every token, by depth
    wide = torch.full((B, T, heads + 3, d), 7.0, dtype=DT[dtype], device="cuda")
    part = wide[:, :, 1:1 + heads]
    part.copy_(xd)
    _, parent = tree_masks(rng, B, T)
    off = depths(parent)
    lib.specexit_rope(lib.dtype_code(DT[dtype]), desc, turns, B, T, heads, d, part, part, i32(pos), i32(off))
    ref = r.heads(x, pos[:, None] + off)
    check(H.host(part), ref, r.bound(x, ref, dtype), "in place")
    assert bool((wide[:, :, 0] == 7).all()) and bool((wide[:, :, 1 + heads:] == 7).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions_and_values_that_are_not_finite(dtype):
    lib, rng = H.sx(), np.random.default_rng(5)
    r = Rope(64, theta=1e4)
    desc, turns = r.gpu()
    pos = np.array([2 ** 31 - 2, 2 ** 30 + 12345, 10 ** 6 + 1])
    x = stored(rng.standard_normal((3, 1, 4, 128)), dtype)
    x[2, 0, 3, 64:] = [np.inf, -np.inf, np.nan, 1.0] * 16          # not rotated: stays
    ref = r.heads(x, pos[:, None])
    out = torch.zeros((3, 1, 4, 128), dtype=DT[dtype], device="cuda")
    lib.specexit_rope(lib.dtype_code(DT[dtype]), desc, turns, 3, 1, 4, 128, dev(x, dtype), out, i32(pos))
    got = H.host(out)
    assert np.array_equal(got[2, 0, 3, 64:], x[2, 0, 3, 64:], equal_nan=True)
    # the table's rounding (32 units of 2^-53 of a frequency of at most one) at the position, as an angle of |x| + |y|
    slack = pos[:, None, None, None] * 32.0 * 2.0 ** -53 * 2 * np.abs(x[..., :64]).max()
    over = np.abs(got - ref)[..., :64] / (r.bound(x, ref, dtype)[..., :64] + slack)
    assert over.max() <= 1.0, over.max()


def test_positions_out_of_range_are_forced_and_reported():
    lib = H.sx()
    r = Rope(64)
    desc, turns = r.gpu()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.randn((2, 1, 2, 64), device="cuda")
    out = torch.zeros_like(x)
    lib.specexit_set_dev_status(word)
    try:
        lib.specexit_rope(lib.F32, desc, turns, 2, 1, 2, 64, x, out, i32([5, 2 ** 31 - 1]), i32([[-9], [7]]), flags=lib.FLAG_VALIDATE)
        torch.cuda.synchronize()
        assert int(word.item()) == lib.STATUS_BAD_LENGTH
    finally:
        lib.specexit_set_dev_status(None)
    assert torch.equal(out[0], x[0])                               # position 0
    ref = r.heads(x.cpu().numpy(), np.array([[0], [2 ** 31 - 1]]))
    assert np.abs(H.host(out) - ref).max() < 1e-4


def places(rng, B, Hkv, d, need, page, dtype):
    if page is None:
        k = torch.full((B, Hkv, max(need), d), -5.0, dtype=DT[dtype], device="cuda")
        return k, k.clone(), None, lambda b, p: (b, slice(None), p)
    lat = Latent(rng, B, 128, need, dtype, page)
    k = torch.full((lat.c.shape[0], Hkv, page, d), -5.0, dtype=DT[dtype], device="cuda")
    return k, k.clone(), lat.table, lambda b, p: (int(lat.table[b, p // page]), slice(None), p % page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16, 48])
@pytest.mark.parametrize("d,rot,interleaved,Hq,Hkv,T", [(128, 128, False, 32, 8, 7), (64, 32, True, 6, 2, 33), (128, 26, False, 0, 3, 1), (64, 64, False, 5, 5, 600)])
def test_write(dtype, page, d, rot, interleaved, Hq, Hkv, T):
    lib, rng = H.sx(), np.random.default_rng(T + d)
    r = Rope(rot, interleaved=interleaved)
    desc, turns = r.gpu()
    B = 3
    pos, count = np.array([0, 15, 47]), np.array([T, max(T - 1, 0), (T + 1) // 2])
    k, v, table, at = places(rng, B, Hkv, d, [int(p) + T for p in pos], page, dtype)
    view = lib.kv_view(k, v, None if table is None else i32(table))
    fused = stored(rng.standard_normal((B, T, Hq + 2 * Hkv, d)), dtype)
    x = dev(fused, dtype)
    guard = H.Guarded()
    q = guard.empty((B, T, Hq, d), DT[dtype])
    q.fill_(-5.0)
    _, parent = tree_masks(rng, B, T)
    off = depths(parent) if T < 64 else None
    lib.specexit_rope_kv_write(view, desc, turns, B, T, Hq, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], q, i32(pos),
                               None if off is None else i32(off), i32(count))
    guard.check()
    ref = r.heads(fused, pos[:, None] + (np.arange(T) if off is None else off))
    bound = r.bound(fused, ref, dtype)
    got, kg, vg = H.host(q), H.host(k), H.host(v)
    want_v, seen = np.full(vg.shape, -5.0, np.float32), np.zeros(kg.shape, bool)
    for b in range(B):
        n = count[b]
        check(got[b, :n], ref[b, :n, :Hq], bound[b, :n, :Hq], "q") if Hq and n else None
        assert (got[b, n:] == -5).all()
        for t in range(n):
            p = at(b, int(pos[b]) + t)
            check(kg[p], ref[b, t, Hq:Hq + Hkv], bound[b, t, Hq:Hq + Hkv], "k")
            want_v[p], seen[p] = fused[b, t, Hq + Hkv:], True
    assert np.array_equal(vg, want_v) and (kg[~seen] == -5).all()


def test_write_outside_the_cache_or_the_pool_is_left_out_and_reported():
    lib, rng = H.sx(), np.random.default_rng(8)
    r = Rope(64)
    desc, turns = r.gpu()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.randn((2, 4, 2, 64), device="cuda")
    lib.specexit_set_dev_status(word)
    try:
        for pos, table, code in (([30, 0], [[0, 1], [2, 3]], lib.STATUS_BAD_LENGTH), ([-2, 0], [[0, 1], [2, 3]], lib.STATUS_BAD_LENGTH),
                                 ([0, 14], [[0, 1], [2, 99]], lib.STATUS_BAD_PAGE), ([0, 14], [[0, 1], [2, -1]], lib.STATUS_BAD_PAGE)):
            k, v = (torch.full((4, 2, 16, 64), -5.0, device="cuda") for _ in range(2))
            view = lib.kv_view(k, v, i32(table))
            print("rope write at", pos, "pages", table, flush=True)
            lib.specexit_rope_kv_write(view, desc, turns, 2, 4, 0, None, x, x, None, i32(pos), flags=lib.FLAG_VALIDATE)
            torch.cuda.synchronize()
            assert int(word.item()) == code
            word.zero_()
            want = torch.full_like(v, -5.0)
            for b in range(2):
                for t in range(4):
                    p = pos[b] + t
                    if 0 <= p < 32 and 0 <= table[b][p // 16] < 4:
                        want[table[b][p // 16], :, p % 16] = x[b, t]
            assert torch.equal(v, want)
            # the same of a latent cache
            c = torch.full((4, 16, 192), -5.0, device="cuda")
            rows = torch.randn((2, 4, 192), device="cuda")
            lib.specexit_latent_kv_write(lib.latent_kv_view(c, 64, i32(table)), desc, turns, 2, 4, 0, rows, None, 0.0, None, None, i32(pos),
                                         flags=lib.FLAG_VALIDATE)
            torch.cuda.synchronize()
            assert int(word.item()) == code
            word.zero_()
            want = torch.full_like(c, -5.0)
            for b in range(2):
                for t in range(4):
                    p = pos[b] + t
                    if 0 <= p < 32 and 0 <= table[b][p // 16] < 4:
                        want[table[b][p // 16], p % 16, :128] = rows[b, t, :128]
            assert torch.equal(c[..., :128], want[..., :128]) and torch.equal(c[..., 128:] == -5, want[..., :64] == -5)
    finally:
        lib.specexit_set_dev_status(None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 64])
@pytest.mark.parametrize("r,heads,T,interleaved,gain", [(512, 16, 7, True, True), (256, 3, 40, False, True), (128, 0, 700, True, False), (512, 33, 1, False, True)])
def test_latent_write(dtype, page, r, heads, T, interleaved, gain):
    lib, rng = H.sx(), np.random.default_rng(r + T)
    ro = Rope(64, theta=1e4, interleaved=interleaved, scaling=3, factor=40.0, amplitude=1.1)
    desc, turns = ro.gpu()
    B, w = 3, r + 64
    pos, count = np.array([0, 15, 47]), np.array([T, max(T - 1, 0), (T + 1) // 2])
    lat = Latent(rng, B, r, pos + T, dtype, page)
    view, c, _ = lat.gpu()
    rows = stored(rng.standard_normal((B, T, w + 8)) * np.exp(rng.standard_normal((B, T, 1))), dtype)
    g = stored(1 + 0.2 * rng.standard_normal(r), dtype) if gain else None
    qp = stored(rng.standard_normal((B, T, max(heads, 1), 192)), dtype)
    q0 = stored(rng.standard_normal((B, T, max(heads, 1), w)), dtype)
    q = dev(q0, dtype)
    lib.specexit_latent_kv_write(view, desc, turns, B, T, heads, dev(rows, dtype)[..., :w], None if g is None else dev(g, dtype), 1e-5,
                                 dev(qp, dtype)[..., 128:] if heads else None, q if heads else None, i32(pos), None, i32(count))
    got, gq, want, bound = H.host(c), H.host(q), lat.c.astype(np.float64), np.zeros(lat.c.shape)
    at = pos[:, None] + np.arange(T)
    for b in range(B):
        if not count[b]:
            continue
        ref = O.latent_rows(rows[b, :, :w], g, float(np.float32(1e-5)), at[b], ro.f, interleaved, ro.amplitude)
        # the sum of squares passes 8 + 6 steps, halved by the root, with quotient, root and two products: 16 roundings
        tol = np.concatenate([(2.0 ** -20 + (HALF[dtype] if dtype == "bf16" else U)) * np.abs(ref[:, :r]),
                              ro.bound(rows[b, :, r:w], ref[:, r:], dtype)], 1)
        for t in range(count[b]):
            want[lat.at(b, int(pos[b]) + t)], bound[lat.at(b, int(pos[b]) + t)] = ref[t], tol[t]
    assert (np.abs(got - want) <= bound).all()
    if not heads:
        return
    ref = ro.heads(qp[..., 128:], at)
    tol = ro.bound(qp[..., 128:], ref, dtype)
    for b in range(B):
        n = count[b]
        assert (np.abs(gq[b, :n, :, r:] - ref[b, :n]) <= tol[b, :n]).all()
        assert np.array_equal(gq[b, n:], q0[b, n:]) and np.array_equal(gq[b, :, :, :r], q0[b, :, :, :r])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16])
@pytest.mark.parametrize("n_q,r", [(2, 128), (16, 512), (64, 512)])
def test_latent_compaction(dtype, page, n_q, r):
    lib, rng = H.sx(), np.random.default_rng(n_q)
    B, layers, D, w = 4, 3, 72, r + 64
    L = np.array([0, 17, 40, 5])
    lat = Latent(rng, B, r, L + n_q, dtype, page)
    one = lat.c.shape
    c0 = stored(rng.standard_normal((layers,) + one), dtype)
    c = dev(c0, dtype)
    path, length, last = np.full((B, n_q), -1, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
    for b in range(1, B):
        m = int(rng.integers(1, n_q)) if b < 3 else n_q - 1
        nodes = np.sort(rng.choice(np.arange(1, n_q), m, replace=False))
        path[b, :m], length[b], last[b] = nodes, m, nodes[-1]
    hidden = stored(rng.standard_normal((B, n_q, D)), dtype)
    nxt = torch.zeros((B, D), dtype=DT[dtype], device="cuda")
    view = lib.latent_kv_view(c[0], 64, None if lat.table is None else i32(lat.table))
    lib.specexit_latent_kv_compact(view, layers, c[0].numel() * c.element_size(), B, n_q, i32(L), i32(path), i32(length), i32(last), dev(hidden, dtype), D, nxt)
    want = c0.copy()
    for b in range(B):
        for j in range(length[b]):
            want[(slice(None),) + lat.at(b, int(L[b]) + 1 + j)] = c0[(slice(None),) + lat.at(b, int(L[b] + path[b, j]))]
    assert np.array_equal(H.host(c), want) and np.array_equal(H.host(nxt), hidden[np.arange(B), last])
