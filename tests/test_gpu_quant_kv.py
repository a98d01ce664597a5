"""GPU: rows written to the 8-bit cache and moved in it, against the oracle; bit for bit."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O
from workloads import gen

import harness as H
from quant_harness import Cache

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()


def rows(rng, shape, dtype):
    x = (rng.standard_normal(shape) * np.exp(2 * rng.standard_normal(shape[:-1] + (1,)))).astype(np.float32)
    return gen.round_to_bf16(x) if dtype == "bf16" else x


def expected(cache, x, pos, count, which):
    """The pools after the call."""
    codes, scale = (cache.k, cache.ks) if which == "k" else (cache.v, cache.vs)
    codes, scale = codes.copy(), scale.copy()
    c, s = O.quant_rows(x)
    for b in range(x.shape[0]):
        for t in range(count[b]):
            at = cache.at(b, pos[b] + t)
            codes[at], scale[at] = c[b, t], s[b, t]
    return codes, scale


def check(cache, t, want_k, want_v):
    got = [a.cpu().numpy() for a in t[:4]]
    for g, w in zip(got, (want_k[0], want_v[0], want_k[1], want_v[1])):
        np.testing.assert_array_equal(g, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [None, 16, 48])
@pytest.mark.parametrize("B,T,Hkv", [(1, 1, 1), (3, 7, 2), (2, 133, 5)])
def test_rows_are_written(dtype, d, page, B, T, Hkv):
    lib, rng = H.sx(), np.random.default_rng(B * 1000 + T)
    pos = rng.integers(0, 70, B)
    cache = Cache(rng, B, Hkv, d, pos + T, page)
    view, t = cache.gpu()
    k, v = rows(rng, (B, T, Hkv, d), dtype), rows(rng, (B, T, Hkv, d), dtype)
    want = [expected(cache, x, pos, [T] * B, n) for x, n in ((k, "k"), (v, "v"))]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lib.specexit_quant_kv_write(view, lib.dtype_code(dt), B, T, torch.from_numpy(k).cuda().to(dt), torch.from_numpy(v).cuda().to(dt), i32(pos))
    torch.cuda.synchronize()
    check(cache, t, *want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ragged_counts_out_of_a_fused_projection(dtype):
    lib, rng = H.sx(), np.random.default_rng(5)
    B, T, Hq, Hkv, d = 4, 40, 6, 2, 128
    pos, count = np.array([0, 33, 5, 70]), np.array([40, 0, 17, 99])
    cache = Cache(rng, B, Hkv, d, pos + T, 32)
    view, t = cache.gpu()
    x = rows(rng, (B, T, Hq + 2 * Hkv, d), dtype)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.from_numpy(x).cuda().to(dt)
    n = np.minimum(count, T)
    want = [expected(cache, x[:, :, Hq + i * Hkv:Hq + (i + 1) * Hkv], pos, n, w) for i, w in enumerate("kv")]
    lib.specexit_quant_kv_write(view, lib.dtype_code(dt), B, T, g[:, :, Hq:Hq + Hkv], g[:, :, Hq + Hkv:], i32(pos), i32(count))
    torch.cuda.synchronize()
    check(cache, t, *want)
    # a negative count writes nothing
    lib.specexit_quant_kv_write(view, lib.dtype_code(dt), B, T, g[:, :, :Hkv], g[:, :, Hkv:2 * Hkv], i32(pos), i32([-1, -7, 0, -2 ** 31]))
    torch.cuda.synchronize()
    check(cache, t, *want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_value_a_row_can_have(dtype):
    lib, rng = H.sx(), np.random.default_rng(7)
    T, d = 64, 64
    x = rows(rng, (1, T, 1, d), dtype)
    x[0, 0] = 0.0
    x[0, 1, 0, 5], x[0, 1, 0, 6], x[0, 1, 0, 7] = np.inf, -np.inf, np.nan
    x[0, 2] = np.nan
    x[0, 3, 0] = 1e-39
    x[0, 4, 0, :2] = 3.3e38, -1e-30
    x[0, 5, 0] = -0.0
    for e in range(6, 40):                                  # the largest at and next to 448 2^e, small ones down to the subnormal codes
        x[0, e, 0] = np.ldexp(rng.standard_normal(d) * np.exp2(-rng.integers(0, 20, d)), e - 20)
        x[0, e, 0, 0] = np.ldexp([448.0, 450.0, 446.0][e % 3], e - 30)
    x = gen.round_to_bf16(x) if dtype == "bf16" else x.astype(np.float32)
    cache = Cache(rng, 1, 1, d, [T], None)
    view, t = cache.gpu()
    want = expected(cache, x, [0], [T], "k"), expected(cache, x, [0], [T], "v")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.from_numpy(x).cuda().to(dt)
    lib.specexit_quant_kv_write(view, lib.dtype_code(dt), 1, T, g, g, i32([0]))
    torch.cuda.synchronize()
    check(cache, t, *want)


def test_entries_outside_the_cache_and_bad_pages_are_skipped_and_reported():
    lib, rng = H.sx(), np.random.default_rng(9)
    B, T, Hkv, d = 3, 20, 2, 128
    cache = Cache(rng, B, Hkv, d, [64] * B, 16)
    view, t = cache.gpu()
    x = rows(rng, (B, T, Hkv, d), "bf16")
    g = torch.from_numpy(x).cuda().bfloat16()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.specexit_set_dev_status(word)
    try:
        pos = np.array([-5, 50, 10])                        # five rows in front, six behind
        codes, scale = [], []
        ck, sk = O.quant_rows(x)
        want = [cache.k.copy(), cache.v.copy(), cache.ks.copy(), cache.vs.copy()]
        for b in range(B):
            for i in range(T):
                if 0 <= pos[b] + i < 64:
                    at = cache.at(b, pos[b] + i)
                    want[0][at] = want[1][at] = ck[b, i]
                    want[2][at] = want[3][at] = sk[b, i]
        lib.specexit_quant_kv_write(view, lib.BF16, B, T, g, g, i32(pos), flags=lib.FLAG_VALIDATE)
        torch.cuda.synchronize()
        assert int(word.item()) == lib.STATUS_BAD_LENGTH
        for a, w in zip(t[:4], want):
            np.testing.assert_array_equal(a.cpu().numpy(), w)
        word.zero_()
        bad = cache.table.copy()
        bad[1, 0], bad[2, 1] = 1 << 30, -1
        t[4].copy_(torch.from_numpy(bad))
        before = [a.clone() for a in t[:4]]
        lib.specexit_quant_kv_write(view, lib.BF16, B, T, g, g, i32([0, 0, 16]), i32([0, 16, 16]), flags=lib.FLAG_VALIDATE)
        torch.cuda.synchronize()
        assert int(word.item()) == lib.STATUS_BAD_PAGE
        for a, w in zip(t[:4], before):
            assert torch.equal(a, w)
    finally:
        lib.specexit_set_dev_status(None)


def compact_case(rng, B, n_q, d, page, layers, Hkv=3):
    L = rng.integers(0, 60, B)
    cache = Cache(rng, B, Hkv, d, L + n_q, page)
    shape = cache.k.shape
    pools = [rng.integers(0, 256, (layers,) + shape).astype(np.uint8) for _ in range(2)]
    pools += [rng.integers(1, 255, (layers,) + shape[:-1]).astype(np.uint8) for _ in range(2)]
    path, length = np.full((B, n_q), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        m = int(rng.integers(0, n_q))
        path[b, :m] = np.sort(rng.choice(np.arange(1, n_q), m, replace=False))
        length[b] = m
    return cache, L, pools, path, length


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,layers,n_q", [(128, None, 3, 16), (64, 16, 2, 7), (128, 48, 1, 64), (64, None, 1, 2)])
def test_accepted_path_moves(dtype, d, page, layers, n_q):
    lib, rng = H.sx(), np.random.default_rng(d + n_q)
    B, D = 5, 64
    cache, L, pools, path, length = compact_case(rng, B, n_q, d, page, layers)
    last = np.array([path[b, length[b] - 1] if length[b] else 0 for b in range(B)], np.int32)
    hidden = gen.round_to_bf16(rng.standard_normal((B, n_q, D)).astype(np.float32))
    want = [np.empty_like(p) for p in pools]
    for l in range(layers):
        want[0][l], want[1][l] = O.kv_compact(pools[0][l], pools[1][l], L, path, length, cache.table, page or 16)
        s = [p[l][..., None] for p in pools[2:]]
        a, b = O.kv_compact(s[0], s[1], L, path, length, cache.table, page or 16)
        want[2][l], want[3][l] = a[..., 0], b[..., 0]
    t = [torch.from_numpy(p).cuda() for p in pools]
    table = None if cache.table is None else torch.from_numpy(cache.table).cuda()
    view = lib.quant_kv_view(t[0][0], t[1][0], t[2][0], t[3][0], table)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    nxt = torch.zeros((B, D), dtype=dt, device="cuda")
    lib.specexit_quant_kv_compact(view, layers, t[0][0].numel(), t[2][0].numel(), B, n_q, i32(L), i32(path), i32(length), lib.dtype_code(dt),
                                  i32(last), torch.from_numpy(hidden).cuda().to(dt), D, nxt)
    torch.cuda.synchronize()
    for a, w in zip(t, want):
        np.testing.assert_array_equal(a.cpu().numpy(), w)
    np.testing.assert_array_equal(nxt.float().cpu().numpy(), hidden[np.arange(B), last])


def test_bad_nodes_lengths_and_pages_move_nothing_and_are_reported():
    lib, rng = H.sx(), np.random.default_rng(3)
    B, n_q, d = 4, 8, 128
    cache, L, pools, path, length = compact_case(rng, B, n_q, d, 16, 1)
    path[:] = -1
    path[:, :2] = [3, 5]
    length[:] = 2
    path[0, 1] = 99                                          # node outside the block: its row stays where it is
    L[1] = 1000000
    L[2] = -3
    length[3] = 500                                          # forced to n_q - 1: the further nodes are -1
    t = [torch.from_numpy(p).cuda() for p in pools]
    table = torch.from_numpy(cache.table).cuda()
    view = lib.quant_kv_view(t[0][0], t[1][0], t[2][0], t[3][0], table)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = [p.copy() for p in pools]
    for b, js in ((0, (0,)), (3, (0, 1))):
        for j in js:
            src, dst = cache.at(b, L[b] + path[b, j]), cache.at(b, L[b] + 1 + j)
            for w, p in zip(want, pools):
                w[0][dst] = p[0][src]
    lib.specexit_set_dev_status(word)
    try:
        lib.specexit_quant_kv_compact(view, 1, 0, 0, B, n_q, i32(L), i32(path), i32(length), flags=lib.FLAG_VALIDATE)
        torch.cuda.synchronize()
        assert int(word.item()) in (lib.STATUS_BAD_LENGTH, lib.STATUS_BAD_NODE)
    finally:
        lib.specexit_set_dev_status(None)
    for a, w in zip(t, want):
        np.testing.assert_array_equal(a.cpu().numpy(), w)


@pytest.mark.parametrize("d,page,n_q", [(128, 16, 17), (128, None, 18), (128, 16, 33), (64, None, 33), (64, 16, 34), (64, 16, 64)])
def test_rows_of_a_wave(d, page, n_q):
    """Blocks on both sides of the size up to which a lane moves four pieces."""
    test_accepted_path_moves("bf16", d, page, 2, n_q)
