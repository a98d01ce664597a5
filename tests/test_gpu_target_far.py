"""GPU: rotary and latent writes of many tokens, caches and logits whose offsets pass 32 bits, lists of equal logits."""
import numpy as np
import pytest
import torch

import harness as H
import test_gpu_rope as small
from target_harness import DT, Rope, dev, i32
from test_gpu_logprobs import check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,interleaved", [(None, True), (16, False)])
def test_latent_writes_of_thousands_of_tokens(dtype, page, interleaved):
    """Eight tokens to a wave, the last of them behind a sequence's count or the batch's end."""
    small.test_latent_write(dtype, page, 256, 3, 1501, interleaved, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_writes_of_thousands_of_tokens(dtype):
    """Several steps of heads to a wave, the last one not full."""
    small.test_write(dtype, 48, 128, 64, False, 13, 2, 1901)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_outside_the_pool_among_many_tokens(dtype):
    """One call of eight tokens a wave and calls of one a wave write the same bits, and neither what has no place."""
    lib, T, r = H.sx(), 4128, 128
    desc, turns = Rope(64, theta=1e4).gpu()
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = torch.randn((1, T, r + 64), generator=g, device="cuda").to(DT[dtype])
    gain = torch.ones(r, device="cuda", dtype=DT[dtype])
    ids = np.random.default_rng(4).permutation(270).astype(np.int32)[None]
    ids[0, [3, 100, 257]] = [270, -1, 1 << 30]
    table, pools = i32(ids), []
    for parts in ([T], [5, 2000, 123, 2000]):
        c = torch.full((270, 16, r + 64), -5.0, device="cuda", dtype=DT[dtype])
        at = 0
        for n in parts:
            lib.specexit_latent_kv_write(lib.latent_kv_view(c, 64, table), desc, turns, 1, n, 0, rows[:, at:at + n], gain, 1e-6, None, None, i32([at + 7]))
            at += n
        pools.append(c)
    assert torch.equal(pools[0], pools[1])
    written = (pools[0] != -5).any(-1)
    want = torch.zeros((270, 16), dtype=torch.bool)
    for p in range(7, 7 + T):
        if 0 <= ids[0, p // 16] < 270:
            want[ids[0, p // 16], p % 16] = True
    assert torch.equal(written.cpu(), want)


@pytest.mark.parametrize("paged", [False, True])
def test_a_latent_cache_past_32_bits(paged):
    """Writes, attention and compaction where entries lie more than 4 GiB behind the cache's start: the bits of a small cache."""
    lib, r, n_q, Hq = H.sx(), 512, 6, 24
    desc, turns = Rope(64, theta=1e4, interleaved=True).gpu()
    g = torch.Generator(device="cuda").manual_seed(5)
    B, L = 2, [20000, 900]
    rows = torch.randn((B, n_q, r + 64), generator=g, device="cuda").bfloat16()
    context = [torch.randn((n, r + 64), generator=g, device="cuda").bfloat16() for n in L]
    q = torch.randn((B, n_q, Hq, r + 64), generator=g, device="cuda").bfloat16()
    path, length, last = i32([[2, 4, -1, -1, -1, -1], [1, 3, 5, -1, -1, -1]]), i32([2, 3]), i32([4, 5])
    outs = []
    for far in (False, True):
        if paged:
            pages, page = (420000 if far else 400), 64            # 420000 pages of 64 entries of 1152 bytes: 31 GB
            c = torch.empty((pages, page, r + 64), dtype=torch.bfloat16, device="cuda")
            ids = np.arange(320)[None] + np.array([[0], [0]])
            ids[1, :20] = 330 + np.arange(20)
            ids = ids + (pages - 400 if far else 0)
            table = i32(ids)
            put = lambda b, n: [(int(ids[b, p]), slice(0, min(page, n - p * page)), slice(p * page, min(n, p * page + page))) for p in range((n + page - 1) // page)]
        else:
            c = torch.empty((B, 4_000_000 if far else 20480, r + 64), dtype=torch.bfloat16, device="cuda")      # the second sequence starts 4.6 GB behind
            table = None
            put = lambda b, n: [(b, slice(0, n), slice(0, n))]
        for b in range(B):
            for block, entries, source in put(b, L[b]):
                c[block, entries] = context[b][source]
        view = lib.latent_kv_view(c, 64, table)
        lib.specexit_latent_kv_write(view, desc, turns, B, n_q, 0, rows, None, 0.0, None, None, i32(L))
        out = torch.zeros((B, n_q, Hq, r), dtype=torch.bfloat16, device="cuda")
        ws = H.workspace(lib.specexit_latent_verify_attn_workspace_bytes(view, B, n_q, Hq))
        lib.specexit_latent_verify_attn(view, B, n_q, Hq, q, i32(L), None, 0.05, out, ws)
        lib.specexit_latent_kv_compact(view, 1, 0, B, n_q, i32(L), path, length, last)
        got = [out]
        for b in range(B):
            got += [c[block, entries].clone() for block, entries, _ in put(b, L[b] + n_q)]
        outs.append(got)
        torch.cuda.synchronize()
        del c, view
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_a_plain_cache_past_32_bits():
    lib, B, T, Hkv, d = H.sx(), 2, 9, 8, 128
    desc, turns = Rope(d).gpu()
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((B, T, 2 * Hkv, d), generator=g, device="cuda").bfloat16()
    got = []
    for l_max, pos in ((4096, 4000), (1_200_000, 4000), (1_200_000, 1_199_991)):              # a sequence: 2.5 GB of keys
        k, v = (torch.empty((B, Hkv, l_max, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lib.specexit_rope_kv_write(lib.kv_view(k, v), desc, turns, B, T, 0, None, x[:, :, :Hkv], x[:, :, Hkv:], None, i32([pos, pos]),
                                   i32([[t + 4000 - pos for t in range(T)]] * B))
        got.append([a[:, :, pos:pos + T].clone() for a in (k, v)])
        torch.cuda.synchronize()
        del k, v
    for other in got[1:]:
        assert torch.equal(got[0][0], other[0]) and torch.equal(got[0][1], other[1])
    assert torch.equal(got[0][1], x[:, :, Hkv:].transpose(1, 2))


def test_logits_past_32_bits():
    """Rows behind 2^31 logits give the bits that they give in a call of their own."""
    M, V, last = 16000, 140001, 300
    x = torch.empty((M, V), dtype=torch.bfloat16, device="cuda")
    x[:-last].fill_(0.0)
    x[-last:] = torch.randn((last, V), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").bfloat16() * 3
    tokens = np.random.default_rng(7).integers(0, V, (M, 1))
    whole = run(x, V, tokens, 5, dtype="bf16")
    part = run(x[-last:], V, tokens[-last:], 5, dtype="bf16")
    for a, b in zip(whole, part):
        assert np.array_equal(a[-last:], b)
    check(x[-3:], V, tokens[-3:], 5, dtype="bf16", got=[a[-3:] for a in whole])
    assert np.array_equal(whole[2][0], np.arange(5)) and abs(whole[0][0, 0] + np.log(V)) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lists_of_equal_logits_that_run_over(dtype):
    """Thousands of candidates in a few groups and in all: the list is cut again and again, in every workgroup of a large call, with the same result each time."""
    V, M = 33000, 300
    x = torch.zeros((M, V), device="cuda")
    x[1::3, 5000:9000] = 1.0
    x[2::3, ::2] = 1.0
    x[::7, 32990:] = 2.0
    x = x.to(DT[dtype])
    tokens = np.zeros((M, 1), int)
    first = run(x, V, tokens, 32, dtype=dtype)
    check(x[:42], V, tokens[:42], 32, dtype=dtype, got=[a[:42] for a in first])
    for _ in range(3):
        for a, b in zip(first, run(x, V, tokens, 32, dtype=dtype)):
            assert np.array_equal(a, b)
