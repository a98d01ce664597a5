"""GPU: rounds of a target served from an 8-bit cache with sampled tokens - block rows written, attention, LM head, draw, acceptance, compaction -
against the oracle, stage by stage on the library's own data, eager and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O
from workloads import gen

import harness as H
from quant_harness import Cache, attn_bound, tree_masks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16])
@pytest.mark.parametrize("tree", [False, True])
def test_rounds(dtype, page, tree):
    lib, rng = H.sx(), np.random.default_rng(21 + tree)
    B, n_q, Hq, Hkv, d, D, V, rounds = 3, 6, 8, 2, 64, 512, 4001, 3
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    code = lib.dtype_code(dt)
    st_ = (lambda x: gen.round_to_bf16(np.asarray(x, np.float32))) if dtype == "bf16" else (lambda x: np.asarray(x, np.float32))
    dev = lambda x, t=None: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(t or dt)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    L = np.array([40, 0, 77])
    cache = Cache(rng, B, Hkv, d, L + rounds * n_q + n_q, page)
    view, t = cache.gpu()
    w_head = dev(st_(rng.standard_normal((V, D)) * 0.08))
    parent = None
    if tree:
        parent = np.full((B, n_q), -1, np.int64)
        for b in range(B):
            for c in range(1, n_q):
                parent[b, c] = rng.integers(0, c)
    mask = gen.ancestor_masks(parent) if tree else None
    gp = None if parent is None else i32(parent)
    gm = None if mask is None else H.dev(mask)
    # one set of buffers, refilled every round: what a graph replays
    k_rows, v_rows = (torch.zeros((B, n_q, Hkv, d), dtype=dt, device="cuda") for _ in range(2))
    q = torch.zeros((B, n_q, Hq, d), dtype=dt, device="cuda")
    hid = torch.zeros((B, n_q, D), dtype=dt, device="cuda")
    out, nxt = torch.zeros_like(q), torch.zeros((B, D), dtype=dt, device="cuda")
    logits = torch.zeros((B * n_q, V), device="cuda")
    am, tok = (torch.zeros((B, n_q), dtype=torch.int32, device="cuda") for _ in range(2))
    block, path = (torch.zeros((B, n_q), dtype=torch.int32, device="cuda") for _ in range(2))
    prob, u = torch.zeros((B, n_q), device="cuda"), torch.zeros((B, n_q), device="cuda")
    ctx, new_ctx = i32(L), i32(L)
    temp, top_k, top_p = torch.tensor([0.6, 1.0, 0.0], device="cuda"), i32([20, 0, 0]), torch.tensor([0.95, 0.9, 1.0], device="cuda")
    sig = torch.full((B, 3), 0.5, device="cuda")
    ewma, n_obs, thinking = torch.zeros((B, 3), device="cuda"), i32([0] * B), i32([1] * B)
    length, recover, last, flag = (i32([0] * B) for _ in range(4))
    split = i32([V - 1])
    cfg = lib.exit_cfg(stop_think_token=5)
    scale = d ** -0.5
    ws_a = H.workspace(lib.specexit_quant_verify_attn_workspace_bytes(view, code, B, n_q, Hq))
    ws_h = H.workspace(lib.specexit_lmhead_argmax_workspace_bytes(code, B * n_q, D, V, 0))
    ws_s = H.workspace(lib.specexit_sample_workspace_bytes(lib.F32, B * n_q, V))

    def one_round(stream):
        lib.specexit_quant_kv_write(view, code, B, n_q, k_rows, v_rows, ctx, stream=stream)
        lib.specexit_quant_verify_attn(view, code, B, n_q, Hq, q, ctx, gm, scale, out, ws_a, stream=stream)
        lib.specexit_lmhead_argmax(code, B * n_q, D, V, 0, hid, w_head, am, logits_dbg=logits, workspace=ws_h, stream=stream)
        lib.specexit_sample(lib.F32, B * n_q, V, logits, u, tok, prob, temp, top_k, top_p, rows_per_seq=n_q, workspace=ws_s, stream=stream)
        lib.specexit_accept_exit(cfg, B, n_q, block, gp, tok, sig, ctx, split, 1, ewma, n_obs, thinking, None, length, path, recover, last, flag,
                                 new_ctx, stream=stream)
        lib.specexit_quant_kv_compact(view, 1, 0, 0, B, n_q, ctx, path, length, code, last, hid, D, nxt, stream=stream)

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = None
    with torch.cuda.stream(stream):
        for rnd in range(rounds + 1):
            x = {n: st_(rng.standard_normal(s) * m) for n, s, m in (("k", (B, n_q, Hkv, d), 1), ("v", (B, n_q, Hkv, d), 2), ("q", (B, n_q, Hq, d), 1),
                                                                    ("h", (B, n_q, D), 1))}
            for name, to in (("k", k_rows), ("v", v_rows), ("q", q), ("h", hid)):
                to.copy_(dev(x[name]))
            un = rng.random((B, n_q), np.float32)
            u.copy_(torch.from_numpy(un))
            # drafts that are sometimes what will be drawn: the oracle's draw of an earlier look at the logits
            lib.specexit_lmhead_argmax(code, B * n_q, D, V, 0, hid, w_head, am, logits_dbg=logits, workspace=ws_h, stream=stream)
            torch.cuda.synchronize()
            z = logits.cpu().numpy()
            per = [(0.6, 20, 0.95), (1.0, 0, 0.9), (0.0, 0, 1.0)]
            drawn = np.array([[O.sample(z[b * n_q + i], un[b, i], float(np.float32(per[b][0])), per[b][1], float(np.float32(per[b][2])))[0]
                               for i in range(n_q)] for b in range(B)])
            blk = rng.integers(0, V, (B, n_q)).astype(np.int32)
            for b in range(B):
                for c in range(1, n_q):
                    if rng.random() < 0.7:
                        blk[b, c] = drawn[b, parent[b, c] if tree else c - 1]
            block.copy_(torch.from_numpy(blk))
            ctx.copy_(i32(L))
            before = [a.clone() for a in t[:4]]
            logits.zero_()
            torch.cuda.synchronize()
            if rnd == rounds:                                    # the last round also from a graph: the same state, replayed twice
                lib.specexit_graph_begin(stream)
                one_round(stream)
                graph = lib.specexit_graph_end(stream)
                thinking0, n0, e0 = thinking.clone(), n_obs.clone(), ewma.clone()
                one_round(stream)
                torch.cuda.synchronize()
                names = dict(out=out, tok=tok, prob=prob, length=length, path=path, recover=recover, nxt=nxt, new_ctx=new_ctx, k=t[0], v=t[1], ks=t[2], vs=t[3])
                eager = {n: a.clone() for n, a in names.items()}
                for rep in range(2):
                    for a, b0 in zip(t[:4], before):
                        a.copy_(b0)
                    thinking.copy_(thinking0); n_obs.copy_(n0); ewma.copy_(e0)
                    for a in (out, tok, prob, length, path, recover, nxt, new_ctx):
                        a.zero_()
                    lib.specexit_graph_launch(graph, stream)
                    torch.cuda.synchronize()
                    for n, a in names.items():
                        assert torch.equal(a, eager[n]), (rep, n)
                lib.specexit_graph_destroy(graph)
                break
            one_round(stream)
            torch.cuda.synchronize()
            # ---- the cache with the block's rows in it
            for which, codes, sc in (("k", cache.k, cache.ks), ("v", cache.v, cache.vs)):
                cq, sq = O.quant_rows(x[which])
                for b in range(B):
                    for i in range(n_q):
                        at = cache.at(b, L[b] + i)
                        codes[at], sc[at] = cq[b, i], sq[b, i]
            k, v = cache.values()
            ref = O.verify_attn(x["q"], k, v, L, mask, scale, cache.table, page or 16)
            weighed = O.verify_attn(x["q"], k, np.abs(v), L, mask, scale, cache.table, page or 16)
            err = np.abs(out.float().cpu().numpy() - ref) / attn_bound(ref, weighed, x["q"], k, v, int(L.max()) + n_q, scale, dtype)
            assert err.max() <= 1.0, float(err.max())
            # ---- head, draws, acceptance
            np.testing.assert_array_equal(logits.cpu().numpy(), z)
            assert H.rel_err(z, x["h"].reshape(-1, D).astype(np.float64) @ w_head.double().cpu().numpy().T) < H.TOL[dtype]
            np.testing.assert_array_equal(tok.cpu().numpy(), drawn)
            acc = [O.greedy_accept(blk[b], parent[b] if tree else np.arange(-1, n_q - 1), drawn[b]) for b in range(B)]
            got_path, got_len = path.cpu().numpy(), length.cpu().numpy()
            for b in range(B):
                want = list(acc[b][0]) if isinstance(acc[b], tuple) else list(acc[b])
                assert list(got_path[b, :got_len[b]]) == want, (b, got_path[b], want)
            # ---- the compacted cache, codes and scales
            cache.k, cache.v = O.kv_compact(cache.k, cache.v, L, got_path, got_len, cache.table, page or 16)
            a, b2 = O.kv_compact(cache.ks[..., None], cache.vs[..., None], L, got_path, got_len, cache.table, page or 16)
            cache.ks, cache.vs = a[..., 0], b2[..., 0]
            for a, w in zip(t[:4], (cache.k, cache.v, cache.ks, cache.vs)):
                np.testing.assert_array_equal(a.cpu().numpy(), w)
            L = new_ctx.cpu().numpy().astype(np.int64)


def test_two_streams_at_once():
    """Writes, attention and draws of two inputs on two streams, each with a cache and workspaces of its own, against the same calls one by one."""
    lib, rng = H.sx(), np.random.default_rng(41)
    B, n_q, Hq, Hkv, d, V = 3, 5, 8, 2, 128, 20000
    sets = []
    for i in range(2):
        L = np.array([700 + 900 * i, 33, 2000 - 1000 * i])
        cache = Cache(rng, B, Hkv, d, L + n_q, 16)
        view, t = cache.gpu()
        s = dict(view=view, keep=t, L=torch.from_numpy(L.astype(np.int32)).cuda())
        for n in ("k", "v"):
            s[n] = torch.from_numpy(rng.standard_normal((B, n_q, Hkv, d)).astype(np.float32)).cuda().bfloat16()
        s["q"] = torch.from_numpy(rng.standard_normal((B, n_q, Hq, d)).astype(np.float32)).cuda().bfloat16()
        s["logits"] = torch.from_numpy((rng.standard_normal((B * n_q, V)) * 2).astype(np.float32)).cuda()
        s["u"] = torch.from_numpy(rng.random(B * n_q).astype(np.float32)).cuda()
        s["p"] = torch.full((B,), 0.9, device="cuda")
        s["ws"] = H.workspace(lib.specexit_quant_verify_attn_workspace_bytes(view, lib.BF16, B, n_q, Hq))
        s["ws2"] = H.workspace(lib.specexit_sample_workspace_bytes(lib.F32, B * n_q, V))
        sets.append(s)

    def outputs():
        return [(torch.empty((B, n_q, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty(B * n_q, dtype=torch.int32, device="cuda"),
                 torch.empty(B * n_q, device="cuda")) for _ in range(2)]

    def calls(s, o, stream):
        lib.specexit_quant_kv_write(s["view"], lib.BF16, B, n_q, s["k"], s["v"], s["L"], stream=stream)
        lib.specexit_quant_verify_attn(s["view"], lib.BF16, B, n_q, Hq, s["q"], s["L"], None, d ** -0.5, o[0], s["ws"], stream=stream)
        lib.specexit_sample(lib.F32, B * n_q, V, s["logits"], s["u"], o[1], o[2], top_p=s["p"], rows_per_seq=n_q, workspace=s["ws2"], stream=stream)

    alone = outputs()
    for s, o in zip(sets, alone):
        calls(s, o, torch.cuda.current_stream())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(10):
        both = outputs()
        torch.cuda.synchronize()
        for s, o, st in zip(sets, both, streams):
            calls(s, o, st)
        torch.cuda.synchronize()
        for a, b in zip(alone, both):
            for x, y in zip(a, b):
                assert torch.equal(x, y), rep
