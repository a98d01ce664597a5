"""GPU: rounds of a target around its attention - rows rotated and stored, attention over the plain or the latent cache, LM head, log probabilities,
acceptance, compaction - against the oracle, stage by stage on the library's own data, eager and replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O

import harness as H
from target_harness import DT, Latent, Rope, depths, dev, i32, latent_attn_bound, logprob_bound, stored, tree_masks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [None, 16])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("latent", [False, True])
def test_rounds(dtype, page, tree, latent):
    lib, rng = H.sx(), np.random.default_rng(31 + tree + 2 * latent)
    B, n_q, Hq, Hkv, d, r, D, V, rounds = 3, 6, 8, 2, 64, 128, 512, 4001, 3
    dt, code, w = DT[dtype], lib.dtype_code(DT[dtype]), 192
    L = np.array([40, 0, 77])
    ro = Rope(64, theta=1e4, interleaved=latent, scaling=3 if latent else 0, factor=8.0)
    desc, turns = ro.gpu()
    pool = Latent(rng, B, r, L + (rounds + 1) * n_q, dtype, page)
    if latent:
        caches = [dev(pool.c, dtype)]
        model = [pool.c.copy()]
        table = None if pool.table is None else i32(pool.table)
        view = lib.latent_kv_view(caches[0], 64, table)
    else:
        lead = pool.c.shape[:-1]
        model = [stored(rng.standard_normal((lead[0], Hkv, lead[1], d)), dtype) for _ in range(2)]
        caches = [dev(m, dtype) for m in model]
        table = None if pool.table is None else i32(pool.table)
        view = lib.kv_view(caches[0], caches[1], table)
    width = w if latent else d
    parent = None
    mask = None
    if tree:
        mask, parent = tree_masks(rng, B, n_q)
    off = depths(parent) if tree else np.tile(np.arange(n_q, dtype=np.int32), (B, 1))
    gp, gm, go = None if parent is None else i32(parent), None if mask is None else H.dev(mask), i32(off) if tree else None
    w_head = dev(stored(rng.standard_normal((V, D)) * 0.08, dtype), dtype)
    gain = stored(1 + 0.1 * rng.standard_normal(r), dtype)
    gg = dev(gain, dtype)
    zeros = lambda *s, t=dt: torch.zeros(s, dtype=t, device="cuda")
    rows = zeros(B, n_q, w) if latent else zeros(B, n_q, Hq + 2 * Hkv, d)
    q_pe = zeros(B, n_q, Hq, 64)
    q, out = zeros(B, n_q, Hq, width), zeros(B, n_q, Hq, r if latent else d)
    hid, nxt, logits = zeros(B, n_q, D), zeros(B, D), zeros(B * n_q, V, t=torch.float32)
    am, block, path = (zeros(B, n_q, t=torch.int32) for _ in range(3))
    lp, ent = zeros(B * n_q, 1, t=torch.float32), zeros(B * n_q, t=torch.float32)
    top, top_lp = zeros(B * n_q, 3, t=torch.int32), zeros(B * n_q, 3, t=torch.float32)
    ctx, new_ctx = i32(L), i32(L)
    sig = torch.full((B, 3), 0.5, device="cuda")
    ewma, n_obs, thinking = zeros(B, 3, t=torch.float32), i32([0] * B), i32([1] * B)
    length, recover, last, flag = (i32([0] * B) for _ in range(4))
    split, cfg, scale = i32([V - 1]), lib.exit_cfg(stop_think_token=5), 0.09
    ws_a = H.workspace(lib.specexit_latent_verify_attn_workspace_bytes(view, B, n_q, Hq) if latent else
                       lib.specexit_verify_attn_workspace_bytes(view, B, n_q, Hq))
    ws_h = H.workspace(lib.specexit_lmhead_argmax_workspace_bytes(code, B * n_q, D, V, 0))
    ws_p = H.workspace(lib.specexit_token_logprobs_workspace_bytes(lib.F32, B * n_q, V, 3))

    def one_round(stream):
        if latent:
            lib.specexit_latent_kv_write(view, desc, turns, B, n_q, Hq, rows, gg, 1e-6, q_pe, q, ctx, go, stream=stream)
            lib.specexit_latent_verify_attn(view, B, n_q, Hq, q, ctx, gm, scale, out, ws_a, stream=stream)
        else:
            lib.specexit_rope_kv_write(view, desc, turns, B, n_q, Hq, rows[:, :, :Hq], rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:], q, ctx, go,
                                       stream=stream)
            lib.specexit_verify_attn(view, B, n_q, Hq, q, ctx, gm, scale, out, ws_a, stream=stream)
        lib.specexit_lmhead_argmax(code, B * n_q, D, V, 0, hid, w_head, am, logits_dbg=logits, workspace=ws_h, stream=stream)
        lib.specexit_token_logprobs(lib.F32, B * n_q, V, logits, ent, block.view(-1, 1), lp, top, top_lp, workspace=ws_p, stream=stream)
        lib.specexit_accept_exit(cfg, B, n_q, block, gp, am, sig, ctx, split, 1, ewma, n_obs, thinking, None, length, path, recover, last, flag,
                                 new_ctx, stream=stream)
        compact = lib.specexit_latent_kv_compact if latent else lib.specexit_kv_compact
        compact(view, 1, 0, B, n_q, ctx, path, length, last, hid, D, nxt, stream=stream)

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for rnd in range(rounds + 1):
            x = stored(rng.standard_normal(tuple(rows.shape)), dtype)
            xq = stored(rng.standard_normal(tuple(q.shape)), dtype)            # the caller's part of a latent target's queries
            xp = stored(rng.standard_normal(tuple(q_pe.shape)), dtype)
            for a, v in ((rows, x), (q, xq), (q_pe, xp), (hid, stored(rng.standard_normal((B, n_q, D)), dtype))):
                a.copy_(dev(v, dtype))
            lib.specexit_lmhead_argmax(code, B * n_q, D, V, 0, hid, w_head, am, workspace=ws_h, stream=stream)
            best = am.cpu().numpy()
            blk = rng.integers(0, V, (B, n_q)).astype(np.int32)
            for b in range(B):
                for c in range(1, n_q):
                    if rng.random() < 0.7:
                        blk[b, c] = best[b, parent[b, c] if tree else c - 1]
            block.copy_(torch.from_numpy(blk))
            ctx.copy_(i32(L))
            torch.cuda.synchronize()
            if rnd == rounds:                      # the last round also from a graph: the same state, replayed three times, other work in between
                before, state = [c.clone() for c in caches], [a.clone() for a in (thinking, n_obs, ewma, q)]
                lib.specexit_graph_begin(stream)
                one_round(stream)
                graph = lib.specexit_graph_end(stream)
                names = dict(out=out, q=q, lp=lp, ent=ent, top=top, top_lp=top_lp, path=path, nxt=nxt, new_ctx=new_ctx, **{f"c{i}": c for i, c in enumerate(caches)})
                one_round(stream)
                torch.cuda.synchronize()
                eager = {n: a.clone() for n, a in names.items()}
                for rep in range(3):
                    for c, b0 in zip(caches, before):
                        c.copy_(b0)
                    for a in (out, lp, ent, top, top_lp, path, nxt, new_ctx):
                        a.zero_()
                    ws_a.fill_(255)
                    ws_p.fill_(255)
                    for a, s0 in zip((thinking, n_obs, ewma, q), state):
                        a.copy_(s0)
                    (w_head.float().sum() + rep).item()
                    lib.specexit_graph_launch(graph, stream)
                    torch.cuda.synchronize()
                    for n, a in names.items():
                        assert torch.equal(a, eager[n]), (rep, n)
                lib.specexit_graph_destroy(graph)
                break
            one_round(stream)
            torch.cuda.synchronize()
            pos = L[:, None] + off
            q_got = H.host(q)
            after = [H.host(c) for c in caches]
            got_path, got_len = path.cpu().numpy(), length.cpu().numpy()
            # ---- rows in the cache (read back before compaction would need another copy: moved rows are checked where they went), queries
            if latent:
                ref = np.stack([O.latent_rows(x[b], gain, 1e-6, pos[b], ro.f, True) for b in range(B)])
                tol = np.concatenate([(2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0)) * np.abs(ref[..., :r]),
                                      ro.bound(x[:, :, None, r:], ref[:, :, None, r:], dtype)[:, :, 0]], -1)
                want_q, tol_q = ro.heads(xp, pos), None
                tol_q = ro.bound(xp, want_q, dtype)
                assert (np.abs(q_got[..., r:] - want_q) <= tol_q).all() and np.array_equal(q_got[..., :r], xq[..., :r].astype(np.float32))
                at = lambda b, p: pool.at(b, p)
                parts = [(0, ref, tol)]
            else:
                turned = ro.heads(x, pos)
                tol_all = ro.bound(x, turned, dtype)
                assert (np.abs(q_got - turned[:, :, :Hq]) <= tol_all[:, :, :Hq]).all()
                at = lambda b, p: (pool.at(b, p)[0], slice(None), pool.at(b, p)[1])
                parts = [(0, turned[:, :, Hq:Hq + Hkv], tol_all[:, :, Hq:Hq + Hkv]), (1, x[:, :, Hq + Hkv:], np.zeros_like(x[:, :, Hq + Hkv:]))]
            for which, ref, tol in parts:
                for b in range(B):
                    moved = {int(L[b] + 1 + j): int(got_path[b, j]) for j in range(got_len[b])}
                    for i in range(n_q):
                        p = int(L[b]) + i
                        src = moved.get(p, i)
                        assert (np.abs(after[which][at(b, p)] - ref[b, src]) <= tol[b, src]).all(), (rnd, which, b, i)
            # ---- attention over the cache as it was, from the library's own rows
            full = [a.copy() for a in after]
            for f, m in zip(full, model):
                for b in range(B):
                    moved = {int(L[b] + 1 + j): int(got_path[b, j]) for j in range(got_len[b])}
                    own = {src: f[at(b, p)].copy() for p, src in moved.items()}
                    for i in range(n_q):
                        if int(L[b]) + i not in moved:
                            own.setdefault(i, f[at(b, int(L[b]) + i)].copy())
                    for i in range(n_q):
                        if i in own:
                            f[at(b, int(L[b]) + i)] = own[i]
                        else:                      # overwritten by a moved row: as it was written, rounded
                            which = [id(z) for z in full].index(id(f))
                            f[at(b, int(L[b]) + i)] = stored(parts[which][1][b, i], dtype)
            if latent:
                refo = O.latent_attn(q_got, full[0], r, L, mask, scale, pool.table, page or 16)
                weighed = O.latent_attn(q_got, full[0], r, L, mask, scale, pool.table, page or 16, absolute=True)
                tol = latent_attn_bound(refo, weighed, q_got, full[0], r, int(L.max()) + n_q, scale, dtype)
                if dtype == "bf16":
                    tol = tol + 2.0 ** -6         # (entries that a move overwrote are known to a rounding of the type)
                else:
                    tol = tol + 2.0 ** -18
                assert (np.abs(H.host(out) - refo) <= tol).all()
            else:
                refo = O.verify_attn(q_got, full[0], full[1], L, mask, scale, pool.table, page or 16)
                assert H.rel_err(H.host(out), refo) < H.TOL[dtype]
            # ---- log probabilities of the drafted tokens from the library's logits
            z = logits.cpu().numpy()
            for row in range(B * n_q):
                want = O.token_logprobs(z[row], [blk.reshape(-1)[row]], 3)
                y = z[row].astype(np.float64) - z[row].max()
                weight = float((np.exp(y - np.log(np.exp(y).sum())) * -y).sum())
                assert abs(float(lp[row, 0]) - want[0][0]) <= logprob_bound(y[blk.reshape(-1)[row]], want[0][0], weight)
                assert top[row].cpu().numpy().tolist() == want[2].tolist() and want[2][0] == best.reshape(-1)[row]
            acc = [O.greedy_accept(blk[b], parent[b] if tree else np.arange(-1, n_q - 1), best[b]) for b in range(B)]
            for b in range(B):
                want = list(acc[b][0]) if isinstance(acc[b], tuple) else list(acc[b])
                assert list(got_path[b, :got_len[b]]) == want
            L = new_ctx.cpu().numpy().astype(np.int64)


def test_rotated_keys_into_the_8_bit_cache():
    """specexit_rope on the keys of the fused rows, in place, then specexit_quant_kv_write from there: the codes of the rotated rows as stored."""
    lib, rng = H.sx(), np.random.default_rng(3)
    B, T, Hq, Hkv, d = 2, 5, 8, 2, 128
    ro = Rope(d)
    desc, turns = ro.gpu()
    x = dev(stored(rng.standard_normal((B, T, Hq + 2 * Hkv, d)), "bf16"), "bf16")
    pos = i32([3, 20])
    part = x[:, :, :Hq + Hkv]                      # queries and keys together
    lib.specexit_rope(lib.BF16, desc, turns, B, T, Hq + Hkv, d, part, part, pos)
    pools = [torch.zeros((B, Hkv, 48, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones((B, Hkv, 48), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lib.specexit_quant_kv_write(lib.quant_kv_view(*pools, *scales), lib.BF16, B, T, x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos)
    rows = H.host(x)
    for which in range(2):
        codes, s = O.quant_rows(rows[:, :, Hq + which * Hkv:Hq + (which + 1) * Hkv])
        for b, p in ((0, 3), (1, 20)):
            assert np.array_equal(pools[which][b, :, p:p + T].cpu().numpy(), codes[b].transpose(1, 0, 2))
            assert np.array_equal(scales[which][b, :, p:p + T].cpu().numpy(), s[b].T)


def test_two_streams_at_once():
    """Writes, attention and log probabilities of two inputs on two streams, each with a cache and workspaces of its own, against the same calls one by one."""
    lib, rng = H.sx(), np.random.default_rng(41)
    B, n_q, Hq, r, V = 3, 5, 16, 512, 20000
    ro = Rope(64)
    desc, turns = ro.gpu()
    sets = []
    for i in range(2):
        L = np.array([700 + 900 * i, 33, 2000 - 1000 * i])
        lat = Latent(rng, B, r, L + n_q, "bf16", 16)
        view, c, table = lat.gpu()
        s = dict(view=view, keep=(c, table), L=i32(L), rows=dev(rng.standard_normal((B, n_q, r + 64)), "bf16"), qp=dev(rng.standard_normal((B, n_q, Hq, 64)), "bf16"),
                 q=dev(rng.standard_normal((B, n_q, Hq, r + 64)), "bf16"), logits=dev(rng.standard_normal((B * n_q, V)) * 2, "f32"),
                 ws=H.workspace(lib.specexit_latent_verify_attn_workspace_bytes(view, B, n_q, Hq)),
                 ws2=H.workspace(lib.specexit_token_logprobs_workspace_bytes(lib.F32, B * n_q, V, 8)))
        sets.append(s)

    def outputs():
        return [(torch.empty((B, n_q, Hq, r), dtype=torch.bfloat16, device="cuda"), torch.empty(B * n_q, device="cuda"),
                 torch.empty((B * n_q, 8), dtype=torch.int32, device="cuda")) for _ in range(2)]

    def calls(s, o, stream):
        lib.specexit_latent_kv_write(s["view"], desc, turns, B, n_q, Hq, s["rows"], None, 0.0, s["qp"], s["q"], s["L"], stream=stream)
        lib.specexit_latent_verify_attn(s["view"], B, n_q, Hq, s["q"], s["L"], None, 0.07, o[0], s["ws"], stream=stream)
        lib.specexit_token_logprobs(lib.F32, B * n_q, V, s["logits"], o[1], top_token=o[2], workspace=s["ws2"], stream=stream)

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
