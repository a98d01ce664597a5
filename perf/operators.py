"""What is timed of the operators around an 8-bit KV cache and sampled tokens, and their plain forms.

A decode round served that way writes its block's K/V rows in 8 bits, attends to the 8-bit cache, draws the target's
token of every block row, and moves the accepted path's rows next to the context:
  write    specexit_quant_kv_write     rows -> e4m3 codes and one power-of-two scale per (token, KV head)
  attn     specexit_quant_verify_attn  attention of a block against such a cache
  compact  specexit_quant_kv_compact   the accepted path's codes and scales, all layers
  sample   specexit_sample             temperature, top-k, top-p and min-p from given uniform numbers

A case is a dict of plain values, `kind` one of the four.  `run` computes it with elementary tensor operations, or, where
`own` is true, through the library's entry points.  Shapes are those of workloads/gen.py or generic ones near them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FLOOR = 2.0 ** -40          # weights below this fraction of the best token's count as none


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the block rows of one layer, as a round writes them: eight sequences of seven tokens, out of a fused q|k|v projection
        {"name": "write_block_8b", "kind": "write", "dtype": "bf16", "B": 8, "T": 7, "Hkv": 8, "d": 128, "Hq": 32, "lo": 300, "hi": 1500,
         "paged": True, "page": 16, "ragged": False, "fused": True},
        # four ragged prompts of a layer into a contiguous cache
        {"name": "write_prompts_8b", "kind": "write", "dtype": "bf16", "B": 4, "T": 4111, "Hkv": 8, "d": 128, "Hq": 32, "lo": 0, "hi": 0,
         "paged": False, "page": 16, "ragged": True, "fused": False},
        # the tiny fp32 round's block against a short cache: launch latency and nothing else
        {"name": "attn_tiny_f32", "kind": "attn", "dtype": "f32", "B": 1, "n_q": 5, "Hq": 8, "Hkv": 2, "d": 64, "lo": 256, "hi": 256,
         "paged": False, "page": 16, "tree": False},
        # a layer of one user's 4B-like target: a short call
        {"name": "attn_4b_chain", "kind": "attn", "dtype": "bf16", "B": 1, "n_q": 7, "Hq": 32, "Hkv": 8, "d": 128, "lo": 4096, "hi": 4096,
         "paged": False, "page": 16, "tree": False},
        # tree verification, 64-wide heads, larger pages
        {"name": "attn_d64_tree", "kind": "attn", "dtype": "bf16", "B": 8, "n_q": 16, "Hq": 32, "Hkv": 8, "d": 64, "lo": 1000, "hi": 8000,
         "paged": True, "page": 32, "tree": True},
        # an ordinary batch of the 8B-like target
        {"name": "attn_8b_batch8", "kind": "attn", "dtype": "bf16", "B": 8, "n_q": 7, "Hq": 32, "Hkv": 8, "d": 128, "lo": 2048, "hi": 16384,
         "paged": True, "page": 16, "tree": False},
        # the largest: long contexts of a 32B-like target, 72 query rows to a KV head
        {"name": "attn_32b_long", "kind": "attn", "dtype": "bf16", "B": 16, "n_q": 9, "Hq": 64, "Hkv": 8, "d": 128, "lo": 8192, "hi": 32768,
         "paged": True, "page": 16, "tree": False},
        # what closes a round of four sequences with a 16-node tree, 36 layers; and a larger batch of 64 layers, paged
        {"name": "compact_tree_36_layers", "kind": "compact", "dtype": "bf16", "B": 4, "n_q": 16, "Hkv": 8, "d": 128, "D": 4096, "layers": 36,
         "lo": 40, "hi": 75, "paged": False, "page": 16},
        {"name": "compact_batch_64_layers", "kind": "compact", "dtype": "bf16", "B": 16, "n_q": 9, "Hkv": 8, "d": 128, "D": 5120, "layers": 64,
         "lo": 20, "hi": 50, "paged": True, "page": 16},
        # one user's block, with the settings reasoning models are usually served with
        {"name": "sample_user_top_k", "kind": "sample", "dtype": "f32", "M": 7, "per": 7, "V": 151936, "ld": 151936, "mode": "k+p"},
        # the largest block, nucleus only: the whole vocabulary counts
        {"name": "sample_batch_top_p", "kind": "sample", "dtype": "f32", "M": 144, "per": 9, "V": 151936, "ld": 151936, "mode": "p"},
        # bf16 logits of an odd vocabulary behind a widened head, every sequence with settings of its own
        {"name": "sample_bf16_mixed", "kind": "sample", "dtype": "bf16", "M": 48, "per": 4, "V": 128259, "ld": 128262, "mode": "mixed"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choices(["attn", "sample", "write", "compact"], [7, 5, 3, 2])[0]
    c = {"kind": kind, "dtype": "f32" if rng.random() < 0.15 else "bf16"}
    if kind == "sample":
        c["dtype"] = rng.choice(["f32", "f32", "bf16"])
        per = rng.randint(1, 16)
        c.update(per=per, M=per * rng.randint(1, _log_int(rng, 1, 144 // per)), V=rng.choice([151936, _log_int(rng, 2000, 151936)]),
                 mode=rng.choice(["k", "p", "k+p", "m", "none", "mixed"]))
        c["ld"] = c["V"] + rng.choice([0, 0, 3])
        return c
    c.update(Hkv=rng.choice([2, 4, 8, 8]), d=rng.choice([64, 128, 128]))
    G = rng.choice([1, 4, 4, 5, 8])
    c["Hq"] = G * c["Hkv"]
    c["paged"] = rng.random() < 0.6
    c["page"] = rng.choice([16, 16, 32, 48, 64]) if c["paged"] else 16
    if kind == "compact":
        lo = rng.randint(0, 60)
        c.update(B=_log_int(rng, 1, 16), n_q=rng.randint(3, 17), layers=rng.randint(4, 64), D=64 * rng.randint(8, 80), lo=lo, hi=lo + rng.randint(0, 40))
    elif kind == "write":
        B = _log_int(rng, 1, 64)
        c.update(B=B, T=_log_int(rng, 1, 16384 // B), ragged=rng.random() < 0.5, fused=rng.random() < 0.5)
        lo = rng.choice([0, _log_int(rng, 1, 3000 // B + 1)])
        c.update(lo=lo, hi=lo + rng.randint(0, 40))
    else:
        B = _log_int(rng, 1, 64)
        top = (250 << 20) // (B * c["Hkv"] * (c["d"] + 1) * (8 if c["dtype"] == "f32" else 1))
        mid = _log_int(rng, 20, max(40, min(3000 if c["dtype"] == "f32" else 20000, top)))
        c.update(B=B, n_q=rng.randint(1, min(17, 128 // G)), tree=rng.random() < 0.4, lo=max(0, int(mid * 0.5)), hi=int(mid * 1.5))
    return c


def _lengths(c):
    """The lengths of a case's sequences; every seed deals out the same ones."""
    return [(c["lo"] + c["hi"]) // 2] if c["B"] == 1 else [c["lo"] + (c["hi"] - c["lo"]) * b // (c["B"] - 1) for b in range(c["B"])]


def _counts(c):
    return [max(1, c["T"] * (b + 3) // (c["B"] + 2)) if c["ragged"] else c["T"] for b in range(c["B"])]


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "write":
        rows = sum(_counts(c)) * c["Hkv"] * 2
        return {"bytes": rows * (e * c["d"] + c["d"] + 1), "flops": rows * 2 * c["d"]}
    if c["kind"] == "attn":
        keys = sum(_lengths(c)) + c["B"] * c["n_q"]
        return {"bytes": keys * c["Hkv"] * 2 * (c["d"] + 1) + 2 * c["B"] * c["n_q"] * c["Hq"] * c["d"] * e,
                "flops": 4 * keys * c["n_q"] * c["Hq"] * c["d"]}
    if c["kind"] == "compact":
        moved = c["layers"] * c["B"] * c["Hkv"] * 2 * max(1, c["n_q"] // 4)
        return {"bytes": 2 * moved * (c["d"] + 1) + 2 * c["B"] * c["D"] * e, "flops": moved}
    return {"bytes": c["M"] * (c["V"] * e + 8), "flops": 2 * c["M"] * c["V"]}


# ------------------------------------------------------------------------------------ inputs

def _generator(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + sum(ord(x) * 31 for x in c["kind"]) + c.get("V", 0) + 17 * c.get("B", 0) + c.get("hi", 0))
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(g, shape, dtype):
    """K or V rows: normal values, a magnitude of its own for every row, and a few large channels, as keys have them."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.7 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    x[..., :3] *= 4.0
    return x.to(dtype)


def _shuffled(values, rng):
    values = list(values)
    rng.shuffle(values)
    return values


def _table(c, need, rng):
    """Pages of sequences with `need` entries each, in random order; (table [B, max_pages], pages of the pool)."""
    n = [(x + c["page"] - 1) // c["page"] for x in need]
    total = sum(n) + max(2, sum(n) // 10)
    ids = _shuffled(range(total), rng)
    table = np.zeros((len(n), max(max(n), 1)), np.int32)
    at = 0
    for b, k in enumerate(n):
        table[b, :k] = ids[at:at + k]
        at += k
    return torch.from_numpy(table).cuda(), total


def _places(c, s, b, p):
    """Entries p (a tensor) of sequence b: indices of the pools' dimensions in front of and behind the head's."""
    if c["paged"]:
        return s["table"][b, p // c["page"]].long(), p % c["page"]
    return torch.full_like(p, b), p


def _pools(c, s, need, rng, layers=()):
    if c["paged"]:
        s["table"], n = _table(c, need, rng)
        shape = (*layers, n, c["Hkv"], c["page"])
    else:
        s["table"] = None
        shape = (*layers, c["B"], c["Hkv"], (max(need) + 15) // 16 * 16)
    for t in ("k", "v"):
        s[t] = torch.zeros(shape + (c["d"],), dtype=torch.uint8, device="cuda")
        s[t + "s"] = torch.ones(shape, dtype=torch.uint8, device="cuda")


def _view(s, layer=None):
    from paper_2509_24248_amd import binding as sx
    at = (lambda t: t) if layer is None else (lambda t: t[layer])
    return sx.quant_kv_view(at(s["k"]), at(s["v"]), at(s["ks"]), at(s["vs"]), s["table"])


def _bytes(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def _tree(n, rng):
    parent = [-1]
    for c in range(1, n):
        parent.append(rng.randint(max(0, (c - 4) // 2), c - 1))
    return parent


def _masks(c, rng):
    out = []
    for _ in range(c["B"]):
        words = []
        for i, p in enumerate(_tree(c["n_q"], rng)):
            words.append((words[p] if p >= 0 else 0) | (1 << i))
        out.append(words)
    return torch.tensor(out, dtype=torch.int64, device="cuda")


def prepare(c, seed):
    g, rng = _generator(c, seed), random.Random(977 * seed + 5)
    s = {"case": c}
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "write":
        counts, pos = _shuffled(_counts(c), rng), _shuffled(_lengths(c), rng)
        _pools(c, s, [p + n for p, n in zip(pos, counts)], rng)
        B, T, Hkv, d = c["B"], c["T"], c["Hkv"], c["d"]
        if c["fused"]:
            x = _rows(g, (B, T, c["Hq"] + 2 * Hkv, d), dt)
            s["k_rows"], s["v_rows"] = x[:, :, c["Hq"]:c["Hq"] + Hkv], x[:, :, c["Hq"] + Hkv:]
        else:
            s["k_rows"], s["v_rows"] = _rows(g, (B, T, Hkv, d), dt), _rows(g, (B, T, Hkv, d), dt)
        s["pos"], s["count"], s["host"] = _i32(pos), (_i32(counts) if c["ragged"] else None), (pos, counts)
    elif c["kind"] == "attn":
        L = _shuffled(_lengths(c), rng)
        _pools(c, s, [x + c["n_q"] for x in L], rng)
        for b in range(c["B"]):
            p = torch.arange(L[b] + c["n_q"], device="cuda")
            i, j = _places(c, s, b, p)
            for t in ("k", "v"):
                codes, scale = _quantise(_rows(g, (p.numel(), c["Hkv"], c["d"]), torch.bfloat16).float())
                s[t][i, :, j], s[t + "s"][i, :, j] = codes, scale
        s["q"] = torch.randn((c["B"], c["n_q"], c["Hq"], c["d"]), generator=g, device="cuda").to(dt)
        s["L"], s["ctx"] = L, _i32(L)
        s["mask"] = _masks(c, rng) if c["tree"] else None
        s["scale"] = c["d"] ** -0.5
        s["out"] = torch.empty_like(s["q"])
    elif c["kind"] == "compact":
        L = _shuffled(_lengths(c), rng)
        _pools(c, s, [x + c["n_q"] for x in L], rng, (c["layers"],))
        for t in ("k", "v"):
            s[t].random_(0, 127, generator=g)
            s[t + "s"].random_(110, 130, generator=g)
        n, path, length, last = c["n_q"], [], [], []
        for _ in range(c["B"]):
            # some depths in place, then nodes whose entries nothing is moved to, so that a second pass finds the same
            m = max(1, n // 4)
            first = rng.randint(0, m - 1)
            nodes = list(range(1, first + 1)) + sorted(rng.sample(range(m + 1, n), m - first))
            path.append(nodes + [-1] * (n - m))
            length.append(m)
            last.append(nodes[-1])
        s["L"], s["ctx"], s["host"] = L, _i32(L), (path, length, last)
        s["path"], s["len"], s["last"] = _i32(path), _i32(length), _i32(last)
        s["hidden"] = torch.randn((c["B"], n, c["D"]), generator=g, device="cuda").to(dt)
        s["next"] = torch.zeros((c["B"], c["D"]), dtype=dt, device="cuda")
    else:
        M, V, n = c["M"], c["V"], (c["M"] + c["per"] - 1) // c["per"]
        x = torch.randn((M, c["ld"]), generator=g, device="cuda") * 2.2
        # a head's logits: a few dozen candidates stand out, more in some rows than in others
        for r in range(M):
            k = 4 + 7 * (r % 9)
            at = torch.randint(0, V, (k,), generator=g, device="cuda")
            x[r, at] += torch.linspace(14.0, 4.0, k, device="cuda") * (0.6 + 0.1 * (r % 5))
            if r % 4 == 3:
                x[r, V // 3:V // 3 + V // 9] = -math.inf         # tokens that a grammar rules out
        s["logits"] = x.to(dt)
        mode = c["mode"]
        pick = lambda letter, on, off: [on() if letter in mode or (mode == "mixed" and rng.random() < 0.5) else off for _ in range(n)]
        f32 = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")
        s["temperature"] = f32([0.0 if mode == "mixed" and rng.random() < 0.2 else rng.uniform(0.5, 1.1) for _ in range(n)])
        s["top_k"] = _i32(pick("k", lambda: rng.choice([20, 50, 400]), 0)) if mode in ("k", "k+p", "mixed") else None
        s["top_p"] = f32(pick("p", lambda: rng.uniform(0.8, 0.98), 1.0)) if mode in ("p", "k+p", "mixed") else None
        s["min_p"] = f32(pick("m", lambda: rng.uniform(0.01, 0.1), 0.0)) if mode in ("m", "mixed") else None
        s["u"] = torch.rand(M, generator=g, device="cuda")
        s["token"] = torch.empty(M, dtype=torch.int32, device="cuda")
        s["prob"] = torch.empty(M, dtype=torch.float32, device="cuda")
    if own:
        from paper_2509_24248_amd import binding as sx
        s["code"] = sx.dtype_code(dt)
        if c["kind"] == "sample":
            s["ws"] = _bytes(sx.specexit_sample_workspace_bytes(s["code"], c["M"], c["V"]))
        else:
            s["view"] = _view(s, 0 if c["kind"] == "compact" else None)
        if c["kind"] == "attn":
            s["ws"] = _bytes(sx.specexit_quant_verify_attn_workspace_bytes(s["view"], s["code"], c["B"], c["n_q"], c["Hq"]))
    return s


# ------------------------------------------------------------------------------------ one pass

def run(s):
    return {"write": _run_write, "attn": _run_attn, "compact": _run_compact, "sample": _run_sample}[s["case"]["kind"]](s)


def _cache(s):
    return [s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["ks"], s["vs"]]


def _power(n):
    """2^n for whole n of -126 .. 127, exactly, in fp32 (a power function need not be exact)."""
    return ((n.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """fp32 rows [.., d] -> e4m3 codes as bytes, scale bytes: the least power of two that brings the row within 448."""
    ok = torch.isfinite(x)
    m, e = torch.frexp(torch.where(ok, x.abs(), 0.0).amax(-1))
    s = torch.where(m > 0, e + 118 + (m > 0.875), 1).clamp(1, 254).to(torch.int32)
    codes = (x * _power(127 - s).unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(ok, codes, 0x7F + 0x80 * torch.signbit(x).to(torch.uint8)), s.to(torch.uint8)


def _run_write(s):
    c = s["case"]
    if own:
        from paper_2509_24248_amd import binding as sx
        sx.specexit_quant_kv_write(s["view"], s["code"], c["B"], c["T"], s["k_rows"], s["v_rows"], s["pos"], s["count"])
        return _cache(s)
    pos, counts = s["host"]
    for t in ("k", "v"):
        codes, scale = _quantise(s[t + "_rows"].float())
        for b in range(c["B"]):
            i, j = _places(c, s, b, torch.arange(pos[b], pos[b] + counts[b], device="cuda"))
            s[t][i, :, j], s[t + "s"][i, :, j] = codes[b, :counts[b]], scale[b, :counts[b]]
    return _cache(s)


def _values(s, t, b, n, dtype):
    """The first n rows of sequence b's K or V as [Hkv, n, d] numbers."""
    i, j = _places(s["case"], s, b, torch.arange(n, device="cuda"))
    x = s[t].view(torch.float8_e4m3fn)[i, :, j].to(dtype)
    scale = _power(s[t + "s"][i, :, j].to(torch.int32) - 127).to(dtype)
    return (x * scale.unsqueeze(-1)).transpose(0, 1).contiguous()


def _run_attn(s):
    c = s["case"]
    if own:
        from paper_2509_24248_amd import binding as sx
        sx.specexit_quant_verify_attn(s["view"], s["code"], c["B"], c["n_q"], c["Hq"], s["q"], s["ctx"], s["mask"], s["scale"], s["out"], s["ws"])
        return s["out"]
    n_q, G = c["n_q"], c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        L = s["L"][b]
        n = L + n_q
        k, v = _values(s, "k", b, n, torch.float32), _values(s, "v", b, n, torch.float32)
        q = s["q"][b].float().reshape(n_q, c["Hkv"], G, c["d"]).permute(1, 0, 2, 3).reshape(c["Hkv"], n_q * G, c["d"])
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"]
        bits = torch.arange(n_q, device="cuda")
        seen = (s["mask"][b].unsqueeze(1) >> bits) & 1 == 1 if s["mask"] is not None else bits.unsqueeze(0) <= bits.unsqueeze(1)
        x[:, :, L:].masked_fill_(~seen.repeat_interleave(G, 0), -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        s["out"][b] = o.reshape(c["Hkv"], n_q, G, c["d"]).permute(1, 0, 2, 3).reshape(n_q, c["Hq"], c["d"]).to(s["out"].dtype)
    return s["out"]


def _run_compact(s):
    c = s["case"]
    if own:
        from paper_2509_24248_amd import binding as sx
        layer = s["k"][0].numel()
        sx.specexit_quant_kv_compact(s["view"], c["layers"], layer, layer // c["d"], c["B"], c["n_q"], s["ctx"], s["path"], s["len"],
                                     s["code"], s["last"], s["hidden"], c["D"], s["next"])
        return _cache(s) + [s["next"]]
    path, length, last = s["host"]
    for b in range(c["B"]):
        m, L = length[b], s["L"][b]
        i, j = _places(c, s, b, L + torch.tensor(path[b][:m], device="cuda"))
        to_i, to_j = _places(c, s, b, L + 1 + torch.arange(m, device="cuda"))
        for t in ("k", "v", "ks", "vs"):
            rows = s[t][:, i, :, j]
            s[t][:, to_i, :, to_j] = rows.clone()
        s["next"][b] = s["hidden"][b, last[b]]
    return _cache(s) + [s["next"]]


def _run_sample(s):
    c = s["case"]
    if own:
        from paper_2509_24248_amd import binding as sx
        sx.specexit_sample(s["code"], c["M"], c["V"], s["logits"], s["u"], s["token"], s["prob"], s["temperature"], s["top_k"], s["top_p"],
                           s["min_p"], rows_per_seq=c["per"], workspace=s["ws"])
        return [s["token"], s["prob"]]
    M, V = c["M"], c["V"]
    row = lambda t, off: (torch.full((M, 1), off, dtype=torch.float64, device="cuda") if t is None
                          else t.double().repeat_interleave(c["per"])[:M].unsqueeze(1))
    T, k, p, m = row(s["temperature"], 1.0), row(s["top_k"], 0.0), row(s["top_p"], 1.0), row(s["min_p"], 0.0)
    l = s["logits"][:, :V].float()
    greedy = T == 0
    k = torch.where(greedy, 1.0, k)
    # 64 bits: a draw may lie next to the border of two tokens, and a token next to a filter's
    w = torch.exp((l.double() - l.double().amax(1, keepdim=True)) / torch.where(greedy, 1.0, T))
    w = torch.where(w >= FLOOR, w, 0.0)
    _, order = torch.sort(l, dim=1, descending=True, stable=True)
    ranked = torch.gather(w, 1, order)
    ranked = torch.where((k <= 0) | (torch.arange(V, device="cuda").unsqueeze(0) < k), ranked, 0.0)
    better = torch.cumsum(ranked, 1) - ranked
    ranked = torch.where((p >= 1) | (better < p * ranked.sum(1, keepdim=True)), ranked, 0.0)
    ranked = torch.where(ranked >= m, ranked, 0.0)
    kept = torch.zeros_like(w).scatter_(1, order, ranked)
    upto = torch.cumsum(kept, 1)
    total = upto[:, -1:]
    token = (upto > s["u"].double().unsqueeze(1) * total).to(torch.uint8).argmax(1)
    s["token"].copy_(token)
    s["prob"].copy_((torch.gather(kept, 1, token.unsqueeze(1)) / total).squeeze(1))
    return [s["token"], s["prob"]]


# ------------------------------------------------------------------------------------ in 64 bits, from the definitions

def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "compact":
        return _exact_compact(c, s)
    if c["kind"] == "write":
        return _exact_write(c, s)
    return _exact_attn(c, s) if c["kind"] == "attn" else _exact_sample(c, s)


def _powers():
    """2^(n - 300) at n, exactly, in 64 bits."""
    return torch.tensor([math.ldexp(1.0, n - 300) for n in range(600)], dtype=torch.float64, device="cuda")


def _exact_write(c, s):
    two = _powers()
    power = lambda n: two[n.long() + 300]
    pos, counts = s["host"]
    out = []
    for t in ("k", "v"):
        value, byte = torch.zeros(s[t].shape, dtype=torch.float64, device="cuda"), s[t + "s"].clone()
        for b in range(c["B"]):
            x = s[t + "_rows"][b, :counts[b]].double()
            amax = x.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / 448.0))
            e = torch.where(amax * power(-e) > 448.0, e + 1, torch.where(amax * power(1 - e) <= 448.0, e - 1, e))
            e = torch.where(amax > 0, e.clamp(min=-126.0), -126.0)
            y = x * power(-e)
            step = power(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(min=-6.0) - 3)
            at = torch.arange(counts[b], device="cuda") + pos[b]
            i = s["table"][b].long()[at // c["page"]] if c["paged"] else torch.full_like(at, b)
            j = at % c["page"] if c["paged"] else at
            value[i, :, j], byte[i, :, j] = torch.round(y / step) * step, (e + 127).squeeze(-1).to(torch.uint8)
        out += [value, byte]
    return [out[0], out[2], out[1], out[3]]


def _exact_compact(c, s):
    path, length, last = s["host"]
    pools = {t: s[t].cpu().numpy() for t in ("k", "v", "ks", "vs")}
    table = s["table"].cpu().numpy() if c["paged"] else None
    where = lambda b, p: (table[b, p // c["page"]], p % c["page"]) if c["paged"] else (b, p)
    hidden = s["hidden"].double().cpu()
    for pool in pools.values():
        for b in range(c["B"]):
            old = [pool[:, where(b, s["L"][b] + n)[0], :, where(b, s["L"][b] + n)[1]].copy() for n in path[b][:length[b]]]
            for n, row in enumerate(old):
                x, y = where(b, s["L"][b] + 1 + n)
                pool[:, x, :, y] = row
    value = lambda t: torch.from_numpy(pools[t]).view(torch.float8_e4m3fn).double()
    return [value("k"), value("v"), torch.from_numpy(pools["ks"]), torch.from_numpy(pools["vs"]),
            torch.stack([hidden[b, last[b]] for b in range(c["B"])])]


def _exact_attn(c, s):
    two = _powers()
    G, out = c["Hq"] // c["Hkv"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n = s["L"][b] + c["n_q"]
        at = torch.arange(n, device="cuda")
        for h in range(c["Hkv"]):
            if c["paged"]:
                pick = lambda pool: pool[s["table"][b].long()[at // c["page"]], h, at % c["page"]]
            else:
                pick = lambda pool: pool[b, h, :n]
            k, v = (pick(s[t]).view(torch.float8_e4m3fn).double() * two[pick(s[t + "s"]).long() + 173].unsqueeze(1) for t in ("k", "v"))
            for i in range(c["n_q"]):
                word = int(s["mask"][b, i]) if s["mask"] is not None else (2 << i) - 1
                q = s["q"][b, i, h * G:(h + 1) * G].double()
                x = q @ k.t() * s["scale"]
                hidden = [s["L"][b] + j for j in range(c["n_q"]) if not word >> j & 1]
                x[:, hidden] = -math.inf
                out[b, i, h * G:(h + 1) * G] = torch.softmax(x, 1) @ v
    return out


def _exact_sample(c, s):
    l = s["logits"][:, :c["V"]].float().cpu().numpy().astype(np.float64)
    number = lambda t, r, off: off if t is None else float(t[r // c["per"]])
    tokens, probs = np.zeros(c["M"], np.int32), np.zeros(c["M"])
    for r in range(c["M"]):
        T, k, p, m = number(s["temperature"], r, 1.0), number(s["top_k"], r, 0), number(s["top_p"], r, 1.0), number(s["min_p"], r, 0.0)
        x = l[r]
        if T == 0.0:
            tokens[r], probs[r] = int(np.argmax(x)), 1.0
            continue
        w = np.exp((x - x.max()) / T)
        alive = np.flatnonzero(w >= FLOOR)
        best_first = alive[np.argsort(-x[alive], kind="stable")]
        if k > 0:
            best_first = best_first[:int(k)]
        mass = w[best_first]
        if p < 1.0:
            before = np.concatenate([[0.0], np.cumsum(mass)[:-1]])
            best_first = best_first[before < p * mass.sum()]
        chosen = np.sort(best_first[w[best_first] >= m])
        upto = np.cumsum(w[chosen])
        j = int(np.searchsorted(upto, float(s["u"][r]) * upto[-1], side="right"))
        tokens[r], probs[r] = chosen[j], w[chosen[j]] / upto[-1]
    return [torch.from_numpy(tokens), torch.from_numpy(probs)]
