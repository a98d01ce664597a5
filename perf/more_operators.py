"""What is timed of the operators around a target's verification pass, and their plain forms.

  rope     specexit_rope, specexit_rope_kv_write   a block's (or prompt's) heads rotated by position; keys and values appended to the cache
  lwrite   specexit_latent_kv_write                a latent cache's entries: the latent's norm, the rotated key part; the queries' rotated part
  lattn    specexit_latent_verify_attn             attention of a block against a cache of one latent vector a token
  logprob  specexit_token_logprobs                 log probabilities of given tokens, entropy and the best alternatives

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
EPS = 1e-6
NONE, LINEAR, BANDS, RAMP = 0, 1, 2, 3          # how rotary frequencies are scaled


# ------------------------------------------------------------------------------------ the cases

def listed():
    rope = dict(kind="rope", append=True, interleaved=False, rot=128, scaling=NONE, theta=1e6, d=128, page=16, ragged=False, tree=False, fused=True)
    lat = dict(r=512, dr=64, page=64, tree=False)
    return [
        # the block rows of one layer, as a round rotates and stores them: eight sequences of seven tokens out of a fused q|k|v projection
        {"name": "rope_block_8b", **rope, "dtype": "bf16", "B": 8, "T": 7, "Hq": 32, "Hkv": 8, "paged": True, "lo": 300, "hi": 33000},
        # four ragged prompts of a layer into a contiguous cache, frequencies scaled by bands for a longer context
        {"name": "rope_prompts_8b", **rope, "dtype": "bf16", "B": 4, "T": 4111, "Hq": 32, "Hkv": 8, "paged": False, "lo": 0, "hi": 0,
         "ragged": True, "scaling": BANDS, "fused": False},
        # a tree's heads rotated by depth, nothing stored: fp32, neighbouring pairs, half of each head, far positions
        {"name": "rope_tree_f32", **rope, "append": False, "dtype": "f32", "B": 16, "T": 16, "Hq": 72, "Hkv": 0, "paged": False, "lo": 1000,
         "hi": 1000000, "interleaved": True, "rot": 64, "scaling": RAMP, "tree": True},
        # a block's latent entries and its queries' rotated part
        {"name": "lwrite_block", **lat, "kind": "lwrite", "dtype": "bf16", "B": 8, "T": 7, "H": 16, "paged": True, "lo": 300, "hi": 33000,
         "ragged": False},
        # four ragged prompts' entries, no queries
        {"name": "lwrite_prompts", **lat, "kind": "lwrite", "dtype": "bf16", "B": 4, "T": 4111, "H": 0, "paged": False, "lo": 0, "hi": 0,
         "ragged": True},
        # the tiny fp32 round: launch latency and nothing else
        {"name": "lattn_tiny_f32", **lat, "kind": "lattn", "dtype": "f32", "r": 128, "B": 1, "n_q": 5, "H": 8, "lo": 256, "hi": 256, "paged": False},
        # one user's block over a short context, a sixteenth of the heads of a large target or all of a small one
        {"name": "lattn_user_chain", **lat, "kind": "lattn", "dtype": "bf16", "B": 1, "n_q": 7, "H": 16, "lo": 4096, "hi": 4096, "paged": False},
        # plain decoding of a batch over long contexts: one token each, every head of a large target
        {"name": "lattn_single_long", **lat, "kind": "lattn", "dtype": "bf16", "B": 16, "n_q": 1, "H": 128, "lo": 8192, "hi": 32768, "paged": True},
        # tree verification: 16 nodes of 64 heads, 1024 query rows to an entry
        {"name": "lattn_tree_batch", **lat, "kind": "lattn", "dtype": "bf16", "B": 8, "n_q": 16, "H": 64, "lo": 2048, "hi": 16384, "paged": True,
         "tree": True},
        # one user's block: what the target thinks of the drafted token, five alternatives each
        {"name": "logprob_user", "kind": "logprob", "dtype": "f32", "M": 7, "per": 7, "V": 151936, "ld": 151936, "n_tok": 1, "n_top": 5, "heat": False},
        # the largest block, twenty alternatives
        {"name": "logprob_batch", "kind": "logprob", "dtype": "f32", "M": 144, "per": 9, "V": 151936, "ld": 151936, "n_tok": 1, "n_top": 20,
         "heat": False},
        # bf16 logits of an odd vocabulary behind a widened head, a temperature per sequence, three tokens a row, the best one beside them
        {"name": "logprob_bf16_odd", "kind": "logprob", "dtype": "bf16", "M": 48, "per": 4, "V": 128259, "ld": 128262, "n_tok": 3, "n_top": 1,
         "heat": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choices(["lattn", "rope", "logprob", "lwrite"], [6, 4, 4, 3])[0]
    c = {"kind": kind, "dtype": "f32" if rng.random() < 0.2 else "bf16"}
    if kind == "logprob":
        c["dtype"] = rng.choice(["f32", "bf16"])
        per = rng.randint(1, 16)
        c.update(per=per, M=per * rng.randint(1, _log_int(rng, 1, 144 // per)), V=rng.choice([151936, _log_int(rng, 500, 151936)]),
                 n_tok=rng.choice([0, 1, 1, 2, 5]), n_top=rng.choice([0, 1, 5, 20, 32]), heat=rng.random() < 0.4)
        c["ld"] = c["V"] + rng.choice([0, 0, 3])
        return c
    c["paged"] = rng.random() < 0.6 and kind != "rope"
    c["page"] = rng.choice([16, 16, 32, 48, 64]) if c["paged"] else 16
    if kind == "lattn":
        c.update(r=rng.choice([128, 256, 512, 512]), dr=64, H=rng.choice([1, 5, 8, 16, 16, 20, 32, 64, 128]), B=_log_int(rng, 1, 48))
        c["n_q"] = rng.choice([1, 1, rng.randint(2, 17), _log_int(rng, 1, 48)])
        rows, e = c["H"] * c["n_q"], 4 if c["dtype"] == "f32" else 2
        c["B"] = max(1, min(c["B"], 100_000_000 // (rows * (2 * c["r"] + 64) * e)))
        keys = min(250_000, int(6e7 / rows)) // (16 if c["dtype"] == "f32" else 1)
        mid = max(2, min(24000, keys // c["B"]))
        mid = _log_int(rng, min(20, mid), mid)
        c.update(tree=rng.random() < 0.4, lo=rng.choice([0, mid // 2, mid // 2]), hi=mid)
        return c
    B = _log_int(rng, 1, 64)
    c.update(B=B, T=_log_int(rng, 1, 16000 // B), ragged=rng.random() < 0.4)
    if kind == "lwrite":
        c.update(r=rng.choice([128, 256, 512, 512]), dr=64, H=rng.choice([0, 8, 16, 64, 128]) if B * c["T"] <= 1000 else 0, tree=c["T"] <= 48 and rng.random() < 0.4)
    else:
        d = rng.choice([64, 128, 128])
        Hkv = rng.choice([0, 2, 4, 8, 8])
        c.update(d=d, Hkv=Hkv, append=Hkv > 0, Hq=rng.choice([1, 4, 5]) * (Hkv or 8), rot=rng.choice([d, d, d // 2, d // 4, 26]),
                 interleaved=rng.random() < 0.5, scaling=rng.randint(0, 3), theta=rng.choice([1e4, 5e5, 1e6]), fused=rng.random() < 0.5,
                 tree=c["T"] <= 48 and rng.random() < 0.4, paged=Hkv > 0 and rng.random() < 0.6)
        c["page"] = rng.choice([16, 16, 32, 48, 64]) if c["paged"] else 16
        c["T"] = min(c["T"], max(1, 90_000_000 // (B * (c["Hq"] + 2 * Hkv) * d * (2 if c["dtype"] == "f32" else 1))))
    far = 500_000 if c["paged"] or not c.get("append", True) else max(1, 3000 // B)
    lo = rng.choice([0, _log_int(rng, 1, far)])
    c.update(lo=lo, hi=lo + rng.choice([0, rng.randint(0, 40)]))
    return c


def _lengths(c):
    """The lengths of a case's sequences; every seed deals out the same ones."""
    return [(c["lo"] + c["hi"]) // 2] if c["B"] == 1 else [c["lo"] + (c["hi"] - c["lo"]) * b // (c["B"] - 1) for b in range(c["B"])]


def _counts(c):
    return [max(1, c["T"] * (b + 3) // (c["B"] + 2)) if c["ragged"] else c["T"] for b in range(c["B"])]


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        rows = sum(_counts(c))
        return {"bytes": 2 * rows * (c["Hq"] + 2 * c["Hkv"]) * c["d"] * e, "flops": 3 * rows * (c["Hq"] + c["Hkv"]) * c["rot"]}
    if c["kind"] == "lwrite":
        rows, w = sum(_counts(c)), c["r"] + c["dr"]
        return {"bytes": 2 * rows * (w + c["H"] * c["dr"]) * e, "flops": rows * (4 * c["r"] + 3 * c["dr"] * (1 + c["H"]))}
    if c["kind"] == "lattn":
        keys, rows = sum(_lengths(c)) + c["B"] * c["n_q"], c["B"] * c["n_q"] * c["H"]
        pairs = sum(n + c["n_q"] for n in _lengths(c)) * c["n_q"] * c["H"]
        return {"bytes": (keys * (c["r"] + c["dr"]) + rows * (2 * c["r"] + c["dr"])) * e, "flops": 2 * pairs * (2 * c["r"] + c["dr"])}
    return {"bytes": c["M"] * (c["V"] * e + 4 + 8 * (c["n_tok"] + c["n_top"])), "flops": 4 * c["M"] * c["V"]}


# ------------------------------------------------------------------------------------ inputs

def _generator(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + sum(ord(x) * 31 for x in c["kind"]) + c.get("V", 0) + 17 * c.get("B", 0) + c.get("hi", 0))
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(g, shape, dtype):
    """Projected rows: normal values, a magnitude of its own for every row, and a few large channels."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    x[..., :3] *= 4.0
    return x.to(dtype)


def _shuffled(values, rng):
    values = list(values)
    rng.shuffle(values)
    return values


def _table(c, first, need, rng):
    """Pages for entries first[b] .. need[b] - 1 of every sequence, in random order; (table [B, max_pages], pages of the pool)."""
    spans = [(f // c["page"], (x + c["page"] - 1) // c["page"]) for f, x in zip(first, need)]
    total = sum(q - p for p, q in spans)
    total += max(2, total // 10)
    ids = _shuffled(range(total), rng)
    table = np.zeros((c["B"], max(max(q for _, q in spans), 1)), np.int32)
    at = 0
    for b, (p, q) in enumerate(spans):
        table[b, p:q] = ids[at:at + q - p]
        at += q - p
    return torch.from_numpy(table).cuda(), total


def _places(c, s, b, p):
    """Entries p (a tensor) of sequence b: indices of the pools' dimensions in front of and behind the head's."""
    if c["paged"]:
        return s["table"][b, p // c["page"]].long(), p % c["page"]
    return torch.full_like(p, b), p


def _pool(c, s, first, need, rng):
    """The pools' dimensions in front of and behind the head's."""
    if c["paged"]:
        s["table"], n = _table(c, first, need, rng)
        return n, c["page"]
    s["table"] = None
    return c["B"], (max(need) + 15) // 16 * 16


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
        out.append([w - (1 << 64) if w >> 63 else w for w in words])
    return torch.tensor(out, dtype=torch.int64, device="cuda")


def _depths(c, rng):
    """How far a token's rotary position lies behind its sequence's first one: its node's depth, or its number."""
    if not c["tree"]:
        return [list(range(c["T"]))] * c["B"]
    out = []
    for _ in range(c["B"]):
        depth = []
        for p in _tree(c["T"], rng):
            depth.append(depth[p] + 1 if p >= 0 else 0)
        out.append(depth)
    return out


def _rope(c):
    """The rotation of a case: (pairs' layout, rotated values, base, scaling, factor, low, high, length before scaling, amplitude)."""
    if c["kind"] == "lwrite":
        return (True, c["dr"], 1e4, RAMP, 40.0, 1.0, 32.0, 4096, 1.0)
    amplitude = 0.1 * math.log(32.0) + 1.0 if c["scaling"] == RAMP else 1.0
    low, high = (1.0, 4.0) if c["scaling"] == BANDS else (1.0, 32.0)
    return (c["interleaved"], c["rot"], c["theta"], c["scaling"], 1.0 if c["scaling"] == NONE else 32.0 if c["scaling"] == RAMP else 8.0, low, high, 8192,
            float(np.float32(amplitude)))


def _frequencies(rope):
    """Angles per position of every pair, in 64 bits."""
    _, rot, theta, scaling, factor, low, high, length, _ = rope
    c = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = theta ** (-2.0 * c / rot)
    if scaling == LINEAR:
        return f / factor
    if scaling == BANDS:
        keep = ((length * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / factor)
    if scaling == RAMP:
        at = lambda turns: rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(theta))
        first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
        away = ((c - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
        return f * (1.0 - away) + f / factor * away
    return f


def prepare(c, seed):
    g, rng = _generator(c, seed), random.Random(977 * seed + 5)
    s = {"case": c}
    dt = DTYPES[c["dtype"]]
    B = c.get("B")
    if c["kind"] in ("rope", "lwrite"):
        T = c["T"]
        counts, pos, depth = _shuffled(_counts(c), rng), _shuffled(_lengths(c), rng), _depths(c, rng)
        s["host"] = (pos, counts, depth)
        s["pos"], s["count"] = _i32(pos), _i32(counts) if c["ragged"] else None
        s["offset"] = _i32(depth) if c["tree"] else None
        s["at"] = s["pos"].double().unsqueeze(1) + _i32(depth).double()           # rotary positions [B, T]
        s["rope"] = _rope(c)
        lead = _pool(c, s, pos, [p + n for p, n in zip(pos, counts)], rng) if c["kind"] == "lwrite" or c["append"] else None
    if c["kind"] == "rope":
        Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
        if c["fused"]:
            x = _rows(g, (B, T, Hq + 2 * Hkv, d), dt)
            s["q_rows"], s["k_rows"], s["v_rows"] = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
        else:
            s["q_rows"], s["k_rows"], s["v_rows"] = (_rows(g, (B, T, h, d), dt) for h in (Hq, Hkv, Hkv))
        s["q"] = torch.zeros((B, T, Hq, d), dtype=dt, device="cuda")
        if c["append"]:
            s["k"], s["v"] = (torch.zeros((lead[0], Hkv, lead[1], d), dtype=dt, device="cuda") for _ in range(2))
    elif c["kind"] == "lwrite":
        w = c["r"] + c["dr"]
        s["rows"] = _rows(g, (B, T, w), dt)
        s["gain"] = (1.0 + 0.1 * torch.randn(c["r"], generator=g, device="cuda")).to(dt)
        # the rotated part of a head's query follows the part that the latent's projection takes in
        s["q_rows"] = _rows(g, (B, T, c["H"], 2 * c["dr"] + c["dr"]), dt)[..., 2 * c["dr"]:] if c["H"] else None
        s["q"] = torch.randn((B, T, c["H"], w), generator=g, device="cuda").to(dt) if c["H"] else None
        s["c"] = torch.zeros((*lead, w), dtype=dt, device="cuda")
    elif c["kind"] == "lattn":
        L, w = _shuffled(_lengths(c), rng), c["r"] + c["dr"]
        lead = _pool(c, s, [0] * B, [x + c["n_q"] for x in L], rng)
        s["c"] = torch.randn((*lead, w), generator=g, device="cuda").to(dt)
        s["c"][..., c["r"]:] *= 2.0
        s["q"] = torch.randn((B, c["n_q"], c["H"], w), generator=g, device="cuda").to(dt)
        s["L"], s["ctx"] = L, _i32(L)
        s["mask"] = _masks(c, rng) if c["tree"] else None
        s["scale"] = (2 * c["dr"] + c["dr"]) ** -0.5
        s["out"] = torch.empty((B, c["n_q"], c["H"], c["r"]), dtype=dt, device="cuda")
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
        # what was drafted: the target's best token or one of the others
        best = s["logits"][:, :V].float().argmax(1, keepdim=True).to(torch.int32)
        s["token"] = torch.randint(0, V, (M, c["n_tok"]), generator=g, device="cuda", dtype=torch.int32)
        if c["n_tok"]:
            s["token"][::2, :1] = best[::2]
        s["heat"] = torch.tensor([rng.uniform(0.5, 1.3) for _ in range(n)], dtype=torch.float32, device="cuda") if c["heat"] else None
        for name, shape, t in (("logprob", (M, c["n_tok"]), torch.float32), ("entropy", (M,), torch.float32), ("top", (M, c["n_top"]), torch.int32),
                               ("top_logprob", (M, c["n_top"]), torch.float32)):
            s[name] = torch.zeros(shape, dtype=t, device="cuda")
    if own:
        from paper_2509_24248_amd import binding as sx
        s["code"] = sx.dtype_code(dt)
        if "rope" in s:
            pairs, rot, theta, scaling, factor, low, high, length, amplitude = s["rope"]
            s["desc"] = sx.rope_desc(rot, theta, interleaved=pairs, scaling=scaling, factor=factor, low=low, high=high, orig_len=length,
                                     amplitude=amplitude)
            s["turns"] = torch.empty(rot // 2, dtype=torch.int64, device="cuda")
            sx.specexit_rope_table(s["desc"], s["turns"])
        if c["kind"] == "rope" and c["append"]:
            s["view"] = sx.kv_view(s["k"], s["v"], s["table"])
        if c["kind"] in ("lwrite", "lattn"):
            s["view"] = sx.latent_kv_view(s["c"], c["dr"], s["table"])
        if c["kind"] == "lattn":
            s["ws"] = _bytes(sx.specexit_latent_verify_attn_workspace_bytes(s["view"], B, c["n_q"], c["H"]))
        if c["kind"] == "logprob":
            s["ws"] = _bytes(sx.specexit_token_logprobs_workspace_bytes(s["code"], c["M"], c["V"], c["n_top"]))
    return s


# ------------------------------------------------------------------------------------ one pass

def run(s):
    return {"rope": _run_rope, "lwrite": _run_lwrite, "lattn": _run_lattn, "logprob": _run_logprob}[s["case"]["kind"]](s)


def _rotate(s, x):
    """x [B, T, heads, d] with its leading `rot` values rotated, in 32 bits; angles in 64."""
    pairs, rot, _, _, _, _, _, _, amplitude = s["rope"]
    angle = s["at"].unsqueeze(-1) * _frequencies(s["rope"])
    cos, sin = ((f(angle) * amplitude).float().unsqueeze(2) for f in (torch.cos, torch.sin))
    y = x.float().clone()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if pairs else (y[..., :rot // 2], y[..., rot // 2:rot])
    first, second = a * cos - b * sin, a * sin + b * cos
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = first, second
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = first, second
    return y


def _run_rope(s):
    c = s["case"]
    if own:
        from paper_2509_24248_amd import binding as sx
        if not c["append"]:
            sx.specexit_rope(s["code"], s["desc"], s["turns"], c["B"], c["T"], c["Hq"], c["d"], s["q_rows"], s["q"], s["pos"], s["offset"], s["count"])
            return [s["q"]]
        sx.specexit_rope_kv_write(s["view"], s["desc"], s["turns"], c["B"], c["T"], c["Hq"], s["q_rows"], s["k_rows"], s["v_rows"], s["q"], s["pos"],
                                  s["offset"], s["count"])
        return [s["q"], s["k"], s["v"]]
    pos, counts, _ = s["host"]
    q = _rotate(s, s["q_rows"]).to(s["q"].dtype)
    for b in range(c["B"]):
        s["q"][b, :counts[b]] = q[b, :counts[b]]
    if not c["append"]:
        return [s["q"]]
    k = _rotate(s, s["k_rows"]).to(s["k"].dtype)
    for b in range(c["B"]):
        i, j = _places(c, s, b, torch.arange(pos[b], pos[b] + counts[b], device="cuda"))
        s["k"][i, :, j], s["v"][i, :, j] = k[b, :counts[b]], s["v_rows"][b, :counts[b]]
    return [s["q"], s["k"], s["v"]]


def _run_lwrite(s):
    c = s["case"]
    out = [s["c"]] + ([s["q"]] if c["H"] else [])
    if own:
        from paper_2509_24248_amd import binding as sx
        sx.specexit_latent_kv_write(s["view"], s["desc"], s["turns"], c["B"], c["T"], c["H"], s["rows"], s["gain"], EPS, s["q_rows"], s["q"], s["pos"],
                                    s["offset"], s["count"])
        return out
    pos, counts, _ = s["host"]
    r = c["r"]
    x = s["rows"].float()
    lat = x[..., :r] * torch.rsqrt((x[..., :r] * x[..., :r]).mean(-1, keepdim=True) + EPS) * s["gain"].float()
    row = torch.cat([lat, _rotate(s, x[..., r:].unsqueeze(2)).squeeze(2)], -1).to(s["c"].dtype)
    q = _rotate(s, s["q_rows"]).to(s["c"].dtype) if c["H"] else None
    for b in range(c["B"]):
        i, j = _places(c, s, b, torch.arange(pos[b], pos[b] + counts[b], device="cuda"))
        s["c"][i, j] = row[b, :counts[b]]
        if c["H"]:
            s["q"][b, :counts[b], :, r:] = q[b, :counts[b]]
    return out


def _run_lattn(s):
    c = s["case"]
    if own:
        from paper_2509_24248_amd import binding as sx
        sx.specexit_latent_verify_attn(s["view"], c["B"], c["n_q"], c["H"], s["q"], s["ctx"], s["mask"], s["scale"], s["out"], s["ws"])
        return s["out"]
    n_q, H, r = c["n_q"], c["H"], c["r"]
    for b in range(c["B"]):
        L = s["L"][b]
        i, j = _places(c, s, b, torch.arange(L + n_q, device="cuda"))
        k = s["c"][i, j].float()
        x = torch.matmul(s["q"][b].float().reshape(n_q * H, -1), k.t().contiguous()) * s["scale"]
        bits = torch.arange(n_q, device="cuda")
        seen = (s["mask"][b].unsqueeze(1) >> bits) & 1 == 1 if s["mask"] is not None else bits.unsqueeze(0) <= bits.unsqueeze(1)
        x[:, L:].masked_fill_(~seen.repeat_interleave(H, 0), -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        o = torch.matmul(p, k[:, :r].contiguous()) / p.sum(-1, keepdim=True)
        s["out"][b] = o.reshape(n_q, H, r).to(s["out"].dtype)
    return s["out"]


def _run_logprob(s):
    c = s["case"]
    out = [s["logprob"], s["entropy"], s["top"], s["top_logprob"]]
    if own:
        from paper_2509_24248_amd import binding as sx
        sx.specexit_token_logprobs(s["code"], c["M"], c["V"], s["logits"], s["entropy"], token=s["token"], logprob=s["logprob"], top_token=s["top"],
                                   top_logprob=s["top_logprob"], temperature=s["heat"], rows_per_seq=c["per"], workspace=s["ws"])
        return out
    l = s["logits"][:, :c["V"]].float()
    heat = torch.ones((c["M"], 1), device="cuda") if s["heat"] is None else s["heat"].repeat_interleave(c["per"])[:c["M"]].unsqueeze(1)
    # 64 bits: the sum of many small weights beside a large one
    y = (l.double() - l.double().amax(1, keepdim=True)) / heat.double()
    w = torch.exp(y)
    total = w.sum(1, keepdim=True)
    logp = y - torch.log(total)
    s["entropy"].copy_(-torch.where(w > 0, w * logp, 0.0).sum(1) / total.squeeze(1))
    s["logprob"].copy_(torch.gather(logp, 1, s["token"].long()))
    if c["n_top"]:
        _, order = torch.sort(l, dim=1, descending=True, stable=True)
        best = order[:, :c["n_top"]]
        s["top"].copy_(torch.where(torch.isinf(torch.gather(l, 1, best)), -1, best))
        s["top_logprob"].copy_(torch.gather(logp, 1, best))
    return out


# ------------------------------------------------------------------------------------ in 64 bits, from the definitions

def exact(c, seed):
    s = prepare(c, seed)
    return {"rope": _exact_rope, "lwrite": _exact_lwrite, "lattn": _exact_lattn, "logprob": _exact_logprob}[c["kind"]](c, s)


def _turned(c, s, x):
    """x [B, T, heads, d] rotated pair by pair as complex numbers, in 64 bits."""
    pairs, rot, theta, scaling, factor, low, high, length, amplitude = s["rope"]
    pos, _, depth = s["host"]
    rate = []
    for i in range(rot // 2):
        f = math.exp(-2.0 * i / rot * math.log(theta))
        if scaling == LINEAR:
            f /= factor
        elif scaling == BANDS:
            n = length * f / (2.0 * math.pi)
            f = f if n >= high else f / factor if n <= low else f * ((n - low) / (high - low) + (high - n) / (high - low) / factor)
        elif scaling == RAMP:
            border = lambda turns: rot * math.log(length / (2.0 * math.pi * turns)) / (2.0 * math.log(theta))
            a, z = max(math.floor(border(high)), 0), min(math.ceil(border(low)), rot - 1)
            t = min(max((i - a) / max(z - a, 0.001), 0.0), 1.0)
            f = (1.0 - t) * f + t * f / factor
        rate.append(f)
    at = torch.tensor([[p + k for k in row] for p, row in zip(pos, depth)], dtype=torch.float64)
    turn = torch.polar(torch.full((1,), amplitude, dtype=torch.float64), at.unsqueeze(-1) * torch.tensor(rate, dtype=torch.float64)).cuda().unsqueeze(2)
    y = x.double()
    head = y[..., :rot].unflatten(-1, (rot // 2, 2) if pairs else (2, rot // 2))
    z = (torch.complex(head[..., 0], head[..., 1]) if pairs else torch.complex(head[..., 0, :], head[..., 1, :])) * turn
    return torch.cat([torch.stack([z.real, z.imag], -1 if pairs else -2).flatten(-2), y[..., rot:]], -1)


def _index(c, s, b):
    """Where the tokens of sequence b go: indices in front of and behind the head's, and how many there are."""
    pos, counts, _ = s["host"]
    p = torch.arange(counts[b], device="cuda") + pos[b]
    if not c["paged"]:
        return torch.full_like(p, b), p, counts[b]
    row = s["table"][b].long()
    return row[torch.div(p, c["page"], rounding_mode="floor")], torch.remainder(p, c["page"]), counts[b]


def _exact_rope(c, s):
    q, turned = s["q"].double(), _turned(c, s, s["q_rows"])
    for b, n in enumerate(s["host"][1]):
        q[b, :n] = turned[b, :n]
    if not c["append"]:
        return [q]
    k, v, turned = s["k"].double(), s["v"].double(), _turned(c, s, s["k_rows"])
    for b in range(c["B"]):
        i, j, n = _index(c, s, b)
        k[i, :, j], v[i, :, j] = turned[b, :n], s["v_rows"][b, :n].double()
    return [q, k, v]


def _exact_lwrite(c, s):
    r, pool = c["r"], s["c"].double()
    x = s["rows"].double()
    lat = x[..., :r] / torch.sqrt(x[..., :r].pow(2).sum(-1, keepdim=True) / r + EPS) * s["gain"].double()
    pe = _turned(c, s, x[..., None, r:])[..., 0, :]
    q = s["q"].double() if c["H"] else None
    qt = _turned(c, s, s["q_rows"]) if c["H"] else None
    for b in range(c["B"]):
        i, j, n = _index(c, s, b)
        pool[i, j] = torch.cat([lat[b, :n], pe[b, :n]], -1)
        if c["H"]:
            q[b, :n, :, r:] = qt[b, :n]
    return [pool] + ([q] if c["H"] else [])


def _exact_lattn(c, s):
    r, out = c["r"], torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        L, n = s["L"][b], s["L"][b] + c["n_q"]
        at = torch.arange(n, device="cuda")
        rows = s["c"][s["table"][b].long()[at // c["page"]], at % c["page"]] if c["paged"] else s["c"][b, :n]
        rows = rows.double()
        for i in range(c["n_q"]):
            word = int(s["mask"][b, i]) if s["mask"] is not None else (2 << i) - 1
            keys = rows[list(range(L)) + [L + j for j in range(c["n_q"]) if word >> j & 1]] if word + 1 != 1 << c["n_q"] else rows
            out[b, i] = torch.softmax(s["q"][b, i].double() @ keys.t() * s["scale"], 1) @ keys[:, :r]
    return out


def _exact_logprob(c, s):
    l = s["logits"][:, :c["V"]].float().double()
    if s["heat"] is not None:
        l = l / s["heat"].double()[torch.arange(c["M"], device="cuda") // c["per"]].unsqueeze(1)
    logp = torch.log_softmax(l, 1)
    p = torch.exp(logp)
    entropy = -(p * torch.where(p > 0, logp, 0.0)).sum(1)
    raw = s["logits"][:, :c["V"]].float().cpu().numpy()
    top = np.argsort(-raw, axis=1, kind="stable")[:, :c["n_top"]].astype(np.int64)
    best = torch.from_numpy(top).cuda()
    top = np.where(np.take_along_axis(raw, top, 1) == -np.inf, -1, top)
    return [torch.gather(logp, 1, s["token"].long()), entropy, torch.from_numpy(top.astype(np.int32)), torch.gather(logp, 1, best)]
