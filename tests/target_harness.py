"""Plumbing of the tests of rotary writes, the latent cache and log probabilities."""
from __future__ import annotations

import numpy as np
import torch

from oracle import specexit_oracle as O
from workloads import gen

import harness as H

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # a rounding to the type, relative
U = 2.0 ** -24


def stored(x, dtype):
    x = np.asarray(x, np.float32)
    return gen.round_to_bf16(x) if dtype == "bf16" else x


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(DT[dtype])


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


class Rope:
    """A rotation for the oracle and for the library."""

    def __init__(self, rot, theta=1e6, interleaved=False, scaling=0, factor=1.0, low=1.0, high=32.0, orig_len=4096, amplitude=1.0):
        f32 = lambda v: float(np.float32(v))
        theta, factor, low, high, self.amplitude = f32(theta), f32(factor), f32(low), f32(high), f32(amplitude)
        self.rot, self.interleaved = rot, interleaved
        self.f = O.rope_frequencies(rot, theta, scaling, factor, low, high, orig_len)
        self.args = dict(rot_dim=rot, theta=theta, interleaved=interleaved, scaling=scaling, factor=factor, low=low, high=high, orig_len=orig_len,
                         amplitude=self.amplitude)

    def gpu(self):
        lib = H.sx()
        desc = lib.rope_desc(**self.args)
        turns = torch.empty(self.rot // 2, dtype=torch.int64, device="cuda")
        lib.specexit_rope_table(desc, turns)
        return desc, turns

    def heads(self, x, position):
        """[B, T, heads, d] at positions [B, T]"""
        return np.stack([O.rope_heads(x[b], position[b], self.f, self.interleaved, self.amplitude) for b in range(len(x))])

    def bound(self, x, ref, dtype):
        """The result's rounding, and of x cos t - y sin t in fp32: products and sum 2^-23 of |x| + |y|; cosine and sine, of t cut to 2^-32 turns and its conversion and
        factor rounded (2^-23 at most of what lies within pi / 4) and polynomials of six steps whose last two count (2^-23) and times the amplitude (2^-24), 2^-22."""
        x = np.abs(np.asarray(x, np.float64))
        rot = self.rot
        pair = np.zeros_like(x)
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if self.interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        pair[..., a] = pair[..., b] = x[..., a] + x[..., b]
        return (HALF[dtype] if dtype == "bf16" else U) * np.abs(ref) + self.amplitude * pair * (2.0 ** -22 + 2.0 ** -23)


class Latent:
    """A latent cache as a numpy array, contiguous or paged."""

    def __init__(self, rng, B, r, need, dtype, page=None):
        self.r, self.page, self.dtype = r, page, dtype
        need = [int(n) for n in need]
        self.table = None
        if page is None:
            lead = (B, max(need))
        else:
            pages = [(n + page - 1) // page for n in need]
            total = sum(pages) + 2
            perm, at = rng.permutation(total), 0
            self.table = np.zeros((B, max(max(pages), 1)), np.int32)
            for b, n in enumerate(pages):
                self.table[b, :n] = perm[at:at + n]
                at += n
            lead = (total, page)
        self.c = stored(rng.standard_normal(lead + (r + 64,)), dtype)

    def gpu(self):
        """(view, cache tensor, page table or None)"""
        c = dev(self.c, self.dtype)
        table = None if self.table is None else i32(self.table)
        return H.sx().latent_kv_view(c, 64, table), c, table

    def at(self, b, p):
        return (b, p) if self.table is None else (int(self.table[b, p // self.page]), p % self.page)


def run_latent_attn(view, B, n_q, Hq, r, q, L, mask, scale, dtype, flags=0, stream=None):
    lib, guard = H.sx(), H.Guarded()
    out = guard.empty((B, n_q, Hq, r), DT[dtype])
    need = lib.specexit_latent_verify_attn_workspace_bytes(view, B, n_q, Hq)
    assert need > 0, lib.last_error()
    ws = guard.empty(need, torch.uint8)
    lib.specexit_latent_verify_attn(view, B, n_q, Hq, dev(q, dtype), i32(L), None if mask is None else H.dev(mask), scale, out, ws, flags=flags,
                                    stream=stream)
    guard.check()
    return H.host(out)


def latent_attn_bound(ref, weighed, q, c, r, n, scale, dtype):
    """How far the result may be off, element by element.  A product of a score passes through a matrix instruction (32 or 4 products) and the sum over w = r + 64
    dimensions, 32 or 4 at a time: at most `path` roundings of 2^-24 of the sum of |q c|; scaling and the distance from the reference three more; that twice
    (the normaliser has it too) and the exponential's 2^-22 move a probability.  Sums over n keys pass n / 32 (n / 4) steps, the rings' and segments' merges 40 more.
    bf16: probabilities in two parts are off by 2^-16, one part by half a step, 2^-8; and the result's own rounding."""
    w = q.shape[-1]
    reach = scale * float(np.nanmax(np.abs(q).sum(-1)) * np.nanmax(np.abs(c[np.isfinite(c)])))
    per = 32 if dtype == "bf16" else 4
    eps = 2 * ((per + w // per + 6) * U * reach) + 2.0 ** -22 + (n // per + per + 40) * U
    part = 0.0 if dtype == "f32" else (2.0 ** -16 if q.shape[1] * q.shape[2] <= 64 else 2.0 ** -8)
    return (weighed + np.abs(ref)) * (eps + part / 2) + weighed * part / 2 + (HALF[dtype] if dtype == "bf16" else U) * np.abs(ref) + 1e-30


def tree_masks(rng, B, n_q):
    parent = np.full((B, n_q), -1, np.int64)
    for b in range(B):
        for c in range(1, n_q):
            parent[b, c] = rng.integers(max(0, (c - 4) // 2), c)
    return gen.ancestor_masks(parent), parent


def depths(parent):
    out = np.zeros(parent.shape, np.int32)
    for b in range(parent.shape[0]):
        for c in range(1, parent.shape[1]):
            out[b, c] = out[b, parent[b, c]] + 1
    return out


def logprob_bound(y, lp, weight):
    """Absolute error of a log probability (y its logit's distance from the best over the temperature): difference and quotient 2^-23 of |y|; the logarithms' sum: their
    arguments are sums of at most 128 roundings whose weights are off by 2^-22 of their distance (`weight`: its mean) and 2^-22, and 2^-22 of what they come to; the result's rounding."""
    y, lp = np.abs(np.where(np.isfinite(y), y, 0.0)), np.abs(np.where(np.isfinite(lp), lp, 0.0))
    return 2.0 ** -22 * (y + lp + abs(weight) + 2) + 128 * U
