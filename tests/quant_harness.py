"""Plumbing of the tests of the 8-bit cache: caches in the oracle's terms and on the GPU."""
from __future__ import annotations

import numpy as np
import torch

from oracle import specexit_oracle as O
from workloads import gen

import harness as H


class Cache:
    """An 8-bit cache as numpy arrays: codes and scale bytes of random rows, contiguous or paged."""

    def __init__(self, rng, B, Hkv, d, need, page=None, spread=1.0):
        self.B, self.Hkv, self.d, self.page = B, Hkv, d, page
        need = [int(n) for n in need]
        if page is None:
            lead = (B, Hkv, (max(need) + 15) // 16 * 16)
            self.table = None
        else:
            pages = [(n + page - 1) // page for n in need]
            total = sum(pages) + 3
            perm = rng.permutation(total)
            self.table = np.zeros((B, max(max(pages), 1)), np.int32)
            at = 0
            for b, n in enumerate(pages):
                self.table[b, :n] = perm[at:at + n]
                at += n
            lead = (total, Hkv, page)
        x = lambda: rng.standard_normal(lead + (d,)) * np.exp(spread * rng.standard_normal(lead))[..., None]
        (self.k, self.ks), (self.v, self.vs) = O.quant_rows(x()), O.quant_rows(x())

    def values(self):
        return O.dequant_rows(self.k, self.ks), O.dequant_rows(self.v, self.vs)

    def gpu(self):
        """(view, tensors): tensors = [k, v, k_scale, v_scale, page table or None]"""
        t = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (self.k, self.v, self.ks, self.vs)]
        t.append(None if self.table is None else torch.from_numpy(self.table).cuda())
        return H.sx().quant_kv_view(*t), t

    def at(self, b, p):
        """Index of entry p of sequence b in the pools, head left open."""
        if self.table is None:
            return b, slice(None), p
        return int(self.table[b, p // self.page]), slice(None), p % self.page


def attn(cache, q, L, mask=None, scale=None, dtype="bf16", flags=0, view=None):
    lib = H.sx()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    view = cache.gpu() if view is None else view
    B, n_q, Hq, d = q.shape
    code = lib.dtype_code(dt)
    guard = H.Guarded()
    out = guard.empty(q.shape, dt)
    need = lib.specexit_quant_verify_attn_workspace_bytes(view[0], code, B, n_q, Hq)
    assert need > 0, lib.last_error()
    ws = guard.empty(need, torch.uint8)
    lib.specexit_quant_verify_attn(view[0], code, B, n_q, Hq, torch.from_numpy(np.asarray(q, np.float32)).cuda().to(dt),
                                   torch.from_numpy(np.asarray(L, np.int32)).cuda(), None if mask is None else H.dev(mask),
                                   d ** -0.5 if scale is None else scale, out, ws, flags=flags)
    guard.check()
    return out.float().cpu().numpy()


def attn_bound(ref, weighed, q, k, v, n, scale, dtype):
    """How far the result may be off, element by element.

    bf16: the output's rounding (half a step, 2^-8 of the value); the probabilities' roundings, half a step each: the scale of a V row is a power of
    two, so sum p |v| of the row's own probabilities (`weighed`) times 2^-8 at most; a score's sum drops from
    each of the d products of a part what lies 2^-23 below the largest one, d 2^-23 scale max|q| max|k| for the first part and a sixteenth of it for
    the second, which moves a probability by that and the normaliser by as much again; sums over n keys in fp32, 2^-23 n.
    fp32: products are exact, sums of d and of n numbers in fp32: 2^-23 (d + n) of the absolute ones."""
    d = q.shape[-1]
    top = scale * np.nanmax(np.abs(q)) * np.nanmax(np.abs(k))
    vmax = np.nanmax(np.abs(v))
    if dtype == "bf16":
        return 2.0 ** -8 * (np.abs(ref) + weighed) + vmax * (2.0 ** -15 + 2.2 * d * 2.0 ** -23 * top + n * 2.0 ** -23)
    return 2.0 ** -23 * np.abs(ref) + vmax * (2.0 ** -22 + 2 * d * 2.0 ** -23 * top + n * 2.0 ** -23)


def check_attn(cache, q, L, mask=None, scale=None, dtype="bf16", got=None, only=None):
    """GPU result against the oracle's, within attn_bound."""
    k, v = cache.values()
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    if got is None:
        got = attn(cache, q, L, mask, scale, dtype)
    ref = O.verify_attn(q, k, v, L, mask, scale, cache.table, cache.page or 16, only)
    weighed = O.verify_attn(q, k, np.abs(v), L, mask, scale, cache.table, cache.page or 16, only)
    if only is not None:
        sel = tuple(np.array(only).T)
        got, ref, weighed = got[sel], ref[sel], weighed[sel]
    assert np.isfinite(got).all()
    bound = attn_bound(ref, weighed, q, k, v, int(max(L)) + q.shape[1], scale, dtype)
    over = np.abs(got - ref) / bound
    assert over.max() <= 1.0, (float(over.max()), float(np.abs(got - ref).max()))
    return float(over.max())


def queries(rng, B, n_q, Hq, d, dtype):
    q = rng.standard_normal((B, n_q, Hq, d)).astype(np.float32)
    return gen.round_to_bf16(q) if dtype == "bf16" else q


def tree_masks(rng, B, n_q):
    parent = np.full((B, n_q), -1, np.int64)
    for b in range(B):
        for c in range(1, n_q):
            parent[b, c] = rng.integers(max(0, (c - 4) // 2), c)
    return gen.ancestor_masks(parent)
