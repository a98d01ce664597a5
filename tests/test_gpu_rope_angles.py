"""GPU: sines and cosines themselves, read off heads whose pairs are (0, 1), within what the library states of them."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O

import harness as H
from target_harness import Rope, i32
from test_gpu_rope import SCALED

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("scaling", range(4))
def test_sines_and_cosines(scaling, interleaved):
    """Positions from one on, where the slow pairs have hardly turned, to the last one."""
    lib, rng = H.sx(), np.random.default_rng(scaling)
    rot = 128
    r = Rope(rot, interleaved=interleaved, **SCALED[scaling])
    desc, turns = r.gpu()
    pos = np.unique(np.concatenate([np.arange(40), np.exp(rng.uniform(0, np.log(2.0 ** 31 - 1), 200)).astype(np.int64), [2 ** 31 - 1]]))
    x = torch.zeros((len(pos), 1, 1, rot), device="cuda")
    if interleaved:
        x[..., 1::2] = 1.0
    else:
        x[..., rot // 2:] = 1.0
    out = torch.empty_like(x)
    lib.specexit_rope(lib.F32, desc, turns, len(pos), 1, 1, rot, x, out, i32(pos))
    got = H.host(out)[:, 0, 0].astype(O.LONG)
    sn, cs = (-got[:, 0::2], got[:, 1::2]) if interleaved else (-got[:, :rot // 2], got[:, rot // 2:])
    angle = pos.astype(O.LONG)[:, None] * r.f
    two_pi = 2 * O.LONG(np.pi) + O.LONG(2.4492935982947064e-16)
    amplitude = O.LONG(r.amplitude)
    # the angle (64-bit table, the cut at 2^-32 turns), and 32 bits: conversion, factor and product of the angle's rest 3 roundings of 2^-24, the polynomials' last two steps and
    # what is below them 2.3 (sine) or, of at least 0.7, 5, the amplitude one: 2^-21 of the value
    off = amplitude * (pos[:, None] * (two_pi * O.LONG(2.0) ** -64 + O.LONG(2.0) ** -48 * r.f) + two_pi * O.LONG(2.0) ** -32)
    for name, a, b in (("sine", sn, amplitude * np.sin(angle)), ("cosine", cs, amplitude * np.cos(angle))):
        share = np.abs(a - b) / (off + O.LONG(2.0) ** -21 * np.abs(b))
        print(name, "worst share of the bound %.3f" % float(share.max()), flush=True)
        assert share.max() <= 1.0
