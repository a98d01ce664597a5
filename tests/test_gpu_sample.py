"""GPU: sampled tokens against the oracle's; tokens are equal, shares within the rounding to 32 bits."""
import numpy as np
import pytest
import torch

from oracle import specexit_oracle as O
from workloads import gen

import harness as H

pytestmark = pytest.mark.gpu

# the weights' polynomial 3.2e-14, a weight's and the sum's fixed-point steps, 2^-46 of the best weight per token (V 2^-46 of the sum at most), and the
# rounding of the share to fp32
def prob_bound(V):
    return 2.0 ** -24 + V * 2.0 ** -46 + 1e-12


def run(logits, u, dtype="f32", per=1, flags=0, pad=0, guard=None, **kw):
    lib = H.sx()
    M, V = logits.shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    wide = torch.full((M, V + pad), 1e30, dtype=dt, device="cuda")
    wide[:, :V] = torch.from_numpy(logits).cuda().to(dt)
    guard = H.Guarded()
    token, prob = guard.empty(M, torch.int32), guard.empty(M, torch.float32)
    need = lib.specexit_sample_workspace_bytes(lib.dtype_code(dt), M, V)
    ws = guard.empty(need, torch.uint8)
    args = {}
    for n, t in (("temperature", np.float32), ("top_k", np.int32), ("top_p", np.float32), ("min_p", np.float32)):
        args[n] = None if kw.get(n) is None else torch.from_numpy(np.asarray(kw[n], t)).cuda()
    lib.specexit_sample(lib.dtype_code(dt), M, V, wide[:, :V], torch.from_numpy(np.asarray(u, np.float32)).cuda(), token, prob,
                        rows_per_seq=per, workspace=ws, flags=flags, **args)
    guard.check()
    return token.cpu().numpy(), prob.cpu().numpy()


def check(logits, u, dtype="f32", per=1, pad=0, rows=None, **kw):
    if dtype == "bf16":
        fin = np.isfinite(logits)
        logits = np.where(fin, gen.round_to_bf16(np.where(fin, logits, 0).astype(np.float32)), logits).astype(np.float32)
    token, prob = run(logits, u, dtype, per, pad=pad, **kw)
    at = lambda n, r, off: off if kw.get(n) is None else float(np.float32(kw[n][r // per])) if n != "top_k" else int(kw[n][r // per])
    for r in range(logits.shape[0]) if rows is None else rows:
        t, p, _ = O.sample(logits[r], np.float32(u[r]), at("temperature", r, 1.0), at("top_k", r, 0), at("top_p", r, 1.0), at("min_p", r, 0.0))
        assert token[r] == t, (r, int(token[r]), t, {n: at(n, r, None) for n in kw})
        assert abs(prob[r] - p) <= prob_bound(logits.shape[1]) * max(p, 2.0 ** -40) + 2.0 ** -46, (r, prob[r], p)
    return token, prob


def head_like(rng, M, V):
    x = rng.standard_normal((M, V)).astype(np.float32) * 2.2
    for r in range(M):
        k = min(V, 5 + 9 * (r % 6))
        x[r, rng.integers(0, V, k)] += np.linspace(13, 3, k).astype(np.float32) * (0.6 + 0.1 * (r % 5))
    return x


SETTINGS = {
    "none": {},
    "k": dict(top_k=[20, 1, 50, 400]),
    "p": dict(top_p=[0.9, 0.5, 0.99, 0.999]),
    "m": dict(min_p=[0.05, 0.5, 0.001, 1.0]),
    "kp": dict(top_k=[20, 50, 1000, 5], top_p=[0.95, 0.8, 0.99, 0.3]),
    "all": dict(top_k=[40, 0, 1024, -3], top_p=[0.95, 0.9, 1.0, 0.97], min_p=[0.02, 0.01, 0.0, 0.3]),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 37, 511, 512, 513, 4096, 32003])
@pytest.mark.parametrize("mode", list(SETTINGS))
def test_settings(dtype, V, mode):
    rng = np.random.default_rng(V + len(mode))
    M, per = 12, 3
    kw = dict(SETTINGS[mode], temperature=[0.6, 1.0, 1.7, 0.0])
    check(head_like(rng, M, V), rng.random(M, np.float32), dtype, per, pad=V % 4, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 7, 144])
def test_a_whole_vocabulary(dtype, M):
    rng = np.random.default_rng(M)
    V = 151936
    kw = dict(temperature=0.5 + rng.random(M), top_k=rng.choice([0, 20, 300], M), top_p=rng.choice([1.0, 0.95, 0.8], M), min_p=rng.choice([0.0, 0.03], M))
    check(head_like(rng, M, V), rng.random(M, np.float32), dtype, rows=range(0, M, max(1, M // 24)), **kw)


def test_the_widest_vocabulary():
    rng = np.random.default_rng(2)
    V = H.sx().SAMPLE_MAX_V
    check(head_like(rng, 2, V), np.float32([0.3, 0.99999]), top_p=[0.9, 1.0])


@pytest.mark.parametrize("mode", ["none", "k", "p", "kp", "all"])
def test_equal_logits(mode):
    """All tokens of a row alike: ties go to the lowest index; lists that do not fit are done without."""
    rng = np.random.default_rng(3)
    M, V = 8, 20011
    kw = dict(SETTINGS[mode])
    x = np.full((M, V), 3.25, np.float32)
    x[4:] = np.where(np.arange(V) % 3 == 0, 3.25, 1.0)             # two weights
    u = rng.random(M, np.float32)
    check(x, u, per=2, **kw)


@pytest.mark.parametrize("spread", [0.01, 0.3, 1.0])
def test_flat_rows(spread):
    """Thousands of tokens of nearly one weight at the border of top-p and top-k."""
    rng = np.random.default_rng(4)
    M, V = 6, 60000
    x = (rng.standard_normal((M, V)) * spread).astype(np.float32)
    check(x, rng.random(M, np.float32), top_p=[0.9, 0.5, 0.1, 1.0, 0.95, 0.7], top_k=[0, 0, 0, 1000, 900, 7])


def test_every_u():
    rng = np.random.default_rng(5)
    M, V = 200, 3000
    x = np.repeat(head_like(rng, 1, V), M, 0)
    u = np.concatenate([[0.0, 0.99999994, 2.0 ** -24], np.linspace(0, 1, M - 3, endpoint=False)]).astype(np.float32)
    token, _ = check(x, u, temperature=[0.9] * M, top_p=[0.98] * M)
    check(x, u)
    order = np.argsort(u)
    assert (np.diff(token[order]) >= 0).all()                    # a larger number never gives a lower index
    # numbers outside [0, 1) are forced into it
    same = run(x[:4], [np.nan, -1.0, 1.0, 7.0])[0]
    want = run(x[:4], [0.0, 0.0, 0.99999994, 0.99999994])[0]
    np.testing.assert_array_equal(same, want)


def test_rows_with_infinities_nan_and_masks():
    rng = np.random.default_rng(6)
    V, low = 5000, np.finfo(np.float32).min
    x = head_like(rng, 12, V)
    x[0] = -np.inf                                                # nothing left
    x[1] = np.nan
    x[2] = -np.inf
    x[2, 777] = -1e30                                             # one token
    x[3, 100:4900] = -np.inf
    x[4, ::2] = np.nan
    x[5, [5, 4000]] = np.inf                                      # only these two
    x[6] = low                                                    # all alike, at the lowest value
    x[7] = low
    x[7, 4321] = 0.0
    x[8, 200:] = low
    x[9] = -0.0
    x[9, ::3] = 0.0                                               # the zeros are equal
    x[10] = 1e30
    x[10, 17] = np.float32(1.0000001e30)
    x[11] = np.where(np.arange(V) % 2, np.float32(3e38), np.float32(-3e38))
    for kw in ({}, dict(top_k=[3] * 12), dict(top_p=[0.6] * 12), dict(top_k=[7] * 12, top_p=[0.5] * 12, min_p=[0.1] * 12)):
        for dtype in ("f32", "bf16"):
            if dtype == "bf16":
                y = np.where(np.abs(x) > 3e38, np.copysign(3.0e38, x), x).astype(np.float32)
                y[~np.isfinite(x)] = x[~np.isfinite(x)]
            else:
                y = x
            token, prob = check(y, rng.random(12, np.float32), dtype, **kw)
            assert token[0] == token[1] == -1 and prob[0] == prob[1] == 0 and token[2] == 777 and token[5] in (5, 4000)


def test_settings_at_their_edges():
    rng = np.random.default_rng(7)
    M, V = 10, 3000
    x = head_like(rng, M, V)
    u = rng.random(M, np.float32)
    inf, nan = np.inf, np.nan
    check(x, u, temperature=[0.0, -1.0, 2.0 ** -11, 2.0 ** -10, 0.01, 50.0, 1e20, inf, 1e38, nan])
    check(x, u, top_p=[0.0, -1.0, 1e-30, 1.0, 2.0, 0.9999999, inf, 0.5, 1e-3, 0.999])
    check(x, u, min_p=[0.0, -1.0, 1e-30, 1.0, 2.0, 0.9999999, inf, 0.5, 1e-3, nan])
    check(x, u, top_k=[0, -5, 1, 2, 2999, 3000, 2 ** 31 - 1, -2 ** 31, 1024, 5][:4] + [3000, 3001, 2 ** 31 - 1, -2 ** 31, 1024, 5])


def test_a_top_k_out_of_range_is_forced_and_reported():
    lib, rng = H.sx(), np.random.default_rng(8)
    x = head_like(rng, 3, 9000)
    u = rng.random(3, np.float32)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.specexit_set_dev_status(word)
    try:
        token, prob = run(x, u, top_k=[5, 2000, 9000], flags=lib.FLAG_VALIDATE)
        assert int(word.item()) == lib.STATUS_BAD_SETTING
        word.zero_()
        want, _ = run(x, u, top_k=[5, 1024, 0], flags=lib.FLAG_VALIDATE)
        assert int(word.item()) == 0
        np.testing.assert_array_equal(token, want)
    finally:
        lib.specexit_set_dev_status(None)


def test_a_row_does_not_depend_on_its_neighbours():
    """Launches of other shapes cut a row into other chunks: the same bits."""
    rng = np.random.default_rng(9)
    V = 50000
    x, u = head_like(rng, 40, V), rng.random(40, np.float32)
    kw = lambda n: dict(temperature=[0.8] * n, top_p=[0.93] * n)
    token, prob = run(x, u, **kw(40))
    for rows in (slice(0, 1), slice(3, 7), slice(10, 40)):
        t, p = run(x[rows], u[rows], **kw(len(u[rows])))
        np.testing.assert_array_equal(t, token[rows])
        np.testing.assert_array_equal(p, prob[rows])


def test_replays_on_a_stream_of_its_own():
    lib, rng = H.sx(), np.random.default_rng(10)
    M, V = 9, 32003
    x = torch.from_numpy(head_like(rng, M, V)).cuda()
    u = torch.from_numpy(rng.random(M, np.float32)).cuda()
    p, k = torch.full((3,), 0.9, device="cuda"), torch.tensor([0, 50, 0], dtype=torch.int32, device="cuda")
    ws = H.workspace(lib.specexit_sample_workspace_bytes(lib.F32, M, V))
    out = [torch.empty(M, dtype=torch.int32, device="cuda") for _ in range(2)]
    call = lambda o, st: lib.specexit_sample(lib.F32, M, V, x, u, o, None, top_p=p, top_k=k, rows_per_seq=3, workspace=ws, stream=st)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        call(out[0], st)
        torch.cuda.synchronize()
        lib.specexit_graph_begin(st)
        call(out[1], st)
        graph = lib.specexit_graph_end(st)
        try:
            for rep in range(3):
                u.copy_(torch.rand(M, device="cuda"))
                ws.fill_(255)
                lib.specexit_graph_launch(graph, st)
                torch.cuda.synchronize()
                got = out[1].clone()
                call(out[0], st)
                torch.cuda.synchronize()
                assert torch.equal(out[0], got), rep
        finally:
            lib.specexit_graph_destroy(graph)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lists_of_every_length(dtype):
    """The tokens that a border lies among: fewer than the threads that compare them pair by pair, as many, more; with ties in bf16."""
    rng = np.random.default_rng(31)
    ks = [1, 2, 31, 63, 64, 65, 120, 126, 127, 128, 129, 130, 255, 256, 257, 511, 512, 513, 1000, 1024]
    ps = [1.0, 0.9, 0.3, 0.0]
    kw = dict(top_k=np.repeat(ks, len(ps)), top_p=np.tile(ps, len(ks)))
    M = len(kw["top_k"])
    x = (rng.standard_normal((M, 3001)) * 2).astype(np.float32)
    check(x, rng.random(M).astype(np.float32), dtype, **kw)


def test_min_p_inside_and_outside_the_nucleus():
    rng = np.random.default_rng(32)
    M = 16
    x = head_like(rng, M, 32003)
    check(x, rng.random(M).astype(np.float32), temperature=[0.6, 1.3] * 8, top_p=[0.9999, 0.9999, 0.5, 0.5] * 4,
          min_p=[0.3, 1e-6, 0.9, 1e-3, 1.0, 1e-9, 0.01, 0.0] * 2)


def test_logits_far_from_zero():
    """Large logits of both signs, up to where their own spacing is several nats, with and without borders."""
    rng = np.random.default_rng(33)
    V = 700
    tops = [3.2e7, 3.3554e7, 3.36e7, 1e9, -3.2e7, -3.35539e7, -3.3556e7, -3.4e7, -1e9]
    x = np.stack([t - 4.0 * rng.integers(0, 10, V) for t in tops] * 4).astype(np.float32)
    n = len(tops)
    kw = dict(top_k=[0] * n + [20] * n + [0] * n + [300] * n, top_p=[1.0] * n + [1.0] * n + [0.9] * n + [0.8] * n)
    check(x, rng.random(len(x)).astype(np.float32), **kw)
    kw["temperature"] = [0.5] * n + [2.0] * n + [8.0] * n + [20.0] * n
    check(x, rng.random(len(x)).astype(np.float32), **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sd", [1e-4, 0.01, 0.1, 0.4])
def test_flat_rows_of_a_long_vocabulary(dtype, sd):
    """More tokens than 2^16 close together: sums of a bin, bins of their width, borders among thousands; with an offset, and with one stretch
    of the row lower, higher, or closer together than the rest."""
    rng = np.random.default_rng(34)
    V = 200003
    x = (rng.standard_normal((6, V)) * sd).astype(np.float32)
    x[1] += 300.0
    x[2, 60000:90000] -= 5.0
    x[3, 150000:] += 7.0
    x[4, :33000] *= 0.001
    x[5, 70000:140000] = -1e30
    x[5, 3] = 4.0
    for kw in (dict(top_p=[0.9]), dict(top_k=[1000], top_p=[0.8]), dict(top_p=[0.3], min_p=[0.9])):
        check(x, rng.random(6).astype(np.float32), dtype, per=6, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_equal_logits(dtype):
    """Rows of zeros (a padded batch), of another number, with tokens ruled out, or with one other token: the borders go by index."""
    rng = np.random.default_rng(35)
    V = 70001
    x = np.zeros((7, V), np.float32)
    x[1] = -417.25
    x[2, ::3] = -np.inf
    x[3, 20000:60000] = -1e9
    x[4, 33333] = 1.0
    x[5] = 2.0 ** 20
    x[6, 5:] = np.nan
    for kw in (dict(), dict(top_p=[0.9]), dict(top_p=[0.0]), dict(top_k=[1000]), dict(top_k=[77], top_p=[0.5]), dict(min_p=[1.0]),
               dict(temperature=[0.0]), dict(temperature=[3.0], top_p=[0.25], min_p=[0.5])):
        u = rng.random(7).astype(np.float32)
        u[:2] = 0.0, np.float32(1) - np.float32(2.0 ** -24)
        check(x, u, dtype, per=7, **kw)


@pytest.mark.parametrize("sd", [0.003, 0.3, 3.0])
def test_offsets_and_odd_temperatures(sd):
    """Around 2^20 temperatures the bins end; in front of that a logit times the bins per logit is rounded to whole bins."""
    rng = np.random.default_rng(36)
    V = 30011
    tops = [0.0, 999.0, -1000.0, 7e4, 6.6e5, 7.3e5, 7.4e5, -6.9e5, -7.4e5, 3e6]
    x = (np.array(tops)[:, None] + rng.standard_normal((len(tops), V)) * sd).astype(np.float32)
    n = len(tops)
    for T in (0.7, 1.1):
        u = rng.random(n).astype(np.float32)
        check(x, u, temperature=[T] * n, top_p=[0.9, 0.5] * (n // 2))
        check(x, u, temperature=[T] * n, top_k=[100] * n, top_p=[0.95] * n)
