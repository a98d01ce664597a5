"""Sizes and argument checks of the 8-bit cache's and the sampling calls that a program meets as its batch changes (no GPU work)."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_24248_amd", "libspecexit.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libspecexit.so not built")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V", [1, 700, 5000, 32003, 128259, 151936, 262144])
def test_a_sampling_workspace_serves_every_smaller_batch(V, dtype):
    from paper_2509_24248_amd import binding as sx
    last = 0
    for M in list(range(1, 1100)) + [2047, 2048, 4096, 65535]:
        need = sx.specexit_sample_workspace_bytes(dtype, M, V)
        assert need >= last > 0 or M == 1, (M, need, last)
        last = need


def test_a_sampling_workspace_serves_every_smaller_vocabulary():
    from paper_2509_24248_amd import binding as sx
    for M in (1, 7, 30, 144, 600):
        last = 0
        for V in range(1, 262145, 509):
            need = sx.specexit_sample_workspace_bytes(0, M, V)
            assert need >= last, (M, V, need, last)
            last = need


def test_calls_at_the_edge_of_a_launch_are_refused():
    """2^24 workgroups of 256 threads are 2^32 threads, one more than a launch takes."""
    import test_quant_abi_cpu as abi
    from paper_2509_24248_amd import binding as sx
    one = abi.view(n_kv_heads=1)
    for T in (16 * ((1 << 25) - 1), 16 * (1 << 25)):                    # 2^26 - 2 and 2^26 waves
        abi.refused(sx, abi.write(sx, one, B=1, T=T, stride=128), sx.EUNSUPPORTED, "more than one call takes")
    for B, heads, layers in ((2731, 6143, 4), (1, 32768, 2048)):       # 2^26 - 1 and 2^26 + 1 waves
        abi.refused(sx, abi.compact(sx, abi.view(n_kv_heads=heads), layers=layers, B=B), sx.EUNSUPPORTED, "grid")
    # the kernel that merges has a wave per row
    wide = abi.view(n_kv_heads=512, l_max=64)
    assert sx.specexit_quant_verify_attn_workspace_bytes(wide, sx.BF16, 1024, 64, 1024) == 0 and "can split" in sx.last_error()
    assert sx.specexit_quant_verify_attn_workspace_bytes(wide, sx.BF16, 1023, 64, 1024) > 0


def rejected(text, call, *args, **kw):
    with pytest.raises(AssertionError, match=text):
        call(*args, **kw)


def test_the_binding_refuses_tensors_of_another_type_or_length():
    """A list of integers is 64 bits wide in torch, a list of numbers may be: read as 32 bits they are other settings."""
    import torch
    import test_quant_abi_cpu as abi
    from paper_2509_24248_amd import binding as sx

    class OnDevice(torch.Tensor):                  # (for the checks behind the one of where a tensor lies; no call here gets past them)
        is_cuda = True

    f, i = (lambda *s: torch.zeros(s).as_subclass(OnDevice)), (lambda *s: torch.zeros(s, dtype=torch.int32).as_subclass(OnDevice))
    on_host, host = "device-resident", lambda t: t.as_subclass(torch.Tensor)
    M, V = 6, 100
    base = dict(logits=f(M, V), u=f(M), token=i(M), prob=f(M), temperature=f(2), top_k=i(2), top_p=f(2), min_p=f(2), rows_per_seq=3)
    sample = lambda **kw: sx.specexit_sample(sx.F32, M, V, **{**base, **kw})
    for name in ("temperature", "top_k", "top_p", "min_p", "u", "token", "prob"):
        rejected(f"{name}: {on_host}", sample, **{name: host(base[name])})
    rejected("top_k must be torch.int32", sample, top_k=torch.tensor([20, 50]))
    for name in ("temperature", "top_p", "min_p", "u", "prob"):
        rejected(f"{name} must be torch.float32", sample, **{name: base[name].double()})
    rejected("token must be torch.int32", sample, token=torch.zeros(M, dtype=torch.int64))
    rejected("logits must be torch.float32", sample, logits=f(M, V).bfloat16())
    for name in ("temperature", "top_k", "top_p", "min_p"):
        rejected(f"{name} has 1 values, 2 are read", sample, **{name: base[name][:1]})
    rejected("u has 5 values, 6", sample, u=f(5))

    kv, B, T = abi.view(n_kv_heads=2, head_dim=64), 2, 3
    rows = f(B, T, 2, 64).bfloat16()
    write = lambda k=rows, v=rows, pos=i(B), count=None: sx.specexit_quant_kv_write(kv, sx.BF16, B, T, k, v, pos, count)
    rejected("must be torch.bfloat16", write, k=rows.float(), v=rows.float())
    rejected("must be torch.bfloat16", write, v=rows.float())
    rejected("pos must be torch.int32", write, pos=torch.tensor([4, 5]))
    rejected("count has 1 values, 2", write, count=i(1))
    rejected(f"pos: {on_host}", write, pos=host(i(B)))

    base_a = dict(q=f(B, T, 4, 64), ctx_len=i(B), mask=i(B, T).long(), scale=1.0, out=f(B, T, 4, 64), workspace=None)
    attn = lambda **kw: sx.specexit_quant_verify_attn(kv, sx.F32, B, T, 4, **{**base_a, **kw})
    rejected("q must be torch.float32", attn, q=base_a["q"].half())
    rejected("out must be torch.float32", attn, out=base_a["out"].bfloat16())
    rejected("ctx_len must be torch.int32", attn, ctx_len=torch.tensor([4, 5]))
    rejected("mask must be torch.int64", attn, mask=torch.zeros(B, T, dtype=torch.int32))
    rejected("q has", attn, q=f(B, T, 3, 64))
    rejected(f"ctx_len: {on_host}", attn, ctx_len=host(i(B)))

    base_c = dict(ctx_len=i(B), accept_path=i(B, T), accept_len=i(B), last_node=i(B), block_hidden=f(B, T, 8), D=8, hidden_next=f(B, 8))
    compact = lambda **kw: sx.specexit_quant_kv_compact(kv, 1, 0, 0, B, T, dtype=sx.F32, **{**base_c, **kw})
    for name in ("ctx_len", "accept_path", "accept_len", "last_node"):
        rejected(f"{name} must be torch.int32", compact, **{name: base_c[name].long()})
        rejected(f"{name} has", compact, **{name: base_c[name][:1]})
    rejected("block_hidden must be torch.float32", compact, block_hidden=f(B, T, 8).double())
    rejected("hidden_next has 8 values, 16", compact, hidden_next=f(1, 8))
    rejected(f"accept_path: {on_host}", compact, accept_path=host(i(B, T)))
