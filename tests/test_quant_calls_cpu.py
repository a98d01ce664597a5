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
