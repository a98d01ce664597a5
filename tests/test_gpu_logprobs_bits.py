"""GPU: which calls give a row's log probabilities, entropy and best alternatives to the same bits."""
import numpy as np
import pytest
import torch

from target_harness import DT
from test_gpu_logprobs import run

pytestmark = pytest.mark.gpu

ROWS_OF_WIDE_PARTS = 2048          # parts of 2048 logits a row, in all rows of a call, from which on rows are summed in such parts


def row_of(V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(V, generator=g) * 3).to(DT[dtype]).cuda()


def bits(got, r):
    return [np.ascontiguousarray(a[r]).view(np.uint32) for a in got]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [104, 1000, 2040, 2104, 20008, 151936])
def test_other_rows_of_the_call(dtype, V):
    """One row as the first, the last and one between, alone and on either side of the switch, ld a multiple of 16 bytes."""
    border = -(-ROWS_OF_WIDE_PARTS // -(-(V + 7) // 2048))
    row, tokens = row_of(V, dtype, V), [0, V // 2, V - 1]
    for sizes in ((1, 2, border - 1), (border, border + 1, 2 * border)):
        want = None
        for M in sizes:
            x = torch.randn((M, V), generator=torch.Generator(device="cuda").manual_seed(M), device="cuda").to(DT[dtype])
            at = sorted({0, M // 2, M - 1})
            x[at] = row
            got = run(x, V, np.tile(tokens, (M, 1)), 5, [0.7] * M, 1, dtype)
            for r in at:
                want = bits(got, r) if want is None else want
                for a, b in zip(bits(got, r), want):
                    assert np.array_equal(a, b), (M, r)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,M", [(3001, 40), (3001, 1100), (50003, 20), (50003, 90)])
def test_rows_that_begin_alike(dtype, V, M):
    """An odd row stride: of the same row everywhere, those as far behind a multiple of 16 bytes agree, whatever their number."""
    each = 16 // DT[dtype].itemsize
    row, ld = row_of(V, dtype, V + M), V + 2
    x = torch.zeros((M, ld), dtype=DT[dtype], device="cuda")
    assert x.data_ptr() % 16 == 0 and ld % 2 == 1
    x[:, :V] = row
    got = run(x, V, np.tile([0, V // 2, V - 1], (M, 1)), 5, None, 1, dtype)
    for r in range(each, M):
        for a, b in zip(bits(got, r), bits(got, r % each)):
            assert np.array_equal(a, b), r
    # (of another beginning they may differ: how many do)
    print(sum(any((a != b).any() for a, b in zip(bits(got, r), bits(got, 0))) for r in range(1, each)), "of", each - 1, "other beginnings differ", flush=True)
