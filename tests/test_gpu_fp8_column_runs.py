"""Products of runs of columns whose offsets are not multiples of 128: a run to the last
column is whole, one that ends inside a block of columns is NaN and reported; and of long runs in bf16."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300.bsrlib import BSR_ERR_INVALID_ARG, BSR_OK
from tests.test_gpu_fp8 import DT, guarded, near, normal, values

pytestmark = pytest.mark.gpu


def operands(N, M, R, tile):
    return (bsr.bsr_fp8_quantize(normal(R, N, wide=1.0), 1, "e5m2", "columns"),
            bsr.bsr_fp8_quantize(normal(R, M, seed=1), tile, form="columns"))


def product(a, b, at, Y):
    return bsr.bsr_fp8_product(a, b, offsets=torch.tensor(at, dtype=torch.int32, device="cuda"), over="columns", Y=Y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("R,at", [(2000, [0, 2000]), (300, [0, 128, 300]), (77, [0, 77, 77]), (1300, [0, 0, 1300, 1300, 2 ** 31 - 1])])
def test_a_run_to_the_last_column(R, at, tile, dtype):
    N, M = 130, 192
    a, b = operands(N, M, R, tile)
    buf, Y = guarded(dtype, len(at) - 1, N, M)
    product(a, b, at, Y)
    A, B = values(a), values(b)
    for e in range(len(at) - 1):
        near(Y[e], A[:, at[e]:at[e + 1]], B[:, at[e]:at[e + 1]])
    assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()
    assert bsr.bsr_check_status() == BSR_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("R,at,bad", [(640, [0, 100, 256, 640], (0, 1)), (640, [0, 128, 384, 639], (2,)), (1500, [1, 128, 1500], (0,)),
                                      (2600, [0, 1280, 2432, 2599, 2600], (2, 3)), (300, [64, 64, 128], (0, 1))])
def test_a_run_that_ends_inside_a_block(R, at, bad, tile, dtype):
    N, M = 130, 192
    a, b = operands(N, M, R, tile)
    buf, Y = guarded(dtype, len(at) - 1, N, M)
    product(a, b, at, Y)
    assert bsr.bsr_check_status() == BSR_ERR_INVALID_ARG
    assert bsr.bsr_check_status() == BSR_OK   # (cleared)
    A, B = values(a), values(b)
    for e in range(len(at) - 1):
        if e in bad:
            assert Y[e].isnan().all()
        else:
            near(Y[e], A[:, at[e]:at[e + 1]], B[:, at[e]:at[e + 1]])
    assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()


@pytest.mark.parametrize("align", [1, 16])
def test_gradients_of_runs_that_are_not_aligned_for_them(align):
    """The weights' gradients by an order whose runs start anywhere: none is a sum over other tokens than its expert's."""
    N, k, E, K, M = 500, 2, 6, 160, 64
    experts = torch.randint(0, E, (N, k), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(2))
    order = bsr.bsr_expert_order(experts, E, align)
    x = bsr.bsr_fp8_quantize(bsr.bsr_expert_rows(normal(N, K), order), form="columns", used=order.used)
    d = bsr.bsr_fp8_quantize(bsr.bsr_expert_rows(normal(N, M), order), form="columns", used=order.used)
    dW = bsr.bsr_fp8_product(d, x, offsets=order.offsets, over="columns", dtype=torch.float32)
    at = order.offsets.tolist()
    inside = [o % 128 != 0 and o < order.rows for o in at]
    assert any(inside)
    for e in range(E):
        if inside[e] or inside[e + 1]:
            assert dW[e].isnan().all()
        else:
            near(dW[e], values(d)[:, at[e]:at[e + 1]], values(x)[:, at[e]:at[e + 1]])
    assert bsr.bsr_check_status() == BSR_ERR_INVALID_ARG


@pytest.mark.parametrize("M,tile", [(192, 128), (320, 128), (320, 1), (77, 128)])   # straight from tensor memory, or through shared memory
@pytest.mark.parametrize("N,R,at", [(70, 16512, [0, 16512]), (130, 17000, [0, 0, 256, 1408, 1408, 17000]), (300, 40000, [0, 18560, 18560, 39936, 40000]),
                                    (600, 20000, [128, 19200])])
def test_drained_sums_with_bf16_results(N, R, at, M, tile):
    """More than 128 blocks of columns, of runs that are empty, short, longer than that and no multiples
    of the eight blocks of a drained sum: bf16 results are those in fp32, rounded once."""
    a, b = operands(N, M, R, tile)
    E = len(at) - 1
    buf, Y = guarded("bf16", E, N, M)
    product(a, b, at, Y)
    wide = torch.full((E, N, M), 7.0, device="cuda")
    product(a, b, at, wide)
    assert torch.equal(Y, wide.to(torch.bfloat16))
    A, B = values(a), values(b)
    for e in range(E):
        near(Y[e], A[:, at[e]:at[e + 1]], B[:, at[e]:at[e + 1]])
        near(wide[e], A[:, at[e]:at[e + 1]], B[:, at[e]:at[e + 1]])
    assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()
    assert bsr.bsr_check_status() == BSR_OK
