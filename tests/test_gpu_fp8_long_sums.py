"""Sums over many columns that one accumulator takes as a whole, or that are drained: what
the accumulators cut off, always towards zero, does not grow with the columns."""
import ctypes

import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300 import bsrlib
from tests.test_gpu_fp8 import DT, U, normal, values

pytestmark = pytest.mark.gpu
N, M = 4864, 1024   # 76 tiles of 256 x 256, one for each pair of SMs: sums are not split


def operands(K, tile, sign=True):
    x, w = normal(N, K), normal(M, K, seed=1)
    a, b = (x.abs(), w.abs()) if sign else (x, w)
    return bsr.bsr_fp8_quantize(a.to(torch.bfloat16)), bsr.bsr_fp8_quantize(b.to(torch.bfloat16), tile)


def is_whole(a, b, dtype):
    n = ctypes.c_size_t(1)
    assert bsr.load().bsr_fp8_product_workspace(a._c, b._c, bsrlib._DT[dtype], 0, 0, ctypes.byref(n)) == bsrlib.BSR_OK
    return n.value == 0


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("K", [1024, 1152, 16384, 16512, 40000])
def test_of_one_sign(K, tile):
    a, b = operands(K, tile)
    assert is_whole(a, b, torch.float32)
    Y = bsr.bsr_fp8_product(a, b, dtype=torch.float32)
    want = values(a) @ values(b).T
    off = (Y.double() - want) / want
    # An accumulator takes 1024 columns, 32 at a time, and loses at most 2^-23 of the sum with each (64 U); its
    # addition to those before is rounded.
    assert float(off.abs().max()) <= (64 + K / 1024) * U
    # What is cut off is half of that on average, of a sum that grows: 2^-24 times 1 / 32, 2 / 32, ... 32 / 32 of it (2.9 U
    # were measured). A sum that is not drained loses 160 U at 16384 columns.
    assert abs(float(off.mean())) <= 16.5 * U, float(off.mean()) / U

    Yb = bsr.bsr_fp8_product(a, b)
    # bf16: up to 16384 columns in one accumulator, 2^-14 of them at most; more are drained as fp32 results are
    if K > 16384:
        assert torch.equal(Yb, Y.to(torch.bfloat16))
    assert float(((Yb.double() - want) / want).abs().max()) <= 2.0 ** -8 + 2.0 ** -14
    assert bsr.bsr_check_status() == bsrlib.BSR_OK


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("K", [16512, 20000])
def test_drained_sums_with_bf16_results(K, tile):
    a, b = operands(K, tile, False)
    assert is_whole(a, b, torch.bfloat16)
    v = normal(M, seed=2)
    Y = bsr.bsr_fp8_product(a, b, v, dtype=torch.float32)
    assert torch.equal(bsr.bsr_fp8_product(a, b, v), Y.to(torch.bfloat16))
    A, B = values(a), values(b)
    size = A.abs() @ B.abs().T + v.double().abs()
    # as above, of a sum that may be as large as all its terms; then the bias
    assert ((Y.double() - (A @ B.T + v.double())).abs() <= (64 + K / 1024 + 1) * U * size).all()
    assert bsr.bsr_check_status() == bsrlib.BSR_OK
