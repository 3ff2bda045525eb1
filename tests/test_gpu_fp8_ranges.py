"""Products whose scales' product is no fp32 number (2^(128 ..) or below 2^-149) while the
results are: the scales are exponents, and nothing on the way overflows or vanishes."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr
from tests.test_gpu_fp8 import DT, U, normal, values

pytestmark = pytest.mark.gpu


def product(x, w, tile, dtype):
    a, b = bsr.bsr_fp8_quantize(x), bsr.bsr_fp8_quantize(w, tile)
    return bsr.bsr_fp8_product(a, b, dtype=DT[dtype]), values(a), values(b), a, b


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("ea,eb", [(64, 64), (70, 65), (100, 45), (119, 20), (20, 119)])
def test_large_scales(ea, eb, tile, dtype):
    """Each operand's largest value meets a zero of the other; the rest are its least (2^-9 of its scale)."""
    N, M, K = 40, 64, 256
    x, w = (torch.sign(normal(n, K, seed=s)) * 2.0 ** (e - 9) for n, s, e in ((N, 0, ea), (M, 1, eb)))
    x[:, 0::128], w[:, 0::128] = 448 * 2.0 ** ea, 0
    x[:, 1::128], w[:, 1::128] = 0, 448 * 2.0 ** eb
    Y, A, B, a, b = product(x, w, tile, dtype)
    assert (a.scale == 2.0 ** ea).all() and (b.scale == 2.0 ** eb).all()
    want = A @ B.T   # (whole numbers of at most 252, even, times 2^(ea + eb - 18): exact as long as fp32 has them, below 2^128)
    most = float((A.unsqueeze(1) * B).cumsum(2).abs().max())
    if most < 2.0 ** 128:
        assert torch.equal(Y.double(), want)
    else:   # 2^127 is the unit: every sum but 0 is 2^128 or more, and stays infinite (or NaN, of two infinities) once it is
        assert ea + eb - 18 == 127
        assert not torch.isfinite(Y[want != 0]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("ea,eb", [(-64, -63), (-80, -60), (-75, -75), (-126, -24), (-24, -126), (-126, -30)])
def test_small_scales(ea, eb, tile, dtype):
    N, M, K = 40, 64, 1024
    x, w = (normal(n, K, seed=s).abs() + 1 for n, s in ((N, 0), (M, 1)))
    x, w = (t * (448 / t.max()) for t in (x, w))
    x[:, ::128] = 448
    w[:, ::128] = 448
    Y, A, B, a, b = product(x * 2.0 ** ea, w * 2.0 ** eb, tile, dtype)
    assert (a.scale == 2.0 ** ea).all() and (b.scale == 2.0 ** eb).all()
    want = A @ B.T
    # 32 additions, each off by at most 2^-23 of the sum, or by the least fp32 value, then the rounding to the result's type
    bound = (64 * U + (2.0 ** -8 if dtype == "bf16" else U)) * want + 64 * 2.0 ** -149 + (2.0 ** -134 if dtype == "bf16" else 0)
    assert ((Y.double() - want).abs() <= bound).all(), float(((Y.double() - want).abs() / bound).max())
