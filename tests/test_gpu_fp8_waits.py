"""The 8-bit product's bounded waits: a load that never comes ends in a reported
timeout and a usable context, and a limit does not run while an earlier kernel
does."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300.bsrlib import BSR_ERR_TIMEOUT, BSR_OK
from tests.test_gpu_fp8 import near, normal, values

pytestmark = pytest.mark.gpu


def operands(N, M, K, tile):
    return bsr.bsr_fp8_quantize(normal(N, K)), bsr.bsr_fp8_quantize(normal(M, K, seed=1), tile)


# one tile, several a pair, sums that are split, drained ones, results through shared memory
@pytest.mark.parametrize("N,M,K,tile,dtype", [(300, 512, 768, 128, torch.bfloat16), (6000, 4096, 1024, 128, torch.bfloat16),
                                              (200, 1000, 4096, 1, torch.bfloat16), (3000, 2050, 2048, 1, torch.float32),
                                              (5000, 1024, 4096, 128, torch.float32)])
@pytest.mark.parametrize("step", [0, 3, 5])
def test_a_load_that_never_comes(N, M, K, tile, dtype, step, monkeypatch):
    a, b = operands(N, M, K, tile)
    offsets = torch.tensor([0, N // 2, N], dtype=torch.int32, device="cuda")
    two = bsr.bsr_fp8_quantize(normal(2, M, K, seed=2), tile)
    assert bsr.bsr_check_status() == BSR_OK
    monkeypatch.setenv("BSR_WAIT_LIMIT_NS", "2000000")
    monkeypatch.setenv("BSR_TEST_STALL_CHUNK", str(step))
    bsr.bsr_fp8_product(a, b, dtype=dtype)
    assert bsr.bsr_check_status() == BSR_ERR_TIMEOUT
    assert bsr.bsr_check_status() == BSR_OK   # (cleared)
    bsr.bsr_fp8_product(a, two, offsets=offsets, dtype=dtype)
    assert bsr.bsr_check_status() == BSR_ERR_TIMEOUT
    monkeypatch.delenv("BSR_TEST_STALL_CHUNK")
    monkeypatch.delenv("BSR_WAIT_LIMIT_NS")
    near(bsr.bsr_fp8_product(a, b, dtype=dtype), values(a), values(b))
    assert bsr.bsr_check_status() == BSR_OK


def test_a_limit_does_not_run_while_the_previous_kernel_does(monkeypatch):
    a, b = operands(600, 1024, 1024, 128)
    x = torch.full((8192, 8192), 1e-3, device="cuda")
    monkeypatch.setenv("BSR_WAIT_LIMIT_NS", "1000000")
    for _ in range(2):
        x.copy_(x @ x * 1e-3)   # many times the limit
        Y = bsr.bsr_fp8_product(a, b, dtype=torch.float32)
        assert bsr.bsr_check_status() == BSR_OK
    near(Y, values(a), values(b))


def test_the_gated_block_and_the_product_in_turn():
    """Kernels of two files that take all of tensor memory, on two streams."""
    a, b = operands(2000, 1024, 1024, 128)
    X, Wg, Wu = (normal(r, 1024, seed=r).to(torch.bfloat16) for r in (2001, 1024, 1025))
    Wu = Wu[:1024].contiguous()
    want, H = bsr.bsr_fp8_product(a, b), bsr.bsr_gated(X, Wg, Wu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        got = bsr.bsr_fp8_product(a, b, stream=side)
        h = bsr.bsr_gated(X, Wg, Wu)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(h, H)
    assert bsr.bsr_check_status() == BSR_OK
