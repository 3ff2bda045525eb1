"""The gated block's bounded waits: a load that never comes ends in a reported
timeout and a usable context, and a limit does not run while an earlier kernel
does."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300.bsrlib import BSR_ERR_TIMEOUT, BSR_OK
from tests.test_gpu_gated import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,F,K,step", [(300, 512, 768, 0), (300, 512, 768, 3), (600, 4096, 1024, 5), (130, 64, 64, 0)])
def test_a_load_that_never_comes(N, F, K, step, dtype, monkeypatch):
    s, dH = make(N, F, K, dtype)
    assert bsr.bsr_check_status() == BSR_OK
    monkeypatch.setenv("BSR_WAIT_LIMIT_NS", "2000000")
    monkeypatch.setenv("BSR_TEST_STALL_CHUNK", str(step))
    bsr.bsr_gated(s["X"], s["Wg"], s["Wu"])
    assert bsr.bsr_check_status() == BSR_ERR_TIMEOUT
    assert bsr.bsr_check_status() == BSR_OK   # (cleared)
    bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], None, None, dH)
    assert bsr.bsr_check_status() == BSR_ERR_TIMEOUT
    monkeypatch.delenv("BSR_TEST_STALL_CHUNK")
    monkeypatch.delenv("BSR_WAIT_LIMIT_NS")
    check_forward(s, "silu", dtype)
    check_backward(s, dH, "silu", dtype)
    assert bsr.bsr_check_status() == BSR_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_limit_does_not_run_while_the_previous_kernel_does(dtype, monkeypatch):
    s, dH = make(600, 1024, 1024, dtype)
    a = torch.full((8192, 8192), 1e-3, device="cuda")
    monkeypatch.setenv("BSR_WAIT_LIMIT_NS", "1000000")
    for _ in range(2):
        a.copy_(a @ a * 1e-3)   # many times the limit
        H = bsr.bsr_gated(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"])
        bsr.bsr_gated_backward(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], dH)
        assert bsr.bsr_check_status() == BSR_OK
    assert torch.equal(H, check_forward(s, "silu", dtype))
