"""The gated block's bf16 sums over very many tokens or features: sums of one sign,
from which an accumulator that drops bits takes more with every term."""
import math

import pytest
import torch

import paper_2106_08846_gb300 as bsr
from paper_2106_08846_gb300.bsrlib import BSR_ERR_TIMEOUT, BSR_OK
from tests.test_gpu_gated import check_backward

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def positive(g, *shape):
    return torch.rand(*shape, device="cuda", generator=g) + 0.5


@pytest.mark.parametrize("N", [65536, 1 << 20, (1 << 19) + 100])
def test_weights_of_many_tokens(N):
    F = K = 64
    g = torch.Generator(device="cuda").manual_seed(N)
    X, dH = (positive(g, N, K) * positive(g, K)).to(BF16), (positive(g, N, F) * positive(g, F)).to(BF16)
    Wg, Wu = positive(g, F, K).to(BF16), positive(g, F, K).to(BF16)
    got = bsr.bsr_gated_backward(X, Wg, Wu, None, None, dH, act="relu")
    x, d = X.double(), dH.double()
    dU = d * (x @ Wg.double().T)
    dG = d * (x @ Wu.double().T)
    want = {"dWg": dG.T @ x, "dWu": dU.T @ x}
    for k, w in want.items():
        off = got[k].double() / w - 1
        # a 32nd of the most that one is rounded by, for what accumulators lose, and the mean of results' and operands' roundings, spread over an
        # octave and more by the factors above: at most 2^-9 each (2-norm), five times that of their mean
        assert abs(float(off.mean())) <= 2.0 ** -14 + 5 * 2.0 ** -9 / math.sqrt(off.numel()), (k, float(off.mean()))
        assert float(off.abs().max()) <= 2.0 ** -8 + 2.0 ** -10


def test_a_long_inner_sum():
    """dX, over 2 x 70000 features."""
    N, F, K = 64, 70000, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    X, dH = positive(g, N, K).to(BF16), (positive(g, N, F) * positive(g, N, 1)).to(BF16)
    Wg, Wu = ((positive(g, F, K) * positive(g, K)).to(BF16) for _ in range(2))
    dX = bsr.bsr_gated_backward(X, Wg, Wu, None, None, dH, act="relu")["dX"]
    x, d = X.double(), dH.double()
    want = (d * (x @ Wu.double().T)) @ Wg.double() + (d * (x @ Wg.double().T)) @ Wu.double()
    off = dX.double() / want - 1
    assert abs(float(off.mean())) <= 2.0 ** -14 + 5 * 2.0 ** -9 / math.sqrt(off.numel()), float(off.mean())
    assert float(off.abs().max()) <= 2.0 ** -8 + 2.0 ** -10


def long_rows(N, F, K):
    g = torch.Generator(device="cuda").manual_seed(N + K)
    X, (Wg, Wu) = (positive(g, N, K) * positive(g, N, 1)).to(BF16), ((positive(g, F, K) * positive(g, F, 1)).to(BF16) for _ in range(2))
    return X, Wg, Wu


@pytest.mark.parametrize("N,F,K", [(8, 512, 1 << 18), (40, 512, 1 << 18), (300, 100, 20000), (300, 100, 20003), (33, 64, 16385)])
def test_long_rows(N, F, K):
    X, Wg, Wu = long_rows(N, F, K)
    H = bsr.bsr_gated(X, Wg, Wu, act="relu")
    x = X.double()
    off = H.double() / ((x @ Wg.double().T) * (x @ Wu.double().T)) - 1
    assert abs(float(off.mean())) <= 2.0 ** -14 + 5 * 2.0 ** -9 / math.sqrt(off.numel()), float(off.mean())
    assert float(off.abs().max()) <= 2.0 ** -8 + 2.0 ** -10


@pytest.mark.parametrize("N,F,K", [(40, 64, 20000), (300, 72, 16390)])
def test_gradients_of_long_rows(N, F, K):
    """All of them to the bounds of any other size, the biases' in fp32 too."""
    X, Wg, Wu = long_rows(N, F, K)
    g = torch.Generator(device="cuda").manual_seed(3)
    s = dict(X=X, Wg=Wg / 128, Wu=Wu / 128, bg=positive(g, F), bu=positive(g, F))
    check_backward(s, positive(g, N, F).to(BF16), "relu", "bf16")


def test_a_load_that_never_comes_of_a_long_row(monkeypatch):
    X, Wg, Wu = long_rows(40, 96, 20000)
    assert bsr.bsr_check_status() == BSR_OK
    monkeypatch.setenv("BSR_WAIT_LIMIT_NS", "2000000")
    for step in (0, 20, 300):
        monkeypatch.setenv("BSR_TEST_STALL_CHUNK", str(step))
        bsr.bsr_gated(X, Wg, Wu)
        assert bsr.bsr_check_status() == BSR_ERR_TIMEOUT
    monkeypatch.delenv("BSR_TEST_STALL_CHUNK")
    monkeypatch.delenv("BSR_WAIT_LIMIT_NS")
    assert torch.isfinite(bsr.bsr_gated(X, Wg, Wu)).all() and bsr.bsr_check_status() == BSR_OK
