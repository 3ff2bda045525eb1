"""Infinite operands and gradients of the gated block: infinite results where every
term has the same sign, whatever the number of tokens and of parts."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr
from tests.test_gpu_gated import DT

pytestmark = pytest.mark.gpu
INF = float("inf")


def positive(N, F, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(N)
    rand = lambda *s: (torch.rand(*s, device="cuda", generator=g) + 0.5).to(DT[dtype])  # noqa: E731
    return rand(N, K), rand(F, K), rand(F, K), rand(N, F)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [2, 7, 40, 300])
def test_an_infinite_input(N, dtype):
    X, Wg, Wu, dH = positive(N, 72, 40, dtype)
    clean = bsr.bsr_gated(X, Wg, Wu, act="relu")
    X[1, 3] = INF
    H = bsr.bsr_gated(X, Wg, Wu, act="relu")
    assert (H[1] == INF).all() and torch.equal(torch.cat([H[:1], H[2:]]), torch.cat([clean[:1], clean[2:]]))
    got = bsr.bsr_gated_backward(X, Wg, Wu, None, None, dH, act="relu")   # dG = dH U, dU = dH G
    assert (got["dX"][1] == INF).all() and torch.isfinite(got["dX"][0]).all()
    assert (got["dWg"] == INF).all() and (got["dWu"] == INF).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 40, 128, 129, 300])
def test_an_infinite_gradient(N, dtype):
    X, Wg, Wu, dH = positive(N, 72, 40, dtype)
    bg, bu = torch.zeros(72, device="cuda"), torch.zeros(72, device="cuda")
    bg[5] = INF   # relu of it: dU
    got = bsr.bsr_gated_backward(X, Wg, Wu, bg, bu, dH, act="relu")
    assert (got["dX"] == INF).all() and got["dbu"][5] == INF
    rows = torch.arange(72, device="cuda") != 5
    assert (got["dWu"][5] == INF).all() and torch.isfinite(got["dWu"][rows]).all()
    assert torch.isfinite(got["dWg"]).all() and torch.isfinite(got["dbg"]).all()
