"""fp32 products of the gated block out of bf16 parts: single products, in which
nothing averages out, against 64 bits."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr

pytestmark = pytest.mark.gpu
# what the three smallest of nine part products hold, 2^-24; the additions of the others,
# whose last one drops less than 2^-23 and the ones before it 2^-8 of that
ONE = 2.0 ** -22


def values(n, m, seed, spread=20.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.rand(n, m, device="cuda", generator=g) + 1.0   # all 24 bits
    x *= torch.exp2(torch.randint(-int(spread), int(spread), (n, m), device="cuda", generator=g).float())
    return x * torch.sign(torch.rand(n, m, device="cuda", generator=g) - 0.5)


def exact(x, w):
    return x.double() @ w.double().T


@pytest.mark.parametrize("K", [1, 4])
@pytest.mark.parametrize("N", [1, 2, 3, 8, 9, 17, 32])
def test_few_tokens(N, K):
    """U = x w, with one column of K that is not zero, where act(G) is 1."""
    X, W, one = torch.zeros(N, K, device="cuda"), torch.zeros(4096, K, device="cuda"), torch.ones(4096, device="cuda")
    X[:, K - 1:], W[:, K - 1:] = values(N, 1, N), values(4096, 1, 7)
    H = bsr.bsr_gated(X, torch.zeros_like(W), W, one, None, act="relu")
    want = exact(X, W)
    err = ((H.double() - want).abs() / want.abs())
    assert float(err.max()) <= ONE, float(err.max())


@pytest.mark.parametrize("N", [33, 300])
def test_more_tokens(N):
    X, W, one = values(N, 1, N), values(520, 1, 7), torch.ones(520, device="cuda")
    H = bsr.bsr_gated(X, torch.zeros_like(W), W, one, None, act="relu")
    want = exact(X, W)
    err = ((H.double() - want).abs() / want.abs())
    assert float(err.max()) <= ONE, float(err.max())


@pytest.mark.parametrize("N", [1, 33, 300])
def test_gradients(N):
    """F = 1, Wg = 0 and G = 1: dU = dH, dX = dH Wu; of one token dWu = dH X."""
    X, Wu, one = values(N, 200, N), values(1, 200, 5), torch.ones(1, device="cuda")
    dH = values(N, 1, 3)
    got = bsr.bsr_gated_backward(X, torch.zeros_like(Wu), Wu, one, None, dH, act="relu")
    pairs = [(got["dX"], exact(dH, Wu.T))] + ([(got["dWu"], exact(dH, X.T))] if N == 1 else [])
    for x, want in pairs:
        err = ((x.double() - want).abs() / want.abs())
        assert torch.isfinite(x).all() and float(err.max()) <= ONE, float(err.max())


@pytest.mark.parametrize("N", [3, 20, 40])
def test_large_and_infinite_values(N):
    big = torch.finfo(torch.float32).max
    X = torch.tensor([[big, 0.0, 0.0], [-big, 0.0, 0.0], [float("inf"), 0.0, 0.0]], device="cuda").repeat(-(-N // 3), 1)[:N].contiguous()
    W, one = torch.zeros(8, 3, device="cuda"), torch.ones(8, device="cuda")
    W[:, 0] = 0.75
    H = bsr.bsr_gated(X, torch.zeros_like(W), W, one, None, act="relu").double()   # (0 x inf: G of the third row is NaN)
    for n in range(N):
        if n % 3 == 2:
            assert not torch.isfinite(H[n]).any()
        else:
            assert ((H[n] - 0.75 * X[n, 0].double()).abs() <= ONE * big).all()
