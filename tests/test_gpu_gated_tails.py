"""The gated block's activations where their values are small: errors relative to
the value. G is a bias and U is 1, so that both are exact."""
import math

import pytest
import torch

import paper_2106_08846_gb300 as bsr
from tests.test_gpu_gated import ACTS, DT

pytestmark = pytest.mark.gpu
# an activation in fp32: some 20 roundings at most; with the exponential for bf16 results:
# the rounding of its argument's product with 1 / ln 2, up to 2^7 times 2^-24, and as much
# of a square's
NEAR = {"f32": 2.0 ** -19, "bf16": 2.0 ** -15}


def on_a_grid(g, act, dtype, N):
    """H, dG and dU of one token (of N that are alike): act(g), act'(g), act(g)."""
    F, dt = g.numel(), DT[dtype]
    X, W, one = torch.zeros(N, 8, device="cuda", dtype=dt), torch.zeros(F, 8, device="cuda", dtype=dt), torch.ones(F, device="cuda")
    H = bsr.bsr_gated(X, W, W, g, one, act=act)
    assert torch.equal(H, H[:1].expand(N, F))
    got = bsr.bsr_gated_backward(X, W, W, g, one, torch.ones(N, F, device="cuda", dtype=dt), act=act)
    return H[0].double(), got["dbg"].double() / N, got["dbu"].double() / N


def close(got, want, size, rel):
    bad = (got - want).abs() > rel * size
    assert torch.isfinite(got).all() and not bad.any(), (int(bad.sum()), got[bad][:3], want[bad][:3], float(((got - want).abs() / size).max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 5, 64])
def test_gelu(N, dtype):
    g = torch.cat([torch.linspace(-12, -0.01, 900, device="cuda"), torch.linspace(0, 12, 124, device="cuda")])
    H, dG, dU = on_a_grid(g, "gelu", dtype, N)
    x = g.double()
    cdf, density = 0.5 * torch.special.erfc(-x / math.sqrt(2)), torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    rel = NEAR[dtype]
    close(H, x * cdf, x.abs() * cdf, rel + (2.0 ** -8 if dtype == "bf16" else 0.0))
    close(dU, x * cdf, x.abs() * cdf, rel)
    close(dG, cdf + x * density, cdf + x.abs() * density, rel)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 5, 64])
def test_sigmoid(N, dtype):
    g = torch.linspace(-80, 80, 1024, device="cuda")
    H, dG, dU = on_a_grid(g, "sigmoid", dtype, N)
    p, q = torch.sigmoid(g.double()), torch.sigmoid(-g.double())
    rel = NEAR[dtype]
    close(H, p, p, rel + (2.0 ** -8 if dtype == "bf16" else 0.0))
    close(dU, p, p, rel)
    close(dG, p * q, p * q, rel)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sigmoid_where_the_exponential_overflows(dtype):
    g = torch.tensor([-3e38, -1e4, -100.0, -89.0, 89.0, 100.0, 1e4, 3e38], device="cuda").repeat(8)
    H, dG, dU = on_a_grid(g, "sigmoid", dtype, 40)
    want = (g > 0).double()
    assert ((H - want).abs() <= 1e-37).all() and ((dU - want).abs() <= 1e-37).all() and (dG.abs() <= 1e-37).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N", [1, 40])
def test_gates_whose_square_overflows(N, act, dtype):
    """Where an activation is g, 0 or 1 and its slope 1 or 0."""
    g = torch.tensor([-3e38, -1e25, -2e19, -1e4, 1e4, 2e19, 1e25, 3e38], device="cuda").repeat(8)
    H, dG, dU = on_a_grid(g, act, dtype, N)
    x = g.double()
    value, slope = ((x > 0).double(), 0 * x) if act == "sigmoid" else (x.clamp(min=0), (x > 0).double())
    sums = torch.where(value * N > torch.finfo(torch.float32).max, float("inf"), value)   # (dU's sum may overflow)
    for got, want, rel in ((H, value, 2.0 ** -8), (dU, sums, 2.0 ** -19), (dG, slope, 2.0 ** -19)):
        assert ((got == want) | ((got - want).abs() <= rel * value + 1e-37)).all(), (got[:8], want[:8])
