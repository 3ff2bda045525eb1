"""The gated block's gradients of more than 128 bf16 tokens and few features, where
the roundings of dG and dU as operands do not average out: each changes a value by
2^-8 of it at most (bf16 has eight significant bits)."""
import pytest
import torch

from tests.test_gpu_gated import CURVE, FUN, SUM, act64, call, make, near, project

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
@pytest.mark.parametrize("N,F,K", [(129, 1, 43), (404, 8, 588), (1120, 2, 1), (1147, 8, 8), (1531, 8, 1360), (821, 21, 19)])
def test_few_features(N, F, K, act):
    s, dH = make(N, F, K, "bf16", bias=N % 2 == 0)
    got = call(s, act, "bf16", dH)
    X, Wg, Wu, d = (t.double() for t in (s["X"], s["Wg"], s["Wu"], dH))
    (G, mG), (U, mU) = project(s["X"], s["Wg"], s["bg"]), project(s["X"], s["Wu"], s["bu"])
    a, slope = act64(G, act)
    dG, dU = d * U * slope, d * a
    # of the sums, the functions and their curvature, where relu' may fall on its other side, and of the rounding
    eU = d.abs() * (1.13 * SUM * mG + FUN * (1 + G.abs()))
    eG = d.abs() * (1.13 * SUM * mU + (U.abs() + SUM * mU) * (CURVE[act] * SUM * mG + FUN * (1 + G.abs())))
    if act == "relu":
        eG = eG + torch.where(G.abs() <= SUM * mG, d.abs() * (U.abs() + SUM * mU), torch.zeros_like(G))
    eG, eU = eG + 2.0 ** -8 * (dG.abs() + eG), eU + 2.0 ** -8 * (dU.abs() + eU)
    near(got["dX"], dG @ Wg + dU @ Wu, (eG + SUM * dG.abs()) @ Wg.abs() + (eU + SUM * dU.abs()) @ Wu.abs(), torch.bfloat16, 2)
    near(got["dWg"], dG.T @ X, (eG + SUM * dG.abs()).T @ X.abs(), torch.bfloat16, 2)
    near(got["dWu"], dU.T @ X, (eU + SUM * dU.abs()).T @ X.abs(), torch.bfloat16, 2)
