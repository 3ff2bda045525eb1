"""The operators of expert layers one behind the other in the same buffers, and the example
of a layer in 8 bits, forward and backward, at a single token,
a ragged batch and more experts than most tokens' choices reach: every result against double
precision, with the errors that rounding to 8 bits has."""
import importlib.util
import os

import pytest
import torch

import paper_2106_08846_gb300 as bsr

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("N,D,E,k", [(1, 256, 4, 2), (37, 256, 40, 2), (500, 768, 8, 2), (1000, 512, 3, 1)])
def test_layer_forward_and_backward(N, D, E, k):
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    layer = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(layer)
    errors, ms = layer.run(N, D, E, k)
    assert set(errors) == {"h_out", "z", "dx", "dh", "dweights", "dW", "dpost_w", "dpre_w", "dscale"}
    # Each value is off by at most 2^-4 of itself in e4m3 and 2^-3 in e5m2 (half a step); a sum of products
    # of independent values by no more of its 2-norm. y has two such operands, the gradients behind it the
    # difference that y's error makes in the norm (two more), dY in e5m2 and another operand: in quadrature
    # at most sqrt(4 * 2^-8 + 2^-6 + 2^-8), twice that where a factor is the other's derivative.
    for name, e in errors.items():
        assert e <= 2 * (5 * 2.0 ** -8 + 2.0 ** -6) ** 0.5, (name, e)
    assert ms > 0


def test_passes_one_behind_the_other_in_the_same_buffers():
    """Kernels start while the one before them still runs: passes over two inputs in turn, without a wait
    between them and in the same buffers, have the results that each has by itself."""
    N, k, E, K, M = 640, 3, 8, 256, 192
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    X = [normal(N, K).bfloat16() for _ in range(2)]
    experts = [torch.randint(0, E, (N, k), device="cuda", generator=g, dtype=torch.int32) for _ in range(2)]
    weights, bias = [normal(N, k) for _ in range(2)], normal(E, M)
    W = bsr.bsr_fp8_quantize(normal(E, M, K), tile=128)
    order = bsr.bsr_expert_order(experts[0], E, 128)
    Xs, Ys = (torch.zeros(order.rows, D, device="cuda", dtype=torch.bfloat16) for D in (K, M))
    A, At = (bsr.Fp8Matrix(*size) for size in ((order.rows, K), (K, order.rows)))
    Y = torch.zeros(201, N, M, device="cuda", dtype=torch.bfloat16)
    T = torch.zeros(201, E, K, K, device="cuda")
    back, dYs = torch.zeros(201, N, K, device="cuda", dtype=torch.bfloat16), torch.zeros_like(Ys)
    dweights = []

    def one(i, to):
        bsr.bsr_expert_order(experts[i], E, 128, order=order)
        bsr.bsr_expert_rows(X[i], order, Xs=Xs)
        bsr.bsr_fp8_quantize(Xs, form="both", used=order.used, out=(A, At))
        bsr.bsr_fp8_product(A, W, bias, offsets=order.offsets, Y=Ys)
        bsr.bsr_fp8_product(At, At, offsets=order.offsets, over="columns", Y=T[to])
        bsr.bsr_expert_sum(Ys, order, weights[i], Y=Y[to])
        dweights.append(bsr.bsr_expert_sum_backward(Ys, order, weights[i], Y[to], dYs=dYs)["dweights"])
        bsr.bsr_expert_sum(Xs, order, Y=back[to])

    want = []
    for i in range(2):
        one(i, 200)
        torch.cuda.synchronize()
        want.append((Y[200].clone(), T[200].clone(), back[200].clone(), dweights.pop()))
    for r in range(200):
        one(r % 2, r)
    torch.cuda.synchronize()
    for r in range(200):
        for got, right in zip((Y[r], T[r], back[r], dweights[r]), want[r % 2]):
            assert torch.equal(got, right), r
    assert not torch.equal(want[0][0], want[1][0])
