"""The example of expert layers in 8 bits, forward and backward, at a single token,
a ragged batch and more experts than most tokens' choices reach: every result against double
precision, with the errors that rounding to 8 bits has."""
import importlib.util
import os

import pytest

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
