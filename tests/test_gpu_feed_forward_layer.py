"""The example of the operators used together, at a small size, a ragged one and
a single token: every result against double precision."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("N,D,F", [(1, 256, 512), (37, 256, 512), (500, 768, 1024)])
def test_layer_forward_and_backward(N, D, F):
    spec = importlib.util.spec_from_file_location("feed_forward_layer", os.path.join(ROOT, "examples", "feed_forward_layer.py"))
    layer = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(layer)
    errors, ms = layer.run(N, D, F)
    assert set(errors) == {"h_out", "z", "da", "dh", "dWg", "dWu"} | {f"d{n}{k}" for n in ("post_w", "pre_w", "scale") for k in (0, 1)}
    # bf16 values are rounded up to six times on the way (2^-8 at most each, in quadrature half of it on average)
    for name, e in errors.items():
        assert e <= 6 ** 0.5 * 2.0 ** -8, (name, e)
    assert ms > 0
