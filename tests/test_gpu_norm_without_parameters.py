"""bsr_residual_norm and its backward pass with norms that have no weights, scale
or gate, where a row does not fill the threads that hold it: every pair of norms
against the definitions in 64 bits."""
import pytest

from tests.test_gpu_residual_norm import TYPES, check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block,stream", TYPES)
@pytest.mark.parametrize("D,bias", [(1, False), (64, False), (64, True), (100, True), (320, False), (1193, False), (4104, False),
                                    (4104, True)])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
def test_every_pair_of_norms(post, pre, D, bias, block, stream):
    s, p = make(16, D, block, stream, post, pre, weight=False, bias=bias)
    if s["dz"] is not None:
        s["dz"] += 0.5   # (a mean, which the LayerNorm's gradient takes out)
    check_forward(s, p)
    check_backward(s, p)
