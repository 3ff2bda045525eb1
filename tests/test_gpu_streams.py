"""Outputs that calls on another stream allocate themselves: memory that the
current stream still writes is not written before, and memory of an output that is
dropped at once is not handed out before the call's work is done."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def normal(*shape, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def norm_forward():
    y, h, w = normal(700, 768), normal(700, 768), normal(768)
    return lambda stream: dict(zip(("h_out", "z"), bsr.bsr_residual_norm(y, h, pre="rms", pre_w=w, stream=stream)))


def norm_backward():
    y, h, dh, dz, w, gate = normal(700, 768), normal(700, 768), normal(700, 768), normal(700, 768), normal(768), normal(7, 768)
    return lambda stream: bsr.bsr_residual_norm_backward(y, h, dh, dz, gate=gate, gate_tokens=100, pre="rms", pre_w=w,
                                                         stream=stream)


def gated(N):
    def make():
        X, Wg, Wu = normal(N, 768, dtype=BF16), normal(2048, 768, dtype=BF16), normal(2048, 768, dtype=BF16)
        return lambda stream: {"H": bsr.bsr_gated(X, Wg, Wu, stream=stream)}
    return make


def gated_backward():
    X, Wg, Wu = normal(300, 768, dtype=BF16), normal(2048, 768, dtype=BF16), normal(2048, 768, dtype=BF16)
    b, dH = normal(2048), normal(300, 2048, dtype=BF16)
    return lambda stream: bsr.bsr_gated_backward(X, Wg, Wu, b, b, dH, stream=stream)


def product():
    W, X = normal(768, 768), normal(700, 768)
    h = bsr.bsr_create(*bsr.bsr_from_dense(W, 16, 16), 16, 16, 768, 768)
    return lambda stream: {"Y": h.spmm(X, stream=stream)}


CALLS = [norm_forward, norm_backward, gated(6), gated(300), gated_backward, product]


def long_work():
    """Some milliseconds of the current stream."""
    a = torch.full((8192, 8192), 1e-3, device="cuda")
    for _ in range(3):
        a = a @ a * 1e-3


@pytest.mark.parametrize("make", CALLS)
def test_memory_that_the_current_stream_still_writes(make):
    call = make()
    want = {k: t.clone() for k, t in call(None).items()}
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty_like(t) for t in want.values()]
    places = {t.data_ptr() for t in old}
    long_work()
    for t in old:
        t.fill_(float("nan"))
    del t, old
    got = call(other)
    assert places & {t.data_ptr() for t in got.values()}   # (the allocator hands them out again)
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("make", CALLS)
def test_outputs_that_are_dropped_at_once(make):
    call = make()
    sizes = [t.shape for t in call(None).values()]
    types = [t.dtype for t in call(None).values()]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        long_work()
    call(other)
    new = [torch.full(n, 7.0, dtype=t, device="cuda") for n, t in zip(sizes, types)]
    torch.cuda.synchronize()
    for t in new:
        assert (t == 7).all()


def test_no_tokens_on_another_stream():
    other = torch.cuda.Stream()
    y, W, b = normal(0, 64), normal(32, 64), normal(32)
    h_out, z = bsr.bsr_residual_norm(y, y, pre="rms", stream=other)
    assert h_out.shape == z.shape == (0, 64)
    assert bsr.bsr_gated(y, W, W, stream=other).shape == (0, 32)
    got = bsr.bsr_gated_backward(y, W, W, b, b, normal(0, 32), stream=other)
    torch.cuda.synchronize()
    assert not got["dWg"].any() and not got["dbu"].any()


def test_a_stream_by_its_handle():
    call = gated(40)()
    want, other = call(None)["H"], torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = call(other.cuda_stream)["H"]
    other.synchronize()
    assert torch.equal(want, got)
    got = call(0)["H"]   # the default stream
    torch.cuda.synchronize()
    assert torch.equal(want, got)
