"""Argument checks of the operators beside the product that return before any
device work (no GPU needed)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2106_08846_gb300 import _build
    _build.build()
    import paper_2106_08846_gb300 as pkg
    return pkg.load()


def test_residual_norm_refusals(lib):
    from paper_2106_08846_gb300 import bsrlib as b
    d = ctypes.c_void_p(256)
    n = ctypes.c_size_t(7)

    def op(**k):
        c = b._ResidualNorm(64, 1, b.BSR_F32, b.BSR_F32, b.BSR_NORM_NONE, b.BSR_NORM_RMS, 1e-5, 1e-5, 1.0)
        for name, v in k.items():
            setattr(c, name, v)
        return c

    def forward(c, y=d, h=None, gate=None, h_out=None, z=d, N=4):
        return lib.bsr_residual_norm(c, y, h, gate, h_out, z, N, None)

    assert forward(None) == b.BSR_ERR_INVALID_ARG
    assert forward(op(), N=-1) == b.BSR_ERR_INVALID_ARG
    assert forward(op(D=0)) == forward(op(D=16385)) == b.BSR_ERR_SHAPE
    assert forward(op(block_dt=2)) == forward(op(stream_dt=b.BSR_BF16)) == b.BSR_ERR_UNSUPPORTED
    assert forward(op(post=3)) == forward(op(pre=-1)) == b.BSR_ERR_UNSUPPORTED
    assert forward(op(pre_eps=-1.0)) == forward(op(pre_eps=float("nan"))) == b.BSR_ERR_INVALID_ARG
    assert forward(op(post_w=256)) == b.BSR_ERR_INVALID_ARG            # a weight without its norm
    assert forward(op(gate_tokens=0), gate=d) == b.BSR_ERR_INVALID_ARG
    assert forward(op(), z=None) == forward(op(pre=0)) == b.BSR_ERR_INVALID_ARG
    assert forward(op(pre=0), z=None) == b.BSR_ERR_INVALID_ARG         # nothing to write
    assert forward(op(), y=None) == b.BSR_ERR_INVALID_ARG
    assert forward(op(), N=0) == b.BSR_OK
    assert lib.bsr_residual_norm_workspace(op(), 4, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_residual_norm_workspace(op(D=0), 4, ctypes.byref(n)) == b.BSR_ERR_SHAPE and n.value == 0
    assert lib.bsr_residual_norm_workspace(op(), 0, ctypes.byref(n)) == b.BSR_OK and n.value == 0

    def backward(c, y=d, h_out=d, gate=None, dh_out=None, dz=d, dy=None, dh=None, grads=None, N=4):
        return lib.bsr_residual_norm_backward(c, y, h_out, gate, dh_out, dz, dy, dh, grads, N, None, 1 << 40, None)

    assert backward(op(), y=None) == backward(op(), h_out=None) == backward(op(), dz=None) == b.BSR_ERR_INVALID_ARG
    assert backward(op(pre=0)) == b.BSR_ERR_INVALID_ARG                # dz without a norm
    for name in ("dgate", "dscale", "dpost_w", "dpost_b", "dpre_w", "dpre_b"):   # gradients of what is not there
        g = b._ResidualNormGrads()
        setattr(g, name, 256)
        assert backward(op(), grads=g) == b.BSR_ERR_INVALID_ARG


def test_gated_refusals(lib):
    from paper_2106_08846_gb300 import bsrlib as b
    d, e = ctypes.c_void_p(256), ctypes.c_void_p(1 << 30)
    n = ctypes.c_size_t(7)
    for N, F, K, dt, want in ((4, 64, 64, 2, b.BSR_ERR_UNSUPPORTED), (-1, 64, 64, 0, b.BSR_ERR_INVALID_ARG),
                              (4, 0, 64, 0, b.BSR_ERR_SHAPE), (4, 64, 0, 0, b.BSR_ERR_SHAPE),
                              (4, (1 << 20) + 1, 64, 0, b.BSR_ERR_SHAPE), (1 << 31, 64, 64, 0, b.BSR_ERR_SHAPE),
                              (1 << 30, 64, 1 << 20, 0, b.BSR_ERR_SHAPE)):
        assert lib.bsr_gated_workspace(N, F, K, dt, 0, ctypes.byref(n)) == want and n.value == 0
        assert lib.bsr_gated(d, d, d, None, None, e, N, F, K, dt, 0, d, 1 << 40, None) == want
        assert lib.bsr_gated_backward(d, d, d, None, None, d, e, None, None, None, None, N, F, K, dt, 0, d, 1 << 40, None) == want
    assert lib.bsr_gated_workspace(4, 64, 64, 0, 0, None) == b.BSR_ERR_INVALID_ARG
    for bad in (-1, 5):
        assert lib.bsr_gated(d, d, d, None, None, e, 4, 64, 64, 0, bad, d, 1 << 40, None) == b.BSR_ERR_UNSUPPORTED
    assert lib.bsr_gated(None, d, d, None, None, e, 4, 64, 64, 0, 0, d, 1 << 40, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_gated(None, None, None, None, None, None, 0, 64, 64, 0, 0, None, 0, None) == b.BSR_OK

    def backward(dWg=None, dWu=None, dbg=None, bg=None, dH=d):
        return lib.bsr_gated_backward(d, d, d, bg, None, dH, e, dWg, dWu, dbg, None, 4, 64, 64, 0, 0, d, 1 << 40, None)

    assert backward(dH=None) == backward(dWg=e) == backward(dWu=e) == backward(dbg=e) == b.BSR_ERR_INVALID_ARG
