"""Argument checks of expert layers and 8-bit products that return before any
device work (no GPU needed)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2106_08846_gb300 import _build
    _build.build()
    import paper_2106_08846_gb300 as pkg
    return pkg.load()


def test_capacity(lib):
    from paper_2106_08846_gb300 import bsrlib as b
    n = ctypes.c_int64(7)
    for (N, k, E, align), want in {(0, 2, 8, 128): 0, (1, 2, 8, 1): 2, (1, 2, 8, 128): 256, (100, 4, 64, 1): 400,
                                   (100, 4, 64, 128): (400 + 64 * 127) // 128 * 128, (3, 1, 2, 7): 14}.items():
        assert lib.bsr_expert_capacity(N, k, E, align, ctypes.byref(n)) == b.BSR_OK and n.value == want
    for bad in ((-1, 2, 8, 1),):
        assert lib.bsr_expert_capacity(*bad, ctypes.byref(n)) == b.BSR_ERR_INVALID_ARG
    for bad in ((1, 0, 8, 1), (1, 65, 8, 1), (1, 2, 0, 1), (1, 2, 1025, 1), (1, 2, 8, 0), (1, 2, 8, 1025), (1 << 30, 1, 1, 1),
                ((1 << 30) - 1, 64, 1, 1)):
        assert lib.bsr_expert_capacity(*bad, ctypes.byref(n)) == b.BSR_ERR_SHAPE and n.value == 0
    assert lib.bsr_expert_capacity(1, 2, 8, 1, None) == b.BSR_ERR_INVALID_ARG


def test_expert_refusals(lib):
    from paper_2106_08846_gb300 import bsrlib as b
    d, e = ctypes.c_void_p(256), ctypes.c_void_p(1 << 30)

    def op(N=4, R=8, k=2, E=8, align=1, offsets=1 << 20, place=1 << 21, source=1 << 22):
        return b._Experts(N, R, k, E, align, offsets, place, source)

    assert lib.bsr_expert_order(None, d, None) == lib.bsr_expert_order(op(N=-1), d, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_order(op(), None, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_order(op(offsets=None), d, None) == lib.bsr_expert_order(op(place=None), d, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_order(op(R=7), d, None) == lib.bsr_expert_order(op(align=128), d, None) == b.BSR_ERR_CAPACITY
    for bad in (dict(k=0), dict(k=65), dict(E=0), dict(E=1025), dict(align=0), dict(R=1 << 31)):
        assert lib.bsr_expert_order(op(**bad), d, None) == b.BSR_ERR_SHAPE
        assert lib.bsr_expert_rows(op(**bad), d, e, 64, 0, None) == b.BSR_ERR_SHAPE
    for D, dt, want in ((0, 0, b.BSR_ERR_SHAPE), ((1 << 20) + 1, 0, b.BSR_ERR_SHAPE), (64, 2, b.BSR_ERR_UNSUPPORTED)):
        assert lib.bsr_expert_rows(op(), d, e, D, dt, None) == want
        assert lib.bsr_expert_sum(op(), d, None, e, D, dt, None) == want
        assert lib.bsr_expert_sum_backward(op(), d, d, d, e, None, D, dt, None) == want
    assert lib.bsr_expert_rows(op(), None, e, 64, 0, None) == lib.bsr_expert_rows(op(), d, None, 64, 0, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_sum(op(), None, None, e, 64, 0, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_sum_backward(op(), d, None, d, e, e, 64, 0, None) == b.BSR_ERR_INVALID_ARG   # dweights without weights
    assert lib.bsr_expert_sum_backward(op(), None, d, d, e, e, 64, 0, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_sum_backward(op(), d, d, None, e, None, 64, 0, None) == b.BSR_ERR_INVALID_ARG
    # overlaps and alignment are found before the device is asked
    assert lib.bsr_expert_rows(op(), d, ctypes.c_void_p(256 + 64), 64, 0, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_rows(op(), ctypes.c_void_p(260), e, 64, 0, None) == b.BSR_ERR_ALIGNMENT
    assert lib.bsr_expert_order(op(place=(1 << 20) + 4), d, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_expert_rows(op(N=0, R=0), None, None, 64, 0, None) == b.BSR_OK


def test_fp8_refusals(lib):
    from paper_2106_08846_gb300 import bsrlib as b
    n = ctypes.c_size_t(7)
    d, e, f = ctypes.c_void_p(256), ctypes.c_void_p(1 << 30), ctypes.c_void_p(1 << 32)

    def m(rows=64, cols=256, tile=1, type=0, batch=1, q=1 << 20, exponent=1 << 24, scale=1 << 27):
        return b._Fp8Matrix(batch, rows, cols, tile, type, q, exponent, scale)

    def quantize(rows=None, columns=None, x=d, dt=0, used=None):
        return lib.bsr_fp8_quantize(x, dt, rows, columns, used, None)

    assert quantize() == quantize(m(), x=None) == quantize(m(q=None)) == quantize(m(exponent=None)) == b.BSR_ERR_INVALID_ARG
    assert quantize(m(rows=-1)) == quantize(m(), m(rows=256, cols=-1)) == b.BSR_ERR_INVALID_ARG
    assert quantize(m(tile=64)) == quantize(m(type=2)) == quantize(m(), dt=2) == b.BSR_ERR_UNSUPPORTED
    for other in (m(rows=256, cols=65), m(rows=255, cols=64), m(rows=256, cols=64, tile=128), m(rows=256, cols=64, type=1),
                  m(rows=256, cols=64, batch=2)):
        assert quantize(m(), other) == b.BSR_ERR_SHAPE
    assert quantize(m(batch=2), used=d) == quantize(m(batch=65536)) == quantize(m(rows=1 << 31)) == b.BSR_ERR_SHAPE
    assert quantize(m(rows=1 << 30, cols=1 << 20)) == b.BSR_ERR_SHAPE
    assert quantize(m(rows=0), x=None) == quantize(m(cols=0), x=None) == b.BSR_OK
    assert quantize(m(), x=ctypes.c_void_p(264)) == quantize(m(q=(1 << 20) + 8)) == quantize(m(exponent=(1 << 24) + 8)) == b.BSR_ERR_ALIGNMENT
    assert quantize(m(q=512)) == b.BSR_ERR_INVALID_ARG   # over x

    def product(a=None, w=None, bias=None, Y=f, dt=1, group=0, offsets=None, groups=0, ws=None, size=0):
        a, w = a or m(), w or m(rows=32, tile=128, q=1 << 25, exponent=1 << 26)
        return lib.bsr_fp8_product(a, w, bias, Y, dt, group, offsets, groups, ws, size, None)

    for bad in (dict(w=m(cols=255)), dict(a=m(batch=2)), dict(w=m(batch=2)), dict(group=1, groups=0, offsets=d),
                dict(group=1, groups=2, offsets=d), dict(group=2, groups=1025, offsets=d),
                dict(a=m(rows=1 << 25), w=m(rows=1 << 25)), dict(a=m(rows=1 << 29), group=2, groups=1024, offsets=d)):
        assert product(**bad) == b.BSR_ERR_SHAPE
    for bad in (dict(dt=2), dict(group=3), dict(a=m(tile=2)), dict(w=m(type=-1))):
        assert product(**bad) == b.BSR_ERR_UNSUPPORTED
    for bad in (dict(offsets=d), dict(group=2, groups=2), dict(group=2, groups=2, offsets=d, bias=d), dict(Y=None),
                dict(a=m(q=None)), dict(w=m(exponent=None))):
        assert product(**bad) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_fp8_product(None, m(), None, f, 1, 0, None, 0, None, 0, None) == b.BSR_ERR_INVALID_ARG
    assert product(Y=ctypes.c_void_p((1 << 32) + 8), size=1 << 40, ws=e) == b.BSR_ERR_ALIGNMENT
    assert product(Y=ctypes.c_void_p(1 << 20), size=1 << 40, ws=e) == b.BSR_ERR_INVALID_ARG
    assert product(a=m(rows=0)) == b.BSR_OK
    assert lib.bsr_fp8_product_workspace(m(), m(), 0, 0, 0, None) == b.BSR_ERR_INVALID_ARG
    assert lib.bsr_fp8_product_workspace(m(), m(cols=1), 0, 0, 0, ctypes.byref(n)) == b.BSR_ERR_SHAPE and n.value == 0


def test_python_refusals(lib):
    import paper_2106_08846_gb300 as bsr
    order = bsr.ExpertOrder(4, 2, 8, 1, device="cpu")
    x = torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(TypeError):
        bsr.bsr_expert_order(x.long(), 8)
    with pytest.raises(ValueError):
        bsr.bsr_expert_order(x.view(-1), 8)
    with pytest.raises(ValueError):
        bsr.bsr_expert_order(x, 9, order=order)
    with pytest.raises(AttributeError):
        order.place = x
    X = torch.zeros(4, 16)
    for bad in (torch.zeros(5, 16), torch.zeros(4), torch.zeros(16, 4).T):
        with pytest.raises(ValueError):
            bsr.bsr_expert_rows(bad, order)
    with pytest.raises(TypeError):
        bsr.bsr_expert_rows(X.half(), order)
    with pytest.raises(TypeError):
        bsr.bsr_expert_rows(X, order, Xs=torch.zeros(8, 16, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        bsr.bsr_expert_sum(torch.zeros(8, 16), order, torch.zeros(8))
    with pytest.raises(ValueError):
        bsr.bsr_expert_sum_backward(None, order, torch.zeros(4, 2), X)
    for bad in (dict(tile=2), dict(fmt="e3m4")):
        with pytest.raises(ValueError):
            bsr.Fp8Matrix(4, 128, device="cpu", **bad)
    with pytest.raises(ValueError):
        bsr.bsr_fp8_quantize(X, form="x")
    with pytest.raises(TypeError):
        bsr.bsr_fp8_quantize(X.half())
    with pytest.raises(ValueError):
        bsr.bsr_fp8_quantize(X.T)
    with pytest.raises(ValueError):
        bsr.bsr_fp8_quantize(X, out=bsr.Fp8Matrix(4, 17, device="cpu"))
    a, w = bsr.Fp8Matrix(4, 16, device="cpu"), bsr.Fp8Matrix(8, 16, 128, device="cpu")
    with pytest.raises(AttributeError):
        a.q = a.scale
    for bad in (dict(over="x"), dict(offsets=torch.zeros(3, dtype=torch.int32)), dict(Y=torch.zeros(4, 9)), dict(bias=torch.zeros(9))):
        with pytest.raises(ValueError):
            bsr.bsr_fp8_product(a, w, **bad)
    with pytest.raises(TypeError):
        bsr.bsr_fp8_product(a, w, dtype=torch.float16)
