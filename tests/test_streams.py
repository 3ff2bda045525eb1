"""Calls on a stream that is not the current one, on the CPU with the library and
torch's streams replaced: what a call allocates itself is written only after the
current stream's last use of the memory, and stays taken until the call's work is
done."""
import contextlib
import ctypes
import types

import pytest
import torch

from paper_2106_08846_gb300 import bsrlib

F32 = torch.float32


class Stream:
    def __init__(self, handle, log):
        self.cuda_stream, self.log = handle, log

    def wait_stream(self, other):
        self.log.append(("wait", self.cuda_stream, other.cuda_stream))


@pytest.fixture
def world(monkeypatch):
    """(log, current, other): the log has waits, records, allocations on a stream of their own and launches."""
    log, inside = [], []
    current, other = Stream(11, log), Stream(22, log)
    empty = torch.empty

    def workspace(*a):
        a[-1]._obj.value = 4096
        return 0

    def launch(name):
        return lambda *a: log.append(("launch", name)) or 0

    lib = types.SimpleNamespace(bsr_gated_workspace=workspace, bsr_residual_norm_workspace=workspace,
                                **{n: launch(n) for n in ("bsr_gated", "bsr_gated_backward", "bsr_residual_norm",
                                                          "bsr_residual_norm_backward", "bsr_spmm")})

    def from_dense(*a):
        log.append(("launch", "bsr_from_dense"))
        a[11]._obj.value = 3
        return 0

    lib.bsr_from_dense = from_dense

    @contextlib.contextmanager
    def on(s):
        inside.append(s.cuda_stream)
        yield
        inside.pop()

    def new_empty(*a, **k):
        if inside:
            log.append(("own", inside[-1]))
        return empty(*a, **k)

    monkeypatch.setattr(bsrlib, "_lib", lib)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", new_empty)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("record", t.data_ptr(), s.cuda_stream)),
                        raising=False)
    yield log, current, other


def check(log, outputs, name):
    """Outputs made by a call on stream 22: recorded there, and written after a wait for stream 11."""
    at = log.index(("launch", name))
    assert ("wait", 22, 11) in log[:at]
    for t in outputs:
        assert ("record", t.data_ptr(), 22) in log, tuple(t.shape)


def rows(*shape):
    return torch.zeros(shape, dtype=F32)


def test_residual_norm(world):
    log, _, other = world
    w = rows(8)
    out = bsrlib.bsr_residual_norm(rows(4, 8), rows(4, 8), pre="rms", pre_w=w, stream=other)
    check(log, out, "bsr_residual_norm")


def test_residual_norm_with_one_output_given(world):
    log, _, other = world
    h_out, z = bsrlib.bsr_residual_norm(rows(4, 8), rows(4, 8), pre="rms", h_out=rows(4, 8), stream=other)
    check(log, [z], "bsr_residual_norm")
    assert not [e for e in log if e[0] == "record" and e[1] == h_out.data_ptr()]   # (the caller's)


def test_residual_norm_backward(world):
    log, _, other = world
    out = bsrlib.bsr_residual_norm_backward(rows(4, 8), rows(4, 8), rows(4, 8), rows(4, 8), gate=rows(4, 8), scale=rows(8),
                                            post="rms", post_w=rows(8), post_b=rows(8), pre="layer", pre_w=rows(8),
                                            pre_b=rows(8), stream=other)
    assert len(out) == 8
    check(log, out.values(), "bsr_residual_norm_backward")
    assert ("own", 22) in log   # the workspace


@pytest.mark.parametrize("N", [4, 40])
def test_gated(world, N):
    log, _, other = world
    check(log, [bsrlib.bsr_gated(rows(N, 8), rows(16, 8), rows(16, 8), stream=other)], "bsr_gated")


def test_gated_backward(world):
    log, _, other = world
    out = bsrlib.bsr_gated_backward(rows(4, 8), rows(16, 8), rows(16, 8), rows(16), rows(16), rows(4, 16), stream=other)
    assert len(out) == 5
    check(log, out.values(), "bsr_gated_backward")


def test_product_and_conversion(world):
    log, _, other = world
    h = bsrlib.Handle(ctypes.c_void_p(1), (), 16, 16, 64, 32, F32)
    X = rows(4, 32)
    device_rows = types.SimpleNamespace(shape=X.shape, dtype=F32, device=X.device, is_cuda=True, is_contiguous=lambda: True,
                                        data_ptr=X.data_ptr)
    try:
        check(log, [h.spmm(device_rows, stream=other)], "bsr_spmm")
    finally:
        h._ptr = None
    log.clear()
    W = rows(64, 32)
    weight = types.SimpleNamespace(shape=W.shape, dtype=F32, device=W.device, is_cuda=True, is_contiguous=lambda: True,
                                   data_ptr=W.data_ptr)
    check(log, bsrlib.bsr_from_dense(weight, 16, 16, stream=other), "bsr_from_dense")


def test_nothing_waits_where_the_caller_gave_every_output(world):
    log, _, other = world
    bsrlib.bsr_residual_norm(rows(4, 8), None, h_out=rows(4, 8), stream=other)
    bsrlib.bsr_gated(rows(40, 8), rows(16, 8), rows(16, 8), H=rows(40, 16), stream=other)
    assert not [e for e in log if e[0] in ("wait", "record")]


def test_the_current_stream_needs_neither(world):
    log, current, _ = world
    bsrlib.bsr_gated(rows(40, 8), rows(16, 8), rows(16, 8), stream=current)
    assert not [e for e in log if e[0] in ("wait", "record")]
