"""ctypes binding of include/bsr.h, with the same names.

Argument marshalling only: every step of the product and of the BSR
conversion runs in libbsr_gb300.so. torch supplies device memory, streams and
tensors; tensors cross as ``data_ptr()`` and streams as their ``cuda_stream``.
There is no CPU fallback: if the library is missing, loading raises.
With a `stream` other than the current one, outputs that a call makes itself are
made on the current stream and written after what it still does; they may be used
there once it has waited for `stream`.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbsr_gb300.so")

BSR_OK = 0
BSR_ERR_INVALID_ARG = 1
BSR_ERR_SHAPE = 2
BSR_ERR_UNSUPPORTED = 3
BSR_ERR_CAPACITY = 4
BSR_ERR_STRUCTURE = 5
BSR_ERR_ALIGNMENT = 6
BSR_ERR_CUDA = 7
BSR_ERR_TIMEOUT = 8
BSR_ERR_ALLOC = 9

BSR_F32 = 0
BSR_BF16 = 1

_DT = {torch.float32: BSR_F32, torch.bfloat16: BSR_BF16}
_TORCH_DT = {BSR_F32: torch.float32, BSR_BF16: torch.bfloat16}

BSR_NORM_NONE = 0
BSR_NORM_LAYER = 1
BSR_NORM_RMS = 2

BSR_ACT_SILU = 0
BSR_ACT_GELU = 1
BSR_ACT_GELU_TANH = 2
BSR_ACT_RELU = 3
BSR_ACT_SIGMOID = 4

_ACT = {"silu": BSR_ACT_SILU, "gelu": BSR_ACT_GELU, "gelu_tanh": BSR_ACT_GELU_TANH, "relu": BSR_ACT_RELU,
        "sigmoid": BSR_ACT_SIGMOID}
_NORM = {"none": BSR_NORM_NONE, "layer": BSR_NORM_LAYER, "rms": BSR_NORM_RMS}

_lib = None


class _ResidualNorm(ctypes.Structure):
    """bsr_residual_norm_t"""
    _fields_ = [("D", ctypes.c_int64), ("gate_tokens", ctypes.c_int64), ("block_dt", ctypes.c_int),
                ("stream_dt", ctypes.c_int), ("post", ctypes.c_int), ("pre", ctypes.c_int), ("post_eps", ctypes.c_float),
                ("pre_eps", ctypes.c_float), ("alpha", ctypes.c_float), ("scale", ctypes.c_void_p),
                ("post_w", ctypes.c_void_p), ("post_b", ctypes.c_void_p), ("pre_w", ctypes.c_void_p),
                ("pre_b", ctypes.c_void_p)]


class _ResidualNormGrads(ctypes.Structure):
    """bsr_residual_norm_grads_t"""
    _fields_ = [(k, ctypes.c_void_p) for k in ("dgate", "dscale", "dpost_w", "dpost_b", "dpre_w", "dpre_b")]


class BsrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {bsr_status_str(status)}")


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libbsr_gb300.so (built by ``__graft_entry__.build()``); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build the CUDA library first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(path)
        P, I64, I, U = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int
        lib.bsr_from_dense.argtypes = [P, I64, I64, I, I, ctypes.c_float, U, P, P, P, I64,
                                       ctypes.POINTER(I64), P]
        lib.bsr_from_dense.restype = U
        lib.bsr_create.argtypes = [P, P, P, I, I, I64, I64, U, ctypes.POINTER(P)]
        lib.bsr_create.restype = U
        lib.bsr_reserve.argtypes = [P, I64]
        lib.bsr_reserve.restype = U
        lib.bsr_spmm.argtypes = [P, P, P, P, I64, P]
        lib.bsr_spmm.restype = U
        lib.bsr_spmm_noalloc.argtypes = [P, P, P, P, I64, P]
        lib.bsr_spmm_noalloc.restype = U
        lib.bsr_spmm_batch.argtypes = [ctypes.POINTER(P), ctypes.c_int, P, ctypes.POINTER(P), ctypes.POINTER(P),
                                       I64, P]
        lib.bsr_spmm_batch.restype = U
        lib.bsr_plan_create.argtypes = [ctypes.POINTER(P), ctypes.POINTER(P), ctypes.POINTER(P), ctypes.POINTER(P),
                                        ctypes.POINTER(I64), ctypes.c_int, ctypes.c_int, ctypes.POINTER(P)]
        lib.bsr_plan_create.restype = U
        lib.bsr_plan_launch.argtypes = [P, P]
        lib.bsr_plan_launch.restype = U
        lib.bsr_plan_get_order.argtypes = [P, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int), ctypes.c_int,
                                           ctypes.POINTER(ctypes.c_int)]
        lib.bsr_plan_get_order.restype = U
        lib.bsr_plan_destroy.argtypes = [P]
        lib.bsr_plan_destroy.restype = None
        lib.bsr_check_device_status.argtypes = [P]
        lib.bsr_check_device_status.restype = U
        lib.bsr_get_schedule.argtypes = [P, ctypes.c_char_p, ctypes.c_size_t]
        lib.bsr_get_schedule.restype = U
        lib.bsr_get_call_info.argtypes = [P, I64, ctypes.c_char_p, ctypes.c_size_t]
        lib.bsr_get_call_info.restype = U
        RN = ctypes.POINTER(_ResidualNorm)
        lib.bsr_residual_norm.argtypes = [RN, P, P, P, P, P, I64, P]
        lib.bsr_residual_norm.restype = U
        lib.bsr_residual_norm_workspace.argtypes = [RN, I64, ctypes.POINTER(ctypes.c_size_t)]
        lib.bsr_residual_norm_workspace.restype = U
        lib.bsr_residual_norm_backward.argtypes = [RN, P, P, P, P, P, P, P, ctypes.POINTER(_ResidualNormGrads), I64, P,
                                                   ctypes.c_size_t, P]
        lib.bsr_residual_norm_backward.restype = U
        lib.bsr_gated_workspace.argtypes = [I64, I64, I64, U, I, ctypes.POINTER(ctypes.c_size_t)]
        lib.bsr_gated_workspace.restype = U
        lib.bsr_gated.argtypes = [P, P, P, P, P, P, I64, I64, I64, U, I, P, ctypes.c_size_t, P]
        lib.bsr_gated.restype = U
        lib.bsr_gated_backward.argtypes = [P] * 11 + [I64, I64, I64, U, I, P, ctypes.c_size_t, P]
        lib.bsr_gated_backward.restype = U
        lib.bsr_check_status.argtypes = []
        lib.bsr_check_status.restype = U
        lib.bsr_destroy.argtypes = [P]
        lib.bsr_destroy.restype = None
        lib.bsr_status_str.argtypes = [U]
        lib.bsr_status_str.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def bsr_status_str(status: int) -> str:
    return load().bsr_status_str(status).decode()


def _check(status: int, where: str) -> None:
    if status != BSR_OK:
        raise BsrError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The current stream's handle and device without a Stream object (which takes
# 2.9 us to make, as long as the whole C call); its long form where torch has none.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _cur_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_cur_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_object(stream, device):
    """The torch stream of a call's `stream` argument (a Stream, or its handle as a number)."""
    if hasattr(stream, "cuda_stream"):
        return stream
    return torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else torch.cuda.default_stream(device)


def _lend(stream, device, *tensors) -> None:
    """Lets `stream` write tensors that a call has just made. Their memory is the
    current stream's: work of the call waits for what that stream still does with
    it, and it is handed out again only after the call's work."""
    if stream is None:
        return
    s, current = _stream_object(stream, device), torch.cuda.current_stream(device)
    if s.cuda_stream == current.cuda_stream:
        return
    s.wait_stream(current)
    for t in tensors:
        t.record_stream(s)


def _workspace(nbytes: int, device, stream) -> Optional[torch.Tensor]:
    """Scratch of one call, from torch's allocator and of the call's own stream: it
    waits for nobody else, and is handed out again only to later work of that stream."""
    if nbytes == 0:
        return None
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(_stream_object(stream, device)):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def dtype_code(dtype: torch.dtype) -> int:
    if dtype not in _DT:
        raise TypeError(f"unsupported dtype {dtype}: float32 or bfloat16")
    return _DT[dtype]


def bsr_from_dense(W: torch.Tensor, R: int, C: int, threshold: float = 0.0, stream=None
                   ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """BSR arrays (indptr, indices, data[nnzb, R, C]) of the dense device weight W[M, K].

    Two calls of the C function: a query for nnzb, then the fill into
    tensors allocated here.
    """
    lib = load()
    if not W.is_cuda or not W.is_contiguous():
        raise ValueError("W must be a contiguous CUDA tensor")
    M, K = W.shape
    dt = dtype_code(W.dtype)
    if R <= 0 or C <= 0 or M % R or K % C:
        _check(BSR_ERR_SHAPE, "bsr_from_dense")
    indptr = torch.empty(M // R + 1, dtype=torch.int32, device=W.device)
    nnzb = ctypes.c_int64(0)
    s = _stream(stream)
    _lend(stream, W.device, indptr)
    _check(lib.bsr_from_dense(_ptr(W), M, K, R, C, threshold, dt, _ptr(indptr), None, None, 0,
                              ctypes.byref(nnzb), s), "bsr_from_dense(query)")
    n = nnzb.value
    indices = torch.empty(max(n, 0), dtype=torch.int32, device=W.device)
    data = torch.empty((max(n, 0), R, C), dtype=W.dtype, device=W.device)
    if n > 0:
        _lend(stream, W.device, indices, data)
        _check(lib.bsr_from_dense(_ptr(W), M, K, R, C, threshold, dt, _ptr(indptr), _ptr(indices),
                                  _ptr(data), n, ctypes.byref(nnzb), s), "bsr_from_dense")
    return indptr, indices, data


class Handle:
    """A created BSR operator. Keeps its borrowed arrays alive until destroyed."""

    def __init__(self, ptr: ctypes.c_void_p, arrays, R, C, M, K, dtype):
        self._ptr = ptr
        self._arrays = arrays
        self.R, self.C, self.M, self.K, self.dtype = R, C, M, K, dtype

    @property
    def ptr(self) -> ctypes.c_void_p:
        if self._ptr is None:
            raise RuntimeError("handle destroyed")
        return self._ptr

    def spmm(self, X: torch.Tensor, bias: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
        if Y is None:
            Y = torch.empty((X.shape[0], self.M), dtype=X.dtype, device=X.device,
                            pin_memory=not X.is_cuda)
            if X.is_cuda:
                _lend(stream, X.device, Y)
        bsr_spmm(self, X, bias, Y, X.shape[0], stream)
        return Y

    def reserve(self, N_max: int) -> None:
        bsr_reserve(self, N_max)

    def schedule(self) -> dict:
        return parse_schedule(bsr_get_schedule(self))

    def call_info(self, N: int) -> dict:
        """The kernel that a call of N tokens runs and its launches."""
        return parse_schedule(bsr_get_call_info(self, N))

    def check_device_status(self) -> int:
        return bsr_check_device_status(self)

    def destroy(self) -> None:
        if self._ptr is not None:
            load().bsr_destroy(self._ptr)
            self._ptr = None
            self._arrays = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def bsr_create(indptr: torch.Tensor, indices: torch.Tensor, data: torch.Tensor, R: int, C: int,
               M: int, K: int) -> Handle:
    lib = load()
    for name, t in (("indptr", indptr), ("indices", indices), ("data", data)):
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    if indptr.dtype != torch.int32 or indices.dtype != torch.int32:
        raise TypeError("indptr and indices must be int32")
    out = ctypes.c_void_p()
    _check(lib.bsr_create(_ptr(indptr), _ptr(indices) if indices.numel() else None,
                          _ptr(data) if data.numel() else None, R, C, M, K, dtype_code(data.dtype),
                          ctypes.byref(out)), "bsr_create")
    return Handle(out, (indptr, indices, data), R, C, M, K, data.dtype)


def bsr_reserve(h: Handle, N_max: int) -> None:
    _check(load().bsr_reserve(h.ptr, N_max), "bsr_reserve")


def _check_product(h: Handle, X: torch.Tensor, bias: Optional[torch.Tensor], Y: torch.Tensor, N: Optional[int]) -> int:
    """The checks of one product's tensors; returns N."""
    dt = h.dtype
    if X.dtype is not dt or Y.dtype is not dt:
        raise TypeError("X and Y must have the handle's dtype")
    if not X.is_contiguous() or not Y.is_contiguous():
        raise ValueError("X and Y must be contiguous")
    if bias is not None and (bias.dtype is not torch.float32 or not bias.is_contiguous()):
        raise TypeError("bias must be a contiguous float32 tensor")
    xs, ys = X.shape, Y.shape
    if N is None:
        N = xs[0]
    if xs[-1] != h.K or ys[-1] != h.M or xs[0] < N or ys[0] < N:
        raise ValueError("X must be [N, K] and Y [N, M]")
    return N


def bsr_spmm(h: Handle, X: torch.Tensor, bias: Optional[torch.Tensor], Y: torch.Tensor,
             N: Optional[int] = None, stream=None) -> None:
    """Y[N, M] = X[N, K] W^T + bias; X and Y both on the device or both in host memory."""
    N = _check_product(h, X, bias, Y, N)
    st = (_lib or load()).bsr_spmm(h.ptr, X.data_ptr(), None if bias is None else bias.data_ptr(), Y.data_ptr(), N,
                                   _stream(stream))
    if st:
        _check(st, "bsr_spmm")


def bsr_spmm_noalloc(h: Handle, X: torch.Tensor, bias: Optional[torch.Tensor], Y: torch.Tensor,
                     N: Optional[int] = None, stream=None) -> None:
    """bsr_spmm without any device allocation (device X and Y only): split-row
    partials use the library's fixed scratch array (see include/bsr.h)."""
    N = _check_product(h, X, bias, Y, N)
    _check(load().bsr_spmm_noalloc(h.ptr, _ptr(X), _ptr(bias), _ptr(Y), N, _stream(stream)), "bsr_spmm_noalloc")


def bsr_spmm_batch(handles, X: torch.Tensor, biases, Ys, N: Optional[int] = None, stream=None) -> None:
    """Ys[i][N, M_i] = X[N, K] W_i^T + biases[i] for handles sharing X (device
    tensors only); fused products run as one grid (see include/bsr.h)."""
    n = len(handles)
    if len(Ys) != n or (biases is not None and len(biases) != n):
        raise ValueError("one output (and bias, if given) per handle")
    if not X.is_contiguous():
        raise ValueError("X must be contiguous")
    N = X.shape[0] if N is None else N
    if n and (X.shape[-1] != handles[0].K or X.shape[0] < N):
        raise ValueError("X must be [N, K]")   # (a K that differs between handles: BSR_ERR_SHAPE)
    for h, Y in zip(handles, Ys):
        if X.dtype != h.dtype or Y.dtype != h.dtype:
            raise TypeError("X and every Y must have the handles' dtype")
        if not Y.is_contiguous() or Y.shape[-1] != h.M or Y.shape[0] < N:
            raise ValueError("each Y must be [N, M] and contiguous")
    if biases is not None:
        for b in biases:
            if b is not None and (b.dtype != torch.float32 or not b.is_contiguous()):
                raise TypeError("biases must be contiguous float32 tensors")
    P = ctypes.c_void_p
    harr = (P * max(n, 1))(*[h.ptr for h in handles])
    yarr = (P * max(n, 1))(*[_ptr(Y) for Y in Ys])
    barr = None if biases is None else (P * max(n, 1))(*[_ptr(b) for b in biases])
    _check(load().bsr_spmm_batch(harr, n, _ptr(X), barr, yarr, N, _stream(stream)), "bsr_spmm_batch")


class Plan:
    """A product sequence captured into a CUDA graph (bsr_plan_create). Keeps
    the handles and tensors it was built on alive."""

    def __init__(self, ptr, n, keep):
        self._ptr = ptr
        self.n = n
        self._keep = keep

    def launch(self, stream=None) -> None:
        _check(load().bsr_plan_launch(self._ptr, _stream(stream)), "bsr_plan_launch")

    def order(self):
        """(order, call, n_kernels): the product executed k-th, the library call
        that runs it, and the kernel launches in the graph."""
        n = max(self.n, 1)
        o, c, k = (ctypes.c_int * n)(), (ctypes.c_int * n)(), ctypes.c_int(0)
        _check(load().bsr_plan_get_order(self._ptr, o, c, self.n, ctypes.byref(k)), "bsr_plan_get_order")
        run = [i for i in range(self.n) if o[i] >= 0]
        return [o[i] for i in run], [c[i] for i in run], k.value

    def destroy(self) -> None:
        if self._ptr is not None:
            load().bsr_plan_destroy(self._ptr)
            self._ptr = None
            self._keep = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def bsr_plan_create(handles, Xs, biases, Ys, Ns=None, independent: bool = False) -> Plan:
    """Captures the products Ys[i] = Xs[i] W_i^T + biases[i] (device tensors)
    into one CUDA graph; with ``independent`` the plan may regroup and fuse
    them (see include/bsr.h)."""
    n = len(handles)
    if len(Xs) != n or len(Ys) != n or (biases is not None and len(biases) != n):
        raise ValueError("one X, Y (and bias, if given) per handle")
    Ns = [X.shape[0] for X in Xs] if Ns is None else list(Ns)
    for h, X, Y, N in zip(handles, Xs, Ys, Ns):
        if X.dtype != h.dtype or Y.dtype != h.dtype:
            raise TypeError("X and Y must have the handle's dtype")
        if not X.is_contiguous() or not Y.is_contiguous():
            raise ValueError("X and Y must be contiguous")
        if X.shape[-1] != h.K or Y.shape[-1] != h.M or X.shape[0] < N or Y.shape[0] < N:
            raise ValueError("X must be [N, K] and Y [N, M]")
    if biases is not None:
        for b in biases:
            if b is not None and (b.dtype != torch.float32 or not b.is_contiguous()):
                raise TypeError("biases must be contiguous float32 tensors")
    P = ctypes.c_void_p
    m = max(n, 1)
    harr = (P * m)(*[h.ptr for h in handles])
    xarr = (P * m)(*[_ptr(X) for X in Xs])
    yarr = (P * m)(*[_ptr(Y) for Y in Ys])
    barr = None if biases is None else (P * m)(*[_ptr(b) for b in biases])
    narr = (ctypes.c_int64 * m)(*Ns)
    out = P()
    _check(load().bsr_plan_create(harr, xarr, barr, yarr, narr, n, int(bool(independent)), ctypes.byref(out)),
           "bsr_plan_create")
    return Plan(out, n, (list(handles), list(Xs), list(Ys), None if biases is None else list(biases)))


def bsr_check_device_status(h: Handle) -> int:
    return load().bsr_check_device_status(h.ptr)


def bsr_check_status() -> int:
    """The first error that a kernel of bsr_gated or bsr_gated_backward recorded on the current device (synchronises it)."""
    return load().bsr_check_status()


def bsr_get_schedule(h: Handle) -> str:
    buf = ctypes.create_string_buffer(4096)
    _check(load().bsr_get_schedule(h.ptr, buf, len(buf)), "bsr_get_schedule")
    return buf.value.decode()


def bsr_get_call_info(h: Handle, N: int) -> str:
    buf = ctypes.create_string_buffer(256)
    _check(load().bsr_get_call_info(h.ptr, N, buf, len(buf)), "bsr_get_call_info")
    return buf.value.decode()


def bsr_destroy(h: Handle) -> None:
    h.destroy()


def _check_rows(name: str, t: Optional[torch.Tensor], shape, dtype: torch.dtype) -> None:
    if t is None:
        return
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of shape {list(shape)}")


def _is_rows(t: Optional[torch.Tensor], shape, dtype: torch.dtype) -> bool:
    """Whether _check_rows passes (the calls' fast path: one test, the names only where it fails)."""
    return t is None or (t.dtype is dtype and t.shape == shape and t.is_contiguous())


def _residual_norm(y, stream_dt, gate, gate_tokens, scale, alpha, post, post_w, post_b, pre, pre_w, pre_b, eps, pre_eps):
    """The checked bsr_residual_norm_t of a call."""
    if post not in _NORM or pre not in _NORM:
        raise ValueError("post and pre are 'none', 'layer' or 'rms'")
    if y.dim() != 2:
        raise ValueError("y must be [N, D]")
    N, D = y.shape
    f32, row = torch.float32, (D,)
    ptrs = []
    for w in (scale, post_w, post_b, pre_w, pre_b):
        if w is None:
            ptrs.append(None)
            continue
        if w.dtype is not f32 or w.shape != row or not w.is_contiguous():
            raise TypeError("scale and the norms' weights and biases must be contiguous float32 tensors of D features")
        ptrs.append(w.data_ptr())
    if gate is None:
        gate_tokens = 0
    else:
        if gate_tokens < 1:
            raise ValueError("gate_tokens must be at least 1")
        _check_rows("gate", gate, (-(-N // gate_tokens), D), y.dtype)
    return _ResidualNorm(D, gate_tokens, dtype_code(y.dtype), dtype_code(stream_dt), _NORM[post], _NORM[pre], eps,
                         eps if pre_eps is None else pre_eps, alpha, *ptrs)


def bsr_residual_norm(y: torch.Tensor, h: Optional[torch.Tensor] = None, *, gate: Optional[torch.Tensor] = None,
                      gate_tokens: int = 1, scale: Optional[torch.Tensor] = None, alpha: float = 1.0, post: str = "none",
                      post_w: Optional[torch.Tensor] = None, post_b: Optional[torch.Tensor] = None, pre: str = "none",
                      pre_w: Optional[torch.Tensor] = None, pre_b: Optional[torch.Tensor] = None, eps: float = 1e-5,
                      pre_eps: Optional[float] = None, h_out: Optional[torch.Tensor] = None,
                      z: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(h_out, z): h_out = alpha h + scale * gate * post(y) and z = pre(h_out)
    (None if pre is "none"), for rows y [N, D] of a block's output and h of the
    residual stream (None: no stream yet). gate has a row for each gate_tokens
    tokens; eps is both norms', or post's beside pre_eps. h_out may be h and z may
    be y (see include/bsr.h)."""
    dt, shape = y.dtype, y.shape
    st = (h if h is not None else h_out if h_out is not None else y).dtype
    p = _residual_norm(y, st, gate, gate_tokens, scale, alpha, post, post_w, post_b, pre, pre_w, pre_b, eps, pre_eps)
    made = []
    if h_out is None:
        h_out = torch.empty(shape, dtype=st, device=y.device)
        made.append(h_out)
    if z is None and pre != "none":
        z = torch.empty_like(y)
        made.append(z)
    if not (y.is_contiguous() and _is_rows(h, shape, st) and _is_rows(h_out, shape, st) and _is_rows(z, shape, dt)):
        for name, t, d in (("y", y, dt), ("h", h, st), ("h_out", h_out, st), ("z", z, dt)):
            _check_rows(name, t, shape, d)
    if made:
        _lend(stream, y.device, *made)
    status = (_lib or load()).bsr_residual_norm(p, y.data_ptr(), None if h is None else h.data_ptr(),
                                                None if gate is None else gate.data_ptr(), h_out.data_ptr(),
                                                None if z is None else z.data_ptr(), shape[0], _stream(stream))
    if status:
        _check(status, "bsr_residual_norm")
    return h_out, z


def bsr_residual_norm_backward(y: torch.Tensor, h_out: Optional[torch.Tensor], dh_out: Optional[torch.Tensor],
                               dz: Optional[torch.Tensor], *, gate: Optional[torch.Tensor] = None, gate_tokens: int = 1,
                               scale: Optional[torch.Tensor] = None, alpha: float = 1.0, post: str = "none",
                               post_w: Optional[torch.Tensor] = None, post_b: Optional[torch.Tensor] = None,
                               pre: str = "none", pre_w: Optional[torch.Tensor] = None,
                               pre_b: Optional[torch.Tensor] = None, eps: float = 1e-5, pre_eps: Optional[float] = None,
                               dy: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Gradients of bsr_residual_norm, whose arguments it takes with the h_out
    that it returned (needed if pre is a norm) and the gradients of h_out (None: 0)
    and of z (None if pre is "none"): "dy", "dh", and of each parameter given
    "dgate", "dscale", "dpost_w", "dpost_b", "dpre_w" and "dpre_b"."""
    dt, shape, device = y.dtype, y.shape, y.device
    st = next((t.dtype for t in (h_out, dh_out, dh) if t is not None), dt)
    p = _residual_norm(y, st, gate, gate_tokens, scale, alpha, post, post_w, post_b, pre, pre_w, pre_b, eps, pre_eps)
    made = []
    if dy is None:
        dy = torch.empty_like(y)
        made.append(dy)
    if dh is None:
        dh = torch.empty(shape, dtype=st, device=device)
        made.append(dh)
    if not (y.is_contiguous() and _is_rows(h_out, shape, st) and _is_rows(dh_out, shape, st) and _is_rows(dz, shape, dt)
            and _is_rows(dy, shape, dt) and _is_rows(dh, shape, st)):
        for name, t, d in (("y", y, dt), ("h_out", h_out, st), ("dh_out", dh_out, st), ("dz", dz, dt), ("dy", dy, dt),
                           ("dh", dh, st)):
            _check_rows(name, t, shape, d)
    out = {"dy": dy, "dh": dh}
    ptrs = []
    for name, w in (("dgate", gate), ("dscale", scale), ("dpost_w", post_w), ("dpost_b", post_b), ("dpre_w", pre_w),
                    ("dpre_b", pre_b)):
        if w is None:
            ptrs.append(None)
        else:   # (an allocation each: rows of one, as views, take the host twice as long)
            out[name] = d = torch.empty_like(w)
            made.append(d)
            ptrs.append(d.data_ptr())
    grads = _ResidualNormGrads(*ptrs)
    lib, n = _lib or load(), ctypes.c_size_t(0)
    status = lib.bsr_residual_norm_workspace(p, shape[0], ctypes.byref(n))
    if status:
        _check(status, "bsr_residual_norm_workspace")
    ws = _workspace(n.value, device, stream)
    if made:
        _lend(stream, device, *made)
    status = lib.bsr_residual_norm_backward(p, y.data_ptr(), _ptr(h_out), None if gate is None else gate.data_ptr(),
                                            _ptr(dh_out), _ptr(dz), dy.data_ptr(), dh.data_ptr(), grads, shape[0], _ptr(ws),
                                            n.value, _stream(stream))
    if status:
        _check(status, "bsr_residual_norm_backward")
    return out


def _check_gated(X, Wg, Wu, bg, bu, act: str) -> Tuple[int, int, int, int]:
    """The checks of a gated block's inputs; (N, F, K, type)."""
    if act not in _ACT:
        raise ValueError("act is one of " + ", ".join(_ACT))
    xt = X.dtype
    dt = dtype_code(xt)
    if X.dim() != 2 or Wg.dim() != 2:
        raise ValueError("X must be [N, K] and Wg and Wu [F, K]")
    (N, K), F = X.shape, Wg.shape[0]
    if not (X.is_contiguous() and _is_rows(Wg, (F, K), xt) and _is_rows(Wu, (F, K), xt) and _is_rows(bg, (F,), torch.float32)
            and _is_rows(bu, (F,), torch.float32)):
        for name, t, shape in (("X", X, (N, K)), ("Wg", Wg, (F, K)), ("Wu", Wu, (F, K))):
            _check_rows(name, t, shape, xt)
        _check_rows("bg", bg, (F,), torch.float32)
        _check_rows("bu", bu, (F,), torch.float32)
    return N, F, K, dt


def _gated_workspace(N, F, K, dt, backward, device, stream):
    n = ctypes.c_size_t(0)
    status = (_lib or load()).bsr_gated_workspace(N, F, K, dt, backward, ctypes.byref(n))
    if status:
        _check(status, "bsr_gated_workspace")
    return _workspace(n.value, device, stream), n.value


def bsr_gated(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, bg: Optional[torch.Tensor] = None,
              bu: Optional[torch.Tensor] = None, act: str = "silu", H: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """H = act(X Wg' + bg) * (X Wu' + bu): the gated feed-forward block of X
    [N, K] with dense weights [F, K]; act is "silu", "gelu" (erf), "gelu_tanh",
    "relu" or "sigmoid"."""
    N, F, K, dt = _check_gated(X, Wg, Wu, bg, bu, act)
    if H is None:
        H = torch.empty((N, F), dtype=X.dtype, device=X.device)
        _lend(stream, X.device, H)
    elif not _is_rows(H, (N, F), X.dtype):
        _check_rows("H", H, (N, F), X.dtype)
    ws, n = _gated_workspace(N, F, K, dt, 0, X.device, stream)
    status = _lib.bsr_gated(X.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), None if bg is None else bg.data_ptr(),
                            None if bu is None else bu.data_ptr(), H.data_ptr(), N, F, K, dt, _ACT[act],
                            None if ws is None else ws.data_ptr(), n, _stream(stream))
    if status:
        _check(status, "bsr_gated")
    return H


def bsr_gated_backward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, bg: Optional[torch.Tensor],
                       bu: Optional[torch.Tensor], dH: torch.Tensor, act: str = "silu",
                       dX: Optional[torch.Tensor] = None, dWg: Optional[torch.Tensor] = None,
                       dWu: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Gradients of bsr_gated from that of its result: "dX", "dWg", "dWu", and
    "dbg" and "dbu" where the biases are given. G and U are computed again;
    nothing is kept from the forward call."""
    N, F, K, dt = _check_gated(X, Wg, Wu, bg, bu, act)
    xt, w = X.dtype, Wg.shape
    made = []
    if dX is None:
        dX = torch.empty_like(X)
        made.append(dX)
    if dWg is None:
        dWg = torch.empty_like(Wg)
        made.append(dWg)
    if dWu is None:
        dWu = torch.empty_like(Wu)
        made.append(dWu)
    if not (_is_rows(dH, (N, F), xt) and _is_rows(dX, X.shape, xt) and _is_rows(dWg, w, xt) and _is_rows(dWu, w, xt)):
        for name, t, shape in (("dH", dH, (N, F)), ("dX", dX, X.shape), ("dWg", dWg, w), ("dWu", dWu, w)):
            _check_rows(name, t, shape, xt)
    out = {"dX": dX, "dWg": dWg, "dWu": dWu}
    for name, b in (("dbg", bg), ("dbu", bu)):
        if b is not None:
            out[name] = torch.empty_like(b)
            made.append(out[name])
    if made:
        _lend(stream, X.device, *made)
    ws, n = _gated_workspace(N, F, K, dt, 1, X.device, stream)
    status = _lib.bsr_gated_backward(X.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), _ptr(bg), _ptr(bu), dH.data_ptr(),
                                     dX.data_ptr(), dWg.data_ptr(), dWu.data_ptr(), _ptr(out.get("dbg")),
                                     _ptr(out.get("dbu")), N, F, K, dt, _ACT[act], _ptr(ws), n, _stream(stream))
    if status:
        _check(status, "bsr_gated_backward")
    return out


def parse_schedule(text: str) -> dict:
    out = {}
    for line in text.splitlines():
        m = re.match(r"^(\w+)=(.*)$", line)
        if m:
            k, v = m.groups()
            try:
                out[k] = int(v)
            except ValueError:
                out[k] = v
    return out
