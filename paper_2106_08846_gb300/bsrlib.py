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

BSR_E4M3 = 0
BSR_E5M2 = 1

BSR_GROUP_NONE = 0
BSR_GROUP_ROWS = 1
BSR_GROUP_COLUMNS = 2

BSR_ACT_SILU = 0
BSR_ACT_GELU = 1
BSR_ACT_GELU_TANH = 2
BSR_ACT_RELU = 3
BSR_ACT_SIGMOID = 4

_ACT = {"silu": BSR_ACT_SILU, "gelu": BSR_ACT_GELU, "gelu_tanh": BSR_ACT_GELU_TANH, "relu": BSR_ACT_RELU,
        "sigmoid": BSR_ACT_SIGMOID}
_NORM = {"none": BSR_NORM_NONE, "layer": BSR_NORM_LAYER, "rms": BSR_NORM_RMS}

_FP8 = {"e4m3": BSR_E4M3, "e5m2": BSR_E5M2}
_FP8_TYPE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}

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


class _Experts(ctypes.Structure):
    """bsr_experts_t"""
    _fields_ = [("N", ctypes.c_int64), ("R", ctypes.c_int64), ("k", ctypes.c_int), ("E", ctypes.c_int), ("align", ctypes.c_int),
                ("offsets", ctypes.c_void_p), ("place", ctypes.c_void_p), ("source", ctypes.c_void_p)]


class _Fp8Matrix(ctypes.Structure):
    """bsr_fp8_matrix_t"""
    _fields_ = [("batch", ctypes.c_int64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("tile", ctypes.c_int),
                ("type", ctypes.c_int), ("q", ctypes.c_void_p), ("exponent", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


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
        EX, M8, SIZE = ctypes.POINTER(_Experts), ctypes.POINTER(_Fp8Matrix), ctypes.c_size_t
        lib.bsr_expert_capacity.argtypes = [I64, I, I, I, ctypes.POINTER(I64)]
        lib.bsr_expert_capacity.restype = U
        lib.bsr_expert_order.argtypes = [EX, P, P]
        lib.bsr_expert_order.restype = U
        lib.bsr_expert_rows.argtypes = [EX, P, P, I64, U, P]
        lib.bsr_expert_rows.restype = U
        lib.bsr_expert_sum.argtypes = [EX, P, P, P, I64, U, P]
        lib.bsr_expert_sum.restype = U
        lib.bsr_expert_sum_backward.argtypes = [EX, P, P, P, P, P, I64, U, P]
        lib.bsr_expert_sum_backward.restype = U
        lib.bsr_fp8_quantize.argtypes = [P, U, M8, M8, P, P]
        lib.bsr_fp8_quantize.restype = U
        lib.bsr_fp8_product_workspace.argtypes = [M8, M8, U, U, I64, ctypes.POINTER(SIZE)]
        lib.bsr_fp8_product_workspace.restype = U
        lib.bsr_fp8_product.argtypes = [M8, M8, P, P, U, U, P, I64, P, SIZE, P]
        lib.bsr_fp8_product.restype = U
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
    """The first error that a kernel of bsr_gated, bsr_gated_backward or bsr_fp8_product recorded on the current device
    (synchronises it)."""
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


class ExpertOrder:
    """Which rows N tokens' k choices of E experts have (bsr_expert_order fills it in):
    `offsets` [E + 1], `place` [N, k] and `source` [rows], int32 on the device; see
    include/bsr.h. `rows` is what the sorted tensors must have; `used` is a view of
    the number that is in use, offsets[E]."""

    def __init__(self, N: int, k: int, E: int, align: int = 1, device="cuda"):
        rows = ctypes.c_int64(0)
        _check(load().bsr_expert_capacity(N, k, E, align, ctypes.byref(rows)), "bsr_expert_capacity")
        self.N, self.k, self.E, self.align, self.rows = N, k, E, align, rows.value
        self._offsets = torch.empty(E + 1, dtype=torch.int32, device=device)
        self._place = torch.empty((N, k), dtype=torch.int32, device=device)
        self._source = torch.empty(self.rows, dtype=torch.int32, device=device)
        self._used = self._offsets[E:]
        self._c = _Experts(N, self.rows, k, E, align, _ptr(self._offsets), _ptr(self._place) if N else None,
                           _ptr(self._source) if self.rows else None)

    # (not to be replaced: the calls have their addresses)
    offsets = property(lambda self: self._offsets)
    place = property(lambda self: self._place)
    source = property(lambda self: self._source)
    used = property(lambda self: self._used)


def bsr_expert_order(experts: torch.Tensor, E: int, align: int = 1, order: Optional[ExpertOrder] = None, stream=None) -> ExpertOrder:
    """The order of the tokens' choices `experts` [N, k] (int32; a value outside
    0 .. E - 1 is a dropped choice), each expert's rows from a multiple of `align` on.
    Fills `order` if given. Nothing is read back to the host."""
    shape = experts.shape
    if len(shape) != 2:
        raise ValueError("experts must be [N, k]")
    N, k = shape
    if experts.dtype is not torch.int32 or not experts.is_contiguous():
        _check_rows("experts", experts, shape, torch.int32)
    if order is None:
        order = ExpertOrder(N, k, E, align, experts.device)
        _lend(stream, experts.device, order.offsets, order.place, order.source)
    elif order.N != N or order.k != k or order.E != E or order.align != align:
        raise ValueError("order is of other sizes")
    status = _lib.bsr_expert_order(order._c, experts.data_ptr(), _stream(stream))
    if status:
        _check(status, "bsr_expert_order")
    return order


def _check_sorted(of: str, t: torch.Tensor, rows: int, *others) -> Tuple[int, int]:
    """The features and the type of t, which must have `rows` rows, and the checks of others
    (name, tensor or None, shape's rows), of as many features and its type."""
    shape, dtype = t.shape, t.dtype
    if len(shape) != 2:
        raise ValueError(f"{of} must be [{rows}, D]")
    if shape[0] != rows or not t.is_contiguous():
        _check_rows(of, t, (rows, shape[1]), dtype)
    for name, o, n in others:
        if o is not None and not _is_rows(o, (n, shape[1]), dtype):
            _check_rows(name, o, (n, shape[1]), dtype)
    dt = _DT.get(dtype)
    return shape[1], dtype_code(dtype) if dt is None else dt   # (dtype_code raises)


def _check_weights(order: ExpertOrder, weights: Optional[torch.Tensor]) -> Optional[int]:
    if weights is None:
        return None
    shape = (order.N, order.k)
    if not _is_rows(weights, shape, torch.float32):
        _check_rows("weights", weights, shape, torch.float32)
    return weights.data_ptr()


def _made(rows: int, like: torch.Tensor, stream) -> torch.Tensor:
    t = torch.empty((rows, like.shape[1]), dtype=like.dtype, device=like.device)
    _lend(stream, like.device, t)
    return t


def bsr_expert_rows(X: torch.Tensor, order: ExpertOrder, Xs: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Xs [order.rows, D]: the tokens' rows X [N, D] in the experts' order, zeros behind
    an expert's last one; rows from order.used on are left as they were (of an Xs
    that the call makes: without a value). Its gradient is bsr_expert_sum without weights."""
    D, dt = _check_sorted("X", X, order.N, ("Xs", Xs, order.rows))
    if Xs is None:
        Xs = _made(order.rows, X, stream)
    status = _lib.bsr_expert_rows(order._c, X.data_ptr(), Xs.data_ptr(), D, dt, _stream(stream))
    if status:
        _check(status, "bsr_expert_rows")
    return Xs


def bsr_expert_sum(Ys: torch.Tensor, order: ExpertOrder, weights: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """Y [N, D]: for each token the sum of its choices' rows of Ys [order.rows, D], with
    the router's weights (fp32 [N, k], None: 1)."""
    D, dt = _check_sorted("Ys", Ys, order.rows, ("Y", Y, order.N))
    w = _check_weights(order, weights)
    if Y is None:
        Y = _made(order.N, Ys, stream)
    status = _lib.bsr_expert_sum(order._c, Ys.data_ptr(), w, Y.data_ptr(), D, dt, _stream(stream))
    if status:
        _check(status, "bsr_expert_sum")
    return Y


def bsr_expert_sum_backward(Ys: Optional[torch.Tensor], order: ExpertOrder, weights: Optional[torch.Tensor], dY: torch.Tensor,
                            dYs: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Gradients of bsr_expert_sum: "dYs" (rows from order.used on as in bsr_expert_rows),
    and "dweights" where weights are given; without them Ys is not needed."""
    D, dt = _check_sorted("dY", dY, order.N, ("Ys", Ys, order.rows), ("dYs", dYs, order.rows))
    w = _check_weights(order, weights)
    if w is not None and Ys is None:
        raise ValueError("the gradient of the weights needs Ys")
    out = {"dYs": _made(order.rows, dY, stream) if dYs is None else dYs}
    if w is not None:
        out["dweights"] = torch.empty_like(weights)
        _lend(stream, dY.device, out["dweights"])
    status = _lib.bsr_expert_sum_backward(order._c, _ptr(Ys), w, dY.data_ptr(), out["dYs"].data_ptr(), _ptr(out.get("dweights")), D, dt,
                                          _stream(stream))
    if status:
        _check(status, "bsr_expert_sum_backward")
    return out


class Fp8Matrix:
    """[rows, cols] values in 8 bits (batch: that many, of shape [batch, rows, cols]) with
    a scale for each block of 128 columns of `tile` rows: x[r, c] is
    q[r, c] * scale[c // 128, r // tile]. `q` has cols rounded up to 128, zeros past
    them; `exponent` is what the product reads of the scales, powers of two (include/bsr.h). fmt: "e4m3" or "e5m2"; bsr_fp8_quantize fills it in."""

    __slots__ = ("rows", "cols", "tile", "fmt", "batch", "_base", "_q", "_scale", "_c", "__weakref__")

    def __init__(self, rows: int, cols: int, tile: int = 1, fmt: str = "e4m3", batch: Optional[int] = None, device="cuda"):
        code = _FP8.get(fmt)
        if code is None or (tile != 1 and tile != 128):
            raise ValueError("fmt is 'e4m3' or 'e5m2', tile 1 or 128")
        self.rows, self.cols, self.tile, self.fmt, self.batch = rows, cols, tile, fmt, batch
        blocks, runs, n = (cols + 127) // 128, rows if tile == 1 else (rows + 127) // 128, 1 if batch is None else batch
        # One allocation, of the values, the exponents and the scales, in words (a tensor for each takes the
        # host 3 us more, with their release); views of it are made when they are asked for.
        values, exponents = n * rows * blocks * 32, n * ((blocks + 3) // 4) * ((rows + 127) // 128) * 128
        self._base = torch.empty(values + exponents + n * blocks * runs, dtype=torch.float32, device=device)
        self._q = self._scale = None
        at = self._base.data_ptr() if values else 0
        self._c = _Fp8Matrix(n, rows, cols, tile, code, at, at and at + 4 * values, at and at + 4 * (values + exponents))

    # (to be filled, not replaced: the calls have their addresses)
    @property
    def q(self) -> torch.Tensor:
        if self._q is None:
            r, c = self.rows, (self.cols + 127) // 128 * 128
            flat = self._base.view(_FP8_TYPE[self.fmt])
            self._q = flat.as_strided((r, c), (c, 1)) if self.batch is None else flat.as_strided((self.batch, r, c), (r * c, c, 1))
        return self._q

    @property
    def scale(self) -> torch.Tensor:
        if self._scale is None:
            flat, b = self._base, (self.cols + 127) // 128
            r = self.rows if self.tile == 1 else (self.rows + 127) // 128
            if self.batch is None:
                self._scale = flat.as_strided((b, r), (r, 1), flat.shape[0] - b * r)
            else:
                self._scale = flat.as_strided((self.batch, b, r), (b * r, r, 1), flat.shape[0] - self.batch * b * r)
        return self._scale

    @property
    def exponent(self) -> torch.Tensor:
        w, r = (self.cols + 511) // 512, (self.rows + 127) // 128
        flat, first = self._base.view(torch.uint8), self._c.batch * self.rows * ((self.cols + 127) // 128) * 128
        if self.batch is None:
            return flat.as_strided((w, r, 512), (r * 512, 512, 1), first)
        return flat.as_strided((self.batch, w, r, 512), (w * r * 512, r * 512, 512, 1), first)


def bsr_fp8_quantize(x: torch.Tensor, tile: int = 1, fmt: str = "e4m3", form: str = "rows", used: Optional[torch.Tensor] = None,
                     out=None, stream=None):
    """x [R, C] (or a batch of them) in 8 bits, with the least power of two that fits as
    each block's scale. form "rows": as it lies, an Fp8Matrix of [R, C]; "columns":
    transposed, of [C, R], its blocks along R (an operand of a product that sums over
    rows); "both": the two, from one reading. tile 128: blocks of 128 x 128, as for
    weights. used (device int32 [1], as ExpertOrder.used): rows from there on are not
    read. `out`: what to fill, as it would be returned."""
    shape = x.shape
    if len(shape) == 2:
        (R, C), batch = shape, None
    elif len(shape) == 3:
        batch, R, C = shape
    else:
        raise ValueError("x must be [R, C] or [batch, R, C]")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    dt = _DT.get(x.dtype)
    if dt is None:
        dt = dtype_code(x.dtype)   # (raises)
    if used is not None:
        _check_rows("used", used, (1,), torch.int32)
    if form not in ("rows", "columns", "both"):
        raise ValueError("form is 'rows', 'columns' or 'both'")
    rows = columns = None
    if out is None:
        device = x.device
        if form != "columns":
            rows = Fp8Matrix(R, C, tile, fmt, batch, device)
        if form != "rows":
            columns = Fp8Matrix(C, R, tile, fmt, batch, device)
        out = rows if columns is None else columns if rows is None else (rows, columns)
        if stream is not None:
            _lend(stream, device, *[m._base for m in (rows, columns) if m is not None])
    else:
        rows, columns = (out, None) if form == "rows" else (None, out) if form == "columns" else out
        for m, size in ((rows, (R, C)), (columns, (C, R))):
            if m is not None and (m.rows, m.cols, m.tile, m.fmt, m.batch) != (*size, tile, fmt, batch):
                raise ValueError("out is of other sizes")
    status = (_lib or load()).bsr_fp8_quantize(x.data_ptr(), dt, None if rows is None else rows._c, None if columns is None else columns._c,
                                               None if used is None else used.data_ptr(), _stream(stream))
    if status:
        _check(status, "bsr_fp8_quantize")
    return out


def bsr_fp8_product(a: Fp8Matrix, b: Fp8Matrix, bias: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
                    offsets: Optional[torch.Tensor] = None, over: str = "rows", Y: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """Y [a.rows, b.rows] = a b' + bias, of `dtype` (or that of a given Y).
    offsets (int32 [E + 1] on the device, as ExpertOrder.offsets): over "rows", b is a
    batch of E matrices and each run of a's rows meets its expert's (bias [E, b.rows];
    rows in no run are left as they were); over "columns", Y [E, a.rows, b.rows] has a
    sum over each run of columns, whose offsets are multiples of 128 (an order of align
    128) or the end: at any other the runs beside it are NaN, and bsr_check_status tells."""
    if over != "rows" and over != "columns":
        raise ValueError("over is 'rows' or 'columns'")
    if Y is not None:
        dtype = Y.dtype
    dt = _DT.get(dtype)
    if dt is None:
        dt = dtype_code(dtype)   # (raises)
    group, E, batch, shape = BSR_GROUP_NONE, 0, None, (a.rows, b.rows)
    if offsets is not None:
        E = offsets.shape[0] - 1
        _check_rows("offsets", offsets, (E + 1,), torch.int32)
        if over == "rows":
            group, batch = BSR_GROUP_ROWS, E
        else:
            group, shape = BSR_GROUP_COLUMNS, (E, a.rows, b.rows)
    elif over == "columns":
        raise ValueError("sums over runs of columns need offsets")
    if a.batch is not None or b.batch != batch:
        raise ValueError("a is one matrix, b one for each expert by rows, else one")
    if bias is not None:
        _check_rows("bias", bias, (b.rows,) if batch is None else (E, b.rows), torch.float32)
    if Y is None:
        Y = torch.empty(shape, dtype=dtype, device=a._base.device)
        _lend(stream, Y.device, Y)
    elif Y.shape != shape or not Y.is_contiguous():
        _check_rows("Y", Y, shape, dtype)
    lib, ac, bc, s = _lib or load(), a._c, b._c, _stream(stream)
    ptrs = (None if bias is None else bias.data_ptr(), Y.data_ptr(), dt, group, None if offsets is None else offsets.data_ptr(), E)
    # (most calls need no workspace: it is asked for when a call is refused for want of it)
    status = lib.bsr_fp8_product(ac, bc, *ptrs, None, 0, s)
    if status == BSR_ERR_CAPACITY:
        n = ctypes.c_size_t(0)
        _check(lib.bsr_fp8_product_workspace(ac, bc, dt, group, E, ctypes.byref(n)), "bsr_fp8_product_workspace")
        ws = _workspace(n.value, Y.device, stream)
        status = lib.bsr_fp8_product(ac, bc, *ptrs, ws.data_ptr(), n.value, s)
    if status:
        _check(status, "bsr_fp8_product")
    return Y


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
