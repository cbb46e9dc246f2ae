"""Thin ctypes binding of librecblr.so (the C ABI in include/recblr.h).

Two layers, both pure argument marshalling (every step of the computation runs
in the HIP kernels of librecblr.so):

* ``recblr_*`` functions mirror the C entry points one to one: they take raw
  device pointers (ints) and sizes and return the C status code.
* ``bdlru_scan_forward`` and friends take torch tensors that live on the GPU,
  check their shapes and dtypes, allocate outputs and workspace with torch,
  call the C entry point on the current HIP stream and raise on a non-zero
  status.

There is no fallback: if the library is missing or fails to load, importing
this module raises.  Build it first with ``python -m paper_2406_12580_amd.build``.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librecblr.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing; build it with `python -m paper_2406_12580_amd.build`")
_lib = ctypes.CDLL(LIB_PATH)

OK, ERR_INVALID_ARGUMENT, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_SCRATCH = 0, -1, -2, -3, -4, -5
F32, BF16 = 0, 1
(OP_SCAN_FORWARD, OP_SCAN_BACKWARD, OP_FORWARD, OP_BACKWARD, OP_STEP, OP_GATED_FORWARD,
 OP_GATED_BACKWARD, OP_SCAN_BACKWARD_METHOD) = range(8)
SCAN_CHUNKED, SCAN_SERIAL, SCAN_TREE = range(3)

EXPORTS = (
    "recblr_status_string", "recblr_workspace_size", "recblr_bdlru_scan_forward",
    "recblr_bdlru_scan_backward", "recblr_bdlru_scan_step", "recblr_bdlru_forward",
    "recblr_bdlru_backward", "recblr_bdlru_step", "recblr_linear_scan_forward",
    "recblr_scan_forward_method", "recblr_scan_backward_method", "recblr_gated_forward", "recblr_bdlru_scan_forward_timed",
    "recblr_bdlru_scan_backward_timed", "recblr_gated_backward", "recblr_model_param_count",
    "recblr_model_param_offsets", "recblr_model_workspace_size", "recblr_blas_create",
    "recblr_blas_destroy", "recblr_model_train_step", "recblr_adam_update",
    "recblr_bdlru_scan_backward_noalloc",
)

_p, _i64, _int, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
_f = ctypes.c_float


class ModelDims(ctypes.Structure):
    """recblr_model_dims."""
    _fields_ = [("B", _i64), ("T", _i64), ("D", _i64), ("E", _i64), ("V", _i64),
                ("layers", _i64), ("K", _int), ("ln_eps", _f)]


class ModelStepOpts(ctypes.Structure):
    """recblr_model_step_opts."""
    _fields_ = [("dropout", _f), ("pad_id", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("offset", ctypes.c_uint64)]


_pd = ctypes.POINTER(ModelDims)
_po = ctypes.POINTER(ModelStepOpts)
_SIGS = {
    "recblr_status_string": ([_int], ctypes.c_char_p),
    "recblr_workspace_size": ([_int, _i64, _i64, _i64, _int], _sz),
    "recblr_bdlru_scan_forward": ([_p] * 7 + [_i64] * 3 + [_int, _p, _sz, _p], _int),
    "recblr_bdlru_scan_backward": ([_p] * 13 + [_i64] * 3 + [_int, _p, _sz, _p], _int),
    "recblr_bdlru_scan_forward_timed": ([_p] * 7 + [_i64] * 3 + [_int, _p, _sz, _p, _p, _p], _int),
    "recblr_bdlru_scan_backward_timed": ([_p] * 13 + [_i64] * 3 + [_int, _p, _sz, _p, _p, _p],
                                         _int),
    "recblr_bdlru_scan_backward_noalloc": ([_p] * 13 + [_i64] * 3 + [_int, _p], _int),
    "recblr_bdlru_scan_step": ([_p] * 6 + [_i64] * 2 + [_int, _p], _int),
    "recblr_bdlru_forward": ([_p] * 9 + [_i64] * 3 + [_int, _p, _sz, _p], _int),
    "recblr_bdlru_backward": ([_p] * 17 + [_i64] * 3 + [_int, _p, _sz, _p], _int),
    "recblr_bdlru_step": ([_p] * 8 + [_i64] * 2 + [_int, _p, _sz, _p], _int),
    "recblr_linear_scan_forward": ([_p] * 5 + [_i64] * 3 + [_p], _int),
    "recblr_scan_forward_method": ([_int] + [_p] * 5 + [_i64] * 3 + [_int, _p, _sz, _p], _int),
    "recblr_scan_backward_method": ([_int] + [_p] * 10 + [_i64] * 3 + [_int, _p, _sz, _p],
                                    _int),
    "recblr_gated_forward": ([_p] * 4 + [_int] + [_p] * 9 + [_i64] * 3 + [_int, _p, _sz, _p],
                             _int),
    "recblr_gated_backward": ([_p] * 4 + [_int] + [_p] * 19 + [_i64] * 3 + [_int, _p, _sz, _p],
                              _int),
    "recblr_model_param_count": ([_pd], _sz),
    "recblr_model_param_offsets": ([_pd, _p, _i64], _i64),
    "recblr_model_workspace_size": ([_pd], _sz),
    "recblr_blas_create": ([ctypes.POINTER(_p)], _int),
    "recblr_blas_destroy": ([_p], _int),
    "recblr_model_train_step": ([_pd, _po] + [_p] * 6 + [_sz, _p, _p], _int),
    "recblr_adam_update": ([_p] * 4 + [_i64, _i64, _f, _f, _f, _f, _p], _int),
}
for _name, (_args, _res) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.argtypes = _args
    _fn.restype = _res
    globals()[_name] = _fn


class RecblrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {recblr_status_string(status).decode()} ({status})")


def _check(status: int, where: str):
    if status != OK:
        raise RecblrError(status, where)


# ------------------------------------------------------------------ torch-level helpers

def io_code(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return F32
    if dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported I/O dtype {dtype}; use float32 or bfloat16")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    # torch.cuda.current_stream().cuda_stream without the Stream object around it
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _on_stream(fn):
    """Run a wrapper with its `stream` argument as torch's current stream.

    The workspace and outputs are then allocated by torch's caching allocator
    on the stream the kernels are launched on, so the workspace, released when
    the wrapper returns, is handed out again only to later work on that same
    stream (which runs after the launched kernels).  Without a `stream`
    argument nothing changes: torch's current stream is the launch stream.
    """
    sig = inspect.signature(fn)
    pos = list(sig.parameters).index("stream")

    @functools.wraps(fn)
    def wrapper(*args, **kwargs):
        if len(args) <= pos and kwargs.get("stream") is None:
            return fn(*args, **kwargs)
        bound = sig.bind(*args, **kwargs)
        s = bound.arguments.get("stream")
        if s is None:
            return fn(*args, **kwargs)
        bound.arguments["stream"] = None
        with torch.cuda.stream(s):
            return fn(*bound.args, **bound.kwargs)
    return wrapper


_workspace_size = functools.lru_cache(maxsize=256)(recblr_workspace_size)  # a function of sizes


def _workspace(op: int, B: int, L: int, D: int, io: int, device):
    n = _workspace_size(op, B, L, D, io)
    if n == 0:
        return None, 0
    return torch.empty(n, dtype=torch.uint8, device=device), n


def _f32(t, shape, name):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape:
        raise ValueError(f"{name} must be float32 of shape {tuple(shape)}")
    return t


def _io(t, shape, dtype, name):
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}")
    return t


@_on_stream
def bdlru_scan_forward(x, zr, zi, lam, h0=None, stream=None):
    """Gated BD-LRU scan from pre-activations. Returns (h [B,L,D] io, hT [B,D] float32)."""
    B, L, D = x.shape
    io = io_code(x.dtype)
    _io(zr, x.shape, x.dtype, "zr"), _io(zi, x.shape, x.dtype, "zi")
    _f32(lam, (D,), "lambda"), _f32(h0, (B, D), "h0")
    h = torch.empty_like(x)
    hT = x.new_empty((B, D), dtype=torch.float32)
    ws, nws = _workspace(OP_SCAN_FORWARD, B, L, D, io, x.device)
    _check(recblr_bdlru_scan_forward(_ptr(x), _ptr(zr), _ptr(zi), _ptr(lam), _ptr(h0), _ptr(h),
                                     _ptr(hT), B, L, D, io, _ptr(ws), nws, _stream(stream)),
           "recblr_bdlru_scan_forward")
    return h, hT


@_on_stream
def bdlru_scan_backward(x, zr, zi, lam, h, dh, h0=None, dhT=None, stream=None):
    """Backward of bdlru_scan_forward. Returns dict dx, dzr, dzi, dlambda, dh0."""
    B, L, D = x.shape
    io = io_code(x.dtype)
    for t, n in ((zr, "zr"), (zi, "zi"), (h, "h"), (dh, "dh")):
        _io(t, x.shape, x.dtype, n)
    _f32(lam, (D,), "lambda"), _f32(h0, (B, D), "h0"), _f32(dhT, (B, D), "dhT")
    out = {k: torch.empty_like(x) for k in ("dx", "dzr", "dzi")}
    out["dlambda"] = x.new_empty(D, dtype=torch.float32)
    out["dh0"] = x.new_empty((B, D), dtype=torch.float32)
    ws, nws = _workspace(OP_SCAN_BACKWARD, B, L, D, io, x.device)
    _check(recblr_bdlru_scan_backward(
        _ptr(x), _ptr(zr), _ptr(zi), _ptr(lam), _ptr(h0), _ptr(h), _ptr(dh), _ptr(dhT),
        _ptr(out["dx"]), _ptr(out["dzr"]), _ptr(out["dzi"]), _ptr(out["dlambda"]),
        _ptr(out["dh0"]), B, L, D, io, _ptr(ws), nws, _stream(stream)),
        "recblr_bdlru_scan_backward")
    return out


@_on_stream
def bdlru_scan_step(x, zr, zi, lam, h_prev, out=None, stream=None):
    """One recurrent step over [B, D]; returns h_next (float32). out may be h_prev."""
    B, D = x.shape
    io = io_code(x.dtype)
    _io(zr, x.shape, x.dtype, "zr"), _io(zi, x.shape, x.dtype, "zi")
    _f32(lam, (D,), "lambda"), _f32(h_prev, (B, D), "h_prev")
    h_next = torch.empty((B, D), dtype=torch.float32, device=x.device) if out is None else out
    _check(recblr_bdlru_scan_step(_ptr(x), _ptr(zr), _ptr(zi), _ptr(lam), _ptr(h_prev),
                                  _ptr(h_next), B, D, io, _stream(stream)),
           "recblr_bdlru_scan_step")
    return h_next


@_on_stream
def bdlru_forward(x, Wr, br, Wi, bi, lam, h0=None, stream=None):
    """Full forward with gate projections. Returns (h, hT)."""
    B, L, D = x.shape
    io = io_code(x.dtype)
    for t, n in ((Wr, "Wr"), (Wi, "Wi")):
        _io(t, (D, D), x.dtype, n)
    for t, n in ((br, "br"), (bi, "bi")):
        if t is not None:
            _io(t, (D,), x.dtype, n)
    _f32(lam, (D,), "lambda"), _f32(h0, (B, D), "h0")
    h = torch.empty_like(x)
    hT = torch.empty((B, D), dtype=torch.float32, device=x.device)
    ws, nws = _workspace(OP_FORWARD, B, L, D, io, x.device)
    _check(recblr_bdlru_forward(_ptr(x), _ptr(Wr), _ptr(br), _ptr(Wi), _ptr(bi), _ptr(lam),
                                _ptr(h0), _ptr(h), _ptr(hT), B, L, D, io, _ptr(ws), nws,
                                _stream(stream)), "recblr_bdlru_forward")
    return h, hT


@_on_stream
def bdlru_backward(x, Wr, br, Wi, bi, lam, h, dh, h0=None, dhT=None, stream=None):
    """Full backward. Returns dict dx, dWr, dbr, dWi, dbi, dlambda, dh0."""
    B, L, D = x.shape
    io = io_code(x.dtype)
    for t, n in ((Wr, "Wr"), (Wi, "Wi")):
        _io(t, (D, D), x.dtype, n)
    _io(h, x.shape, x.dtype, "h"), _io(dh, x.shape, x.dtype, "dh")
    _f32(lam, (D,), "lambda"), _f32(h0, (B, D), "h0"), _f32(dhT, (B, D), "dhT")
    f32 = dict(dtype=torch.float32, device=x.device)
    out = {"dx": torch.empty_like(x), "dWr": torch.empty((D, D), **f32),
           "dbr": torch.empty(D, **f32), "dWi": torch.empty((D, D), **f32),
           "dbi": torch.empty(D, **f32), "dlambda": torch.empty(D, **f32),
           "dh0": torch.empty((B, D), **f32)}
    ws, nws = _workspace(OP_BACKWARD, B, L, D, io, x.device)
    _check(recblr_bdlru_backward(
        _ptr(x), _ptr(Wr), _ptr(br), _ptr(Wi), _ptr(bi), _ptr(lam), _ptr(h0), _ptr(h), _ptr(dh),
        _ptr(dhT), _ptr(out["dx"]), _ptr(out["dWr"]), _ptr(out["dbr"]), _ptr(out["dWi"]),
        _ptr(out["dbi"]), _ptr(out["dlambda"]), _ptr(out["dh0"]), B, L, D, io, _ptr(ws), nws,
        _stream(stream)), "recblr_bdlru_backward")
    return out


@_on_stream
def bdlru_step(x, Wr, br, Wi, bi, lam, h_prev, out=None, stream=None):
    """Full single step with gate projections; returns h_next (float32)."""
    B, D = x.shape
    io = io_code(x.dtype)
    _f32(lam, (D,), "lambda"), _f32(h_prev, (B, D), "h_prev")
    h_next = torch.empty((B, D), dtype=torch.float32, device=x.device) if out is None else out
    ws, nws = _workspace(OP_STEP, B, 1, D, io, x.device)
    _check(recblr_bdlru_step(_ptr(x), _ptr(Wr), _ptr(br), _ptr(Wi), _ptr(bi), _ptr(lam),
                             _ptr(h_prev), _ptr(h_next), B, D, io, _ptr(ws), nws,
                             _stream(stream)), "recblr_bdlru_step")
    return h_next


@_on_stream
def linear_scan_forward(a, u, h0=None, stream=None):
    """Raw recurrence h_t = a_t h_{t-1} + u_t (float32). Returns (h, hT)."""
    B, L, D = a.shape
    h = torch.empty_like(a)
    hT = torch.empty((B, D), dtype=torch.float32, device=a.device)
    _check(recblr_linear_scan_forward(_ptr(a), _ptr(u), _ptr(h0), _ptr(h), _ptr(hT), B, L, D,
                                      _stream(stream)), "recblr_linear_scan_forward")
    return h, hT


@_on_stream
def scan_backward_method(method, x, zr, zi, lam, h, dh, stream=None):
    """Gated scan backward (zero initial state, no dL/dh_T) by one of SCAN_CHUNKED,
    SCAN_SERIAL, SCAN_TREE. Returns dict dx, dzr, dzi (dtype of x), dlambda (float32)."""
    B, L, D = x.shape
    io = io_code(x.dtype)
    out = {"dx": torch.empty_like(x), "dzr": torch.empty_like(x), "dzi": torch.empty_like(x),
           "dlambda": torch.empty(D, dtype=torch.float32, device=x.device)}
    ws, nws = _workspace(OP_SCAN_BACKWARD_METHOD, B, L, D, io, x.device)
    _check(recblr_scan_backward_method(method, _ptr(x), _ptr(zr), _ptr(zi), _ptr(lam), _ptr(h),
                                       _ptr(dh), _ptr(out["dx"]), _ptr(out["dzr"]),
                                       _ptr(out["dzi"]), _ptr(out["dlambda"]), B, L, D, io,
                                       _ptr(ws), nws, _stream(stream)),
           "recblr_scan_backward_method")
    return out


@_on_stream
def scan_forward_method(method, x, zr, zi, lam, stream=None):
    """Gated scan forward (zero initial state) by one of SCAN_CHUNKED, SCAN_SERIAL,
    SCAN_TREE (the efficiency-ablation variants). Returns h."""
    B, L, D = x.shape
    io = io_code(x.dtype)
    h = torch.empty_like(x)
    ws, nws = _workspace(OP_SCAN_FORWARD, B, L, D, io, x.device)
    _check(recblr_scan_forward_method(method, _ptr(x), _ptr(zr), _ptr(zi), _ptr(lam), _ptr(h),
                                      B, L, D, io, _ptr(ws), nws, _stream(stream)),
           "recblr_scan_forward_method")
    return h


@_on_stream
def gated_forward(hx, hz, conv_w, conv_b, Wr, br, Wi, bi, lam, h0=None, keep_h=True,
                  stream=None):
    """Gated recurrent layer core: y = BD-LRU(SiLU(conv(hx))) * SiLU(hz).
    conv_w is [D][K] float32. Returns (y, h, hT) (h is None unless keep_h)."""
    B, L, D = hx.shape
    K = conv_w.shape[1]
    io = io_code(hx.dtype)
    y = torch.empty_like(hx)
    h = torch.empty_like(hx) if keep_h else None
    hT = torch.empty((B, D), dtype=torch.float32, device=hx.device)
    ws, nws = _workspace(OP_GATED_FORWARD, B, L, D, io, hx.device)
    _check(recblr_gated_forward(_ptr(hx), _ptr(hz), _ptr(conv_w), _ptr(conv_b), K, _ptr(Wr),
                                _ptr(br), _ptr(Wi), _ptr(bi), _ptr(lam), _ptr(h0), _ptr(y),
                                _ptr(h), _ptr(hT), B, L, D, io, _ptr(ws), nws, _stream(stream)),
           "recblr_gated_forward")
    return y, h, hT


@_on_stream
def gated_backward(hx, hz, conv_w, conv_b, Wr, br, Wi, bi, lam, h, dy, h0=None, dhT=None,
                   stream=None):
    """Backward of gated_forward (h: its BD-LRU output).  Returns a dict with dhx,
    dhz, dconv_w [D][K], dconv_b (None without a conv bias), dWr, dbr, dWi, dbi,
    dlambda, dh0 (None without h0)."""
    B, L, D = hx.shape
    K = conv_w.shape[1]
    io = io_code(hx.dtype)
    f32 = dict(dtype=torch.float32, device=hx.device)
    out = {"dhx": torch.empty_like(hx), "dhz": torch.empty_like(hx),
           "dconv_w": torch.empty((D, K), **f32),
           "dconv_b": torch.empty(D, **f32) if conv_b is not None else None,
           "dWr": torch.empty((D, D), **f32), "dbr": torch.empty(D, **f32),
           "dWi": torch.empty((D, D), **f32), "dbi": torch.empty(D, **f32),
           "dlambda": torch.empty(D, **f32),
           "dh0": torch.empty((B, D), **f32) if h0 is not None else None}
    ws, nws = _workspace(OP_GATED_BACKWARD, B, L, D, io, hx.device)
    _check(recblr_gated_backward(
        _ptr(hx), _ptr(hz), _ptr(conv_w), _ptr(conv_b), K, _ptr(Wr), _ptr(br), _ptr(Wi),
        _ptr(bi), _ptr(lam), _ptr(h0), _ptr(h), _ptr(dy), _ptr(dhT), _ptr(out["dhx"]),
        _ptr(out["dhz"]), _ptr(out["dconv_w"]), _ptr(out["dconv_b"]), _ptr(out["dWr"]),
        _ptr(out["dbr"]), _ptr(out["dWi"]), _ptr(out["dbi"]), _ptr(out["dlambda"]),
        _ptr(out["dh0"]), B, L, D, io, _ptr(ws), nws, _stream(stream)), "recblr_gated_backward")
    return out


# ------------------------------------------------------------------ full model step

def model_dims(B, T, D, E=2, V=3416, layers=2, K=4, eps=1e-12) -> ModelDims:
    return ModelDims(B, T, D, E, V, layers, K, eps)


def model_param_offsets(dims: ModelDims):
    """Offsets (floats) of the flat parameter tensors, in the documented order."""
    n = recblr_model_param_offsets(ctypes.byref(dims), None, 0)
    if n < 0:
        raise RecblrError(ERR_UNSUPPORTED, "recblr_model_param_offsets")
    arr = (ctypes.c_int64 * n)()
    recblr_model_param_offsets(ctypes.byref(dims), arr, n)
    return list(arr)


class ModelStep:
    """One training step of the full model on the GPU: holds the rocBLAS handle
    and the workspace for fixed dimensions."""

    def __init__(self, dims: ModelDims, device="cuda"):
        self.dims = dims
        self.count = recblr_model_param_count(ctypes.byref(dims))
        if self.count == 0:
            raise RecblrError(ERR_UNSUPPORTED, "recblr_model_param_count")
        n = recblr_model_workspace_size(ctypes.byref(dims))
        if n == 0:
            raise RecblrError(ERR_UNSUPPORTED, "recblr_model_workspace_size")
        self.ws = torch.empty(n, dtype=torch.uint8, device=device)
        h = _p()
        _check(recblr_blas_create(ctypes.byref(h)), "recblr_blas_create")
        self.blas = h

    def close(self):
        if self.blas is not None:
            recblr_blas_destroy(self.blas)
            self.blas = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @_on_stream
    def train_step(self, params, ids, targets, grads=None, loss=None, dropout=0.0, seed=0,
                   offset=0, pad_id=-1, stream=None):
        """Loss and gradients (flat, the parameter layout) of one batch; dropout
        with drop probability `dropout` and Philox key (seed, offset), left
        padding with id pad_id (-1: none)."""
        if grads is None:
            grads = torch.empty_like(params)
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=params.device)
        opts = ModelStepOpts(dropout, pad_id, seed, offset)
        _check(recblr_model_train_step(ctypes.byref(self.dims), ctypes.byref(opts), _ptr(params),
                                       _ptr(ids), _ptr(targets), _ptr(grads), _ptr(loss),
                                       _ptr(self.ws), self.ws.numel(), self.blas,
                                       _stream(stream)),
               "recblr_model_train_step")
        return loss, grads


@_on_stream
def adam_update(params, grads, m1, m2, step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                stream=None):
    _check(recblr_adam_update(_ptr(params), _ptr(grads), _ptr(m1), _ptr(m2), params.numel(),
                              step, lr, beta1, beta2, eps, _stream(stream)), "recblr_adam_update")



# ------------------------------------------------------------------ recblr_ops.h

OP_DELTA_FORWARD, OP_DELTA_BACKWARD = 16, 17
DELTA_CHUNK = 64
ADAMW_BLOCK = 256

OPS_EXPORTS = (
    "recblr_delta_workspace_size", "recblr_delta_forward", "recblr_delta_backward",
    "recblr_delta_step", "recblr_adamw_update", "recblr_adamw_moments",
    "recblr_sample_workspace_size", "recblr_sample",
)


class AdamWTensor(ctypes.Structure):
    """recblr_adamw_tensor."""
    _fields_ = [("param", _p), ("grad", _p), ("m1", _p), ("m2", _p), ("scale1", _p),
                ("scale2", _p), ("n", _i64), ("weight_decay", ctypes.c_double)]


_d = ctypes.c_double
_OPS_SIGS = {
    "recblr_delta_workspace_size": ([_int] + [_i64] * 6 + [_int], _sz),
    "recblr_delta_forward": ([_p] * 9 + [_i64] * 6 + [_f, _int, _p, _sz, _p], _int),
    "recblr_delta_backward": ([_p] * 14 + [_i64] * 6 + [_f, _int, _p, _sz, _p], _int),
    "recblr_delta_step": ([_p] * 8 + [_i64] * 5 + [_f, _int, _p], _int),
    "recblr_adamw_update": ([ctypes.POINTER(AdamWTensor), _i64, _int, _int, _i64, _d, _d, _d, _d,
                             _p], _int),
    "recblr_adamw_moments": ([ctypes.POINTER(AdamWTensor), _i64, _p, _p, _p], _int),
    "recblr_sample_workspace_size": ([_i64, _i64, _int], _sz),
    "recblr_sample": ([_p] * 8 + [_i64, _i64, _int, _p, _sz, _p], _int),
}
for _name, (_args, _res) in _OPS_SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.argtypes = _args
    _fn.restype = _res
    globals()[_name] = _fn


def _on_device(fn):
    """Run a wrapper on the device of its first tensor and on its `stream` argument.

    The library launches on the current device; outputs and workspace come from
    torch's allocator on the stream of the launch, as in _on_stream.
    """
    name = next(iter(inspect.signature(fn).parameters))

    @functools.wraps(fn)
    def wrapper(*args, stream=None, **kwargs):
        if not args and name not in kwargs:
            raise TypeError(f"{fn.__name__}() needs the argument {name}")
        dev = (args[0] if args else kwargs[name]).device
        if dev.type != "cuda":
            raise ValueError("tensors must live on the GPU")
        if stream is None and dev.index == torch._C._cuda_getDevice():
            return fn(*args, **kwargs)
        if stream is not None and stream.device != dev:
            raise ValueError("stream belongs to another device than the tensors")
        with torch.cuda.device(dev), torch.cuda.stream(stream):
            return fn(*args, **kwargs)
    return wrapper


def _arg(t, shape, dtype, index, name):
    """The address of a tensor that has to be as described, on the GPU `index`; None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}")
    if t.get_device() != index or index < 0:
        raise ValueError(f"{name} must live on the GPU, with the other tensors")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _delta_heads(q, k, v):
    """Checked sizes (H, HV, Dk, Dv) and scale of the gated delta rule's tensors."""
    if q.dim() < 3 or v.dim() != q.dim() or q.shape[:-2] != v.shape[:-2]:
        raise ValueError("q and v must have the same rows and steps, and a head axis")
    H, Dk, HV, Dv = *q.shape[-2:], *v.shape[-2:]
    if H < 1 or HV < 1 or HV % H:
        raise ValueError("the number of value heads must be a multiple of the query heads")
    return H, HV, Dk, Dv


_delta_workspace_size = functools.lru_cache(maxsize=256)(recblr_delta_workspace_size)


def _delta_inputs(q, k, v, g, beta):
    """Checked sizes and the addresses of a sequence's tensors."""
    if q.dim() != 4:
        raise ValueError("q must be [B, L, H, Dk]")
    H, HV, Dk, Dv = _delta_heads(q, k, v)
    B, L = q.shape[:2]
    dt, at = q.dtype, q.get_device()
    io = io_code(dt)
    ptrs = (_arg(q, (B, L, H, Dk), dt, at, "q"), _arg(k, (B, L, H, Dk), dt, at, "k"),
            _arg(v, (B, L, HV, Dv), dt, at, "v"), _arg(g, (B, L, HV), dt, at, "g"),
            _arg(beta, (B, L, HV), dt, at, "beta"))
    return (B, L, H, HV, Dk, Dv), io, ptrs


def _delta_workspace(op, sizes, io, device):
    n = _delta_workspace_size(op, *sizes, io)
    return (torch.empty(n, dtype=torch.uint8, device=device) if n else None), n


@_on_device
def delta_forward(q, k, v, g, beta, h0=None, scale=None, keep_states=False):
    """Gated delta rule over whole sequences: q, k [B,L,H,Dk], v [B,L,HV,Dv], log decays g and
    strengths beta [B,L,HV], h0 [B,HV,Dk,Dv] float32.  Returns (o [B,L,HV,Dv], hT float32,
    states), states (None unless keep_states) being what delta_backward needs of the forward:
    [B,HV,ceil(L/64),Dk,Dv] float32.  scale defaults to Dk ** -0.5.  Padded steps (g = beta = 0)
    leave the state alone; their q, k and v must be finite, like all inputs."""
    sizes, io, ptrs = _delta_inputs(q, k, v, g, beta)
    B, L, H, HV, Dk, Dv = sizes
    dev, at, f32 = q.device, q.get_device(), torch.float32
    o = torch.empty_like(v)
    hT = torch.empty((B, HV, Dk, Dv), dtype=f32, device=dev)
    states = torch.empty((B, HV, -(-L // DELTA_CHUNK), Dk, Dv), dtype=f32, device=dev) \
        if keep_states else None
    ws, nws = _delta_workspace(OP_DELTA_FORWARD, sizes, io, dev)
    _check(recblr_delta_forward(
        *ptrs, _arg(h0, (B, HV, Dk, Dv), f32, at, "h0"), o.data_ptr(), hT.data_ptr(),
        states.data_ptr() if keep_states else None, *sizes,
        Dk ** -0.5 if scale is None else scale, io, ws.data_ptr() if nws else None, nws,
        _stream()), "recblr_delta_forward")
    return o, hT, states


@_on_device
def delta_backward(q, k, v, g, beta, states, do, dhT=None, scale=None, need_dh0=True):
    """Backward of delta_forward (states: what it kept).  Returns a dict with dq, dk, dv, dg,
    dbeta of the inputs' types and dh0 float32 (None unless need_dh0)."""
    sizes, io, ptrs = _delta_inputs(q, k, v, g, beta)
    B, L, H, HV, Dk, Dv = sizes
    dev, at, f32 = q.device, q.get_device(), torch.float32
    st = (B, HV, Dk, Dv)
    out = {"dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v),
           "dg": torch.empty_like(g), "dbeta": torch.empty_like(beta),
           "dh0": torch.empty(st, dtype=f32, device=dev) if need_dh0 else None}
    ws, nws = _delta_workspace(OP_DELTA_BACKWARD, sizes, io, dev)
    _check(recblr_delta_backward(
        *ptrs, _arg(states, (B, HV, -(-L // DELTA_CHUNK), Dk, Dv), f32, at, "states"),
        _arg(do, (B, L, HV, Dv), q.dtype, at, "do"), _arg(dhT, st, f32, at, "dhT"),
        *(None if t is None else t.data_ptr() for t in out.values()), *sizes,
        Dk ** -0.5 if scale is None else scale, io, ws.data_ptr() if nws else None, nws,
        _stream()), "recblr_delta_backward")
    return out


@_on_device
def delta_step(q, k, v, g, beta, h_prev, out=None, scale=None):
    """One token of the gated delta rule: q, k [B,H,Dk], v [B,HV,Dv], g, beta [B,HV],
    h_prev [B,HV,Dk,Dv] float32.  Returns (o [B,HV,Dv], h_next float32); out, where the new
    state goes, may be h_prev.  scale defaults to Dk ** -0.5."""
    if q.dim() != 3:
        raise ValueError("q must be [B, H, Dk]")
    H, HV, Dk, Dv = _delta_heads(q, k, v)
    B, io, dt, at = q.shape[0], io_code(q.dtype), q.dtype, q.get_device()
    st = (B, HV, Dk, Dv)
    o = torch.empty_like(v)
    h_next = torch.empty_like(h_prev) if out is None else out
    _check(recblr_delta_step(
        _arg(q, (B, H, Dk), dt, at, "q"), _arg(k, (B, H, Dk), dt, at, "k"),
        _arg(v, (B, HV, Dv), dt, at, "v"), _arg(g, (B, HV), dt, at, "g"),
        _arg(beta, (B, HV), dt, at, "beta"), _arg(h_prev, st, torch.float32, at, "h_prev"),
        o.data_ptr(), _arg(h_next, st, torch.float32, at, "out"), B, H, HV, Dk, Dv,
        Dk ** -0.5 if scale is None else scale, io, _stream()), "recblr_delta_step")
    return o, h_next


@_on_device
def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """One item a row of logits [B,V], chosen by u [B] (float32, in [0, 1)).

    temperature, top_p, min_p (float32) and top_k (int32) are [B] tensors or None (1, 1, 0
    and no limit).  Returns (ids [B] int32, prob [B] float32): the item, -1 for a row that has
    none, and its probability among the items that stayed."""
    if logits.dim() != 2:
        raise ValueError("logits must be [B, V]")
    B, V = logits.shape
    io, dev, at, f32 = io_code(logits.dtype), logits.device, logits.get_device(), torch.float32
    ids = torch.empty(B, dtype=torch.int32, device=dev)
    prob = torch.empty(B, dtype=f32, device=dev)
    n = recblr_sample_workspace_size(B, V, io)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _check(recblr_sample(
        _arg(logits, (B, V), logits.dtype, at, "logits"), _arg(u, (B,), f32, at, "u"),
        _arg(temperature, (B,), f32, at, "temperature"),
        _arg(top_k, (B,), torch.int32, at, "top_k"), _arg(top_p, (B,), f32, at, "top_p"),
        _arg(min_p, (B,), f32, at, "min_p"), ids.data_ptr(), prob.data_ptr(), B, V, io,
        ws.data_ptr() if n else None, n, _stream()), "recblr_sample")
    return ids, prob


# A list of tensors is checked by these in a map each: half the time of a loop over attributes,
# and a step over a model's few dozen tensors is bound by them.
_numel, _data_ptr = torch.Tensor.numel, torch.Tensor.data_ptr
_get_device, _is_contiguous = torch.Tensor.get_device, torch.Tensor.is_contiguous
_dtype, _nbytes = torch.Tensor.dtype.__get__, torch.Tensor.nbytes.__get__


class AdamW:
    """AdamW over a list of tensors (float32 or bfloat16, all of one type and device).

    weight_decay is one number or one for each tensor.  state_bits = 32 keeps float32 moments
    m1, m2; 8 keeps codes (m1 int8, m2 uint8) with a float32 scale for each 256 elements (s1,
    s2).  `state` takes over moments that exist: (m1, m2) or (m1, m2, s1, s2), lists of tensors
    with as many elements as the parameters (the scales ceil(n / 256)); `step` counts the
    updates already made.  step(grads) updates parameters and moments in place, on the
    parameters' device; gradients have the parameters' type and number of elements.  The lists
    and their tensors may be given other memory of the same type and size between two calls
    (opt.m1[i] = t, p.data = t).  A captured step replays with the bias corrections, rates and
    addresses of its capture."""

    def __init__(self, params, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
                 state_bits=32, state=None, step=0):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.dtype, self.device = self.params[0].dtype, self.params[0].device
        if not self.params[0].is_cuda:
            raise ValueError("tensors must live on the GPU")
        self._io = io_code(self.dtype)
        self.lr, self.beta1, self.beta2, self.eps = lr, beta1, beta2, eps
        self.state_bits, self.steps = state_bits, step
        sizes = [p.numel() for p in self.params]
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) \
            else [weight_decay] * len(sizes)
        if len(decay) != len(sizes):
            raise ValueError("weight_decay must be a number or one for each parameter")
        codes = state_bits == 8
        types = (torch.int8, torch.uint8) if codes else (torch.float32, torch.float32)
        blocks = [-(-n // ADAMW_BLOCK) for n in sizes]
        if state is None:
            def zeros(counts, dtype):
                return [torch.zeros(n, dtype=dtype, device=self.device) for n in counts]
            state = [zeros(sizes, t) for t in types]
            state += [zeros(blocks, torch.float32) for _ in range(2)] if codes else []
        if len(state) != (4 if codes else 2):
            raise ValueError("state must be (m1, m2), with (s1, s2) too for 8 bits")
        state = [list(s) for s in state]
        self.m1, self.m2 = state[:2]
        self.s1, self.s2 = state[2:] if codes else (None, None)
        self._table = (AdamWTensor * len(sizes))()
        self._sizes = sizes
        # The table's fields with the attributes that hold their tensors.
        self._fields = [("param", "params", self.dtype, sizes), ("m1", "m1", types[0], sizes),
                        ("m2", "m2", types[1], sizes)]
        if codes:
            self._fields += [("scale1", "s1", torch.float32, blocks),
                             ("scale2", "s2", torch.float32, blocks)]
        self._param_bytes = list(map(_nbytes, self.params))
        self._fill()
        for entry, n, w in zip(self._table, sizes, decay):
            entry.n, entry.weight_decay = n, w
        # The table's gradient addresses, as one array to assign.
        self._grads = np.frombuffer(self._table, dtype=np.uint64).reshape(len(sizes), -1)[
            :, AdamWTensor.grad.offset // 8]

    def _flat(self, t, dtype, n, name):
        if t.dtype != dtype or t.numel() != n:
            raise ValueError(f"{name}: a tensor must be {dtype} with {n} elements")
        if t.device != self.device or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name}: tensors must be contiguous, on the parameters' GPU")
        return t.data_ptr()

    def _addresses(self):
        return [list(map(_data_ptr, getattr(self, name))) for _, name, _, _ in self._fields]

    def _fill(self):
        held, found = [], []
        for field, name, dtype, counts in self._fields:
            tensors = getattr(self, name)
            if len(tensors) != len(self._sizes):
                raise ValueError(f"{name}: one tensor for each parameter is needed")
            found.append([self._flat(t, dtype, n, name) for t, n in zip(tensors, counts)])
            if field != "param":
                held += [t.detach() for t in tensors]
        for (field, *_), addresses in zip(self._fields, found):  # all are right: none is kept else
            for entry, address in zip(self._table, addresses):
                setattr(entry, field, address)
        # Moments' memory stays theirs for as long as the table names it, whatever becomes of the
        # tensors: an address that is the same as before is then the same memory.  Parameters'
        # memory is their owner's to free.
        self._held, self._at = held, found

    def _follow(self):
        """Brings the table in line with memory that was replaced since the last call."""
        if not (self._addresses() == self._at and all(map(_is_contiguous, self.params))
                and list(map(_nbytes, self.params)) == self._param_bytes):
            self._fill()

    def step(self, grads, lr=None, stream=None):
        """One update with grads, a tensor for each parameter; lr overrides the rate."""
        if len(grads) != len(self._sizes):
            raise ValueError("grads: one tensor for each parameter is needed")
        if not (list(map(_numel, grads)) == self._sizes and all(map(_is_contiguous, grads))
                and set(map(_get_device, grads)) == {self.device.index}
                and set(map(_dtype, grads)) == {self.dtype}):
            for t, n in zip(grads, self._sizes):
                self._flat(t, self.dtype, n, "grads")  # says what is wrong
        self._grads[:] = list(map(_data_ptr, grads))
        self._follow()
        _adamw_step(self, self.lr if lr is None else lr, stream=stream)
        self.steps += 1

    def moments(self, out=None, stream=None):
        """The moments as float32: (m1, m2), lists of tensors; out, two lists of float32 tensors
        with the parameters' numbers of elements, takes them where given (without it, 32-bit
        moments are the optimiser's own tensors, no copies)."""
        if self.state_bits == 32 and out is None:
            return list(self.m1), list(self.m2)
        self._follow()
        return _adamw_moments(self, out, stream=stream)


@_on_device
def _adamw_step(opt, lr):
    _check(recblr_adamw_update(opt._table, len(opt._sizes), opt.state_bits, opt._io,
                               opt.steps + 1, lr, opt.beta1, opt.beta2, opt.eps, _stream()),
           "recblr_adamw_update")


@_on_device
def _adamw_moments(opt, out):
    if out is None:
        out = tuple([torch.empty(p.shape, dtype=torch.float32, device=opt.device)
                     for p in opt.params] for _ in range(2))
    if len(out) != 2:
        raise ValueError("out must be two lists of tensors")
    ptrs = []
    for tensors in out:
        if len(tensors) != len(opt._sizes):
            raise ValueError("out: one tensor for each parameter is needed")
        ptrs.append((_p * len(tensors))(*(opt._flat(t, torch.float32, n, "out")
                                          for t, n in zip(tensors, opt._sizes))))
    if opt.state_bits == 32:
        for ours, theirs in zip((opt.m1, opt.m2), out):
            for a, b in zip(ours, theirs):
                b.view(-1).copy_(a.view(-1))
        return out
    _check(recblr_adamw_moments(opt._table, len(opt._sizes), *ptrs, _stream()),
           "recblr_adamw_moments")
    return out
