"""Thin Python binding over include/mxq_layers.h: the layers of a language model around its microscaled tensors.

As in mxq.py: argument marshalling only, on tensors that live on the GPU, enqueued on the current stream; nothing is
computed here and there is no CPU fallback.  Gradients are calls of their own (the operators do not record for
autograd; mlp.py wraps them).  Tensors made by a call are allocated on the current stream, workspaces on the stream
that the call is enqueued on.  As for any tensor of torch, a caller who passes another stream makes it wait for the
current one before the call and records it on the outputs after.

As there, each call has a native form (csrc/layers_binding.cpp, built as _mxq_layer_calls.so) that is asked first and
declines, before it has done anything, whatever is not plain; the Python form below is the definition of the call.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
from typing import NamedTuple

import torch

from . import mxq
from .mxq import _check, _done, _dtype_code, _need, _stream_ptr

Q8_BLOCK = 32
SUMS_F32, SUMS_MX = 0, 1                # how linear may hold its sums


class Q8(NamedTuple):
    """A [rows, cols] tensor in 8 bits: E4M3 elements and one power-of-two scale for 32 elements of a row.  The value of an
    element is codes * scales."""
    codes: torch.Tensor                 # float8_e4m3fn [rows, cols]
    scales: torch.Tensor                # float8_e8m0fnu [rows, cols / 32]

    def float(self) -> torch.Tensor:
        """The values in fp32 (plain torch, for inspection)."""
        rows, cols = self.codes.shape
        return (self.codes.float().view(rows, -1, Q8_BLOCK) * self.scales.float().unsqueeze(2)).view(rows, cols)


class W4(NamedTuple):
    """Weights [n, k] as mxq.quantize (or quantize_hier) returns them, with what they were quantised by."""
    codes: torch.Tensor                 # uint8 [n, k / 2]
    scales: torch.Tensor                # uint8 [n, k / block]
    block: int
    scale_fmt: int
    tensor_scale: float | torch.Tensor = 1.0        # or the one-element fp32 tensor of quantize_hier


class Adapters(NamedTuple):
    """Low-rank adapters of one projection: adapter i adds scaling[i] * (x A_i^T) B_i^T.  Smaller ranks are padded with zeros."""
    a: torch.Tensor                     # bfloat16 [count, rank, k]
    b: torch.Tensor                     # bfloat16 [count, n, rank]
    scaling: torch.Tensor               # float32 [count]


class SavedNorm(NamedTuple):
    """What add_rmsnorm keeps for its backward pass: the normalised rows before the weight, and 1 / rms of each."""
    n: Q8
    rstd: torch.Tensor                  # float32 [rows]


class SavedSwiglu(NamedTuple):
    gate: Q8
    up: Q8


class _Linear(ctypes.Structure):
    """struct mxq_linear_args of include/mxq_layers.h"""
    _fields_ = [("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64), ("x_codes", ctypes.c_void_p), ("x_scales", ctypes.c_void_p),
                ("m", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("w_codes", ctypes.c_void_p), ("w_scales", ctypes.c_void_p), ("block", ctypes.c_int), ("scale_fmt", ctypes.c_int),
                ("tensor_scale", ctypes.c_float), ("tensor_scale_dev", ctypes.c_void_p),
                ("adapter_a", ctypes.c_void_p), ("adapter_b", ctypes.c_void_p), ("adapter_scaling", ctypes.c_void_p),
                ("adapter_ids", ctypes.c_void_p), ("adapter_count", ctypes.c_int), ("adapter_rank", ctypes.c_int),
                ("y", ctypes.c_void_p), ("ld_y", ctypes.c_int64), ("y_dtype", ctypes.c_int),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("sums", ctypes.c_int)]


_lib = None
_calls = None                            # native forms of the calls, once the library is loaded


def _native_calls(L: ctypes.CDLL):
    """The module of native calls on the loaded library; None where it has not been built, or was built for another
    interpreter, torch or header: the Python forms then do all the work."""
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_mxq_layer_calls.so")
    try:
        loader = importlib.machinery.ExtensionFileLoader("_mxq_layer_calls", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_mxq_layer_calls", path, loader=loader))
        loader.exec_module(module)
        header = ctypes.string_at(ctypes.addressof(ctypes.c_char.in_dll(L, "mxq_layers_header_id"))).decode()
    except (ImportError, ValueError):
        return None
    if module.built_for() != (mxq.calls_abi(), header):
        return None
    module.use(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.mxq_add_rmsnorm, L.mxq_add_rmsnorm_backward, L.mxq_add_rmsnorm_backward_workspace_size, L.mxq_swiglu,
        L.mxq_swiglu_backward, L.mxq_linear, L.mxq_linear_workspace_size)), Q8, SavedNorm, SavedSwiglu)
    return module


def _layers() -> ctypes.CDLL:
    global _lib, _calls
    if _lib is not None:
        return _lib
    L = mxq.lib()
    i64, i32, f32, vp, size = ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    L.mxq_add_rmsnorm.restype = i32
    L.mxq_add_rmsnorm.argtypes = [vp, i64, vp, i64, vp, i64, i64, f32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.mxq_add_rmsnorm_backward_workspace_size.restype = size
    L.mxq_add_rmsnorm_backward_workspace_size.argtypes = [i64, i64]
    L.mxq_add_rmsnorm_backward.restype = i32
    L.mxq_add_rmsnorm_backward.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, vp, vp, size, vp]
    L.mxq_swiglu.restype = i32
    L.mxq_swiglu.argtypes = [vp, i64, vp, i64, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.mxq_swiglu_backward.restype = i32
    L.mxq_swiglu_backward.argtypes = [vp, i64, vp, vp, vp, vp, i64, i64, i32, vp, i64, vp, i64, vp, vp]
    L.mxq_linear_workspace_size.restype = size
    L.mxq_linear_workspace_size.argtypes = [ctypes.POINTER(_Linear)]
    L.mxq_linear.restype = i32
    L.mxq_linear.argtypes = [ctypes.POINTER(_Linear), vp]
    _lib, _calls = L, _native_calls(L)
    return L


def _rows(t: torch.Tensor, name: str, like: torch.Tensor | None = None) -> torch.Tensor:
    """A 2-D GPU tensor whose rows are contiguous (any row stride), of the type, shape and device of `like`."""
    if not t.is_cuda or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a 2-D tensor on the GPU with contiguous rows")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{name} must have dtype {like.dtype}")
        if t.shape != like.shape:
            raise ValueError(f"{name} must have shape {tuple(like.shape)}")
        if t.device != like.device:
            raise ValueError(f"{name} must be on {like.device}")
    return t


def _whole(t: torch.Tensor, name: str, shape, dtype, device) -> torch.Tensor:
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}")
    if not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != tuple(shape) or t.device != device:
        raise ValueError(f"{name} must be a contiguous tensor of shape {tuple(shape)} on {device}")
    return t


def _q8_like(rows: int, cols: int, device) -> Q8:
    return Q8(torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=device),
              torch.empty((rows, cols // Q8_BLOCK), dtype=torch.float8_e8m0fnu, device=device))


def _check_q8(q: Q8, name: str, shape, device) -> None:
    _whole(q[0], f"{name} codes", shape, torch.float8_e4m3fn, device)
    _whole(q[1], f"{name} scales", (shape[0], shape[1] // Q8_BLOCK), torch.float8_e8m0fnu, device)


def _workspace(nbytes: int, device, stream) -> torch.Tensor:
    """Scratch memory of one call, allocated on the stream that uses it: memory that was freed on the current stream may still be
    written there, and the caller, who does not see the workspace, could not make `stream` wait for that."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def add_rmsnorm(x: torch.Tensor, weight: torch.Tensor | None = None, residual: torch.Tensor | None = None, eps: float = 1e-6,
                dense: bool = False, checkpoint: bool = False, hidden_out: torch.Tensor | None = None, stream=None):
    """mxq_add_rmsnorm: t = x + residual, y = t / rms(t) * weight.  Returns (y, hidden, saved): y as Q8, or in x's type if
    `dense`; hidden = t in x's type (x itself without a residual; `hidden_out` may be the residual, which is then updated in
    place); saved = SavedNorm for add_rmsnorm_backward if `checkpoint`, else None."""
    if _calls is not None and stream is None:
        done = _calls.add_rmsnorm(x, weight, residual, eps, dense, checkpoint, hidden_out)
        if done is not None:
            return _done(done)
    _rows(x, "x")
    rows, cols = x.shape
    dt, dev = _dtype_code(x), x.device
    if residual is not None:
        _rows(residual, "residual", x)
    if weight is not None:
        _whole(weight, "weight", (cols,), x.dtype, dev)
    if residual is None and hidden_out is not None:
        raise ValueError("hidden_out without a residual")
    if hidden_out is not None:
        _whole(hidden_out, "hidden_out", (rows, cols), x.dtype, dev)
    elif residual is not None:
        hidden_out = torch.empty((rows, cols), dtype=x.dtype, device=dev)
    y = torch.empty((rows, cols), dtype=x.dtype, device=dev) if dense else _q8_like(rows, cols, dev)
    saved = SavedNorm(_q8_like(rows, cols, dev), torch.empty(rows, dtype=torch.float32, device=dev)) if checkpoint else None
    _check(_layers().mxq_add_rmsnorm(
        x.data_ptr(), x.stride(0), _ptr(residual), residual.stride(0) if residual is not None else 0, _ptr(weight), rows, cols,
        float(eps), dt, _ptr(hidden_out), None if dense else y[0].data_ptr(), None if dense else y[1].data_ptr(),
        y.data_ptr() if dense else None, saved[0][0].data_ptr() if checkpoint else None,
        saved[0][1].data_ptr() if checkpoint else None, saved[1].data_ptr() if checkpoint else None, _stream_ptr(stream)))
    return y, x if residual is None else hidden_out, saved


def add_rmsnorm_backward(dy: torch.Tensor, saved: SavedNorm, weight: torch.Tensor | None = None, dhidden: torch.Tensor | None = None,
                         dx_out: torch.Tensor | None = None, want_dweight: bool = True, stream=None):
    """mxq_add_rmsnorm_backward: (dx, dweight) from the 8-bit checkpoint.  dx, in dy's type, is the gradient of x and of the
    residual; `dhidden` is added to it (the gradient that reaches hidden by its other way).  dweight is fp32, None without a
    weight or if not wanted."""
    if _calls is not None and stream is None:
        done = _calls.add_rmsnorm_backward(dy, saved, weight, dhidden, dx_out, want_dweight)
        if done is not None:
            return _done(done)
    _rows(dy, "dy")
    rows, cols = dy.shape
    dt, dev = _dtype_code(dy), dy.device
    _check_q8(saved[0], "saved", (rows, cols), dev)
    _whole(saved[1], "saved rstd", (rows,), torch.float32, dev)
    if weight is not None:
        _whole(weight, "weight", (cols,), dy.dtype, dev)
    if dhidden is not None:
        _rows(dhidden, "dhidden", dy)
    if dx_out is not None:
        _whole(dx_out, "dx_out", (rows, cols), dy.dtype, dev)
    else:
        dx_out = torch.empty((rows, cols), dtype=dy.dtype, device=dev)
    L = _layers()
    dweight = workspace = None
    bytes_ = 0
    if weight is not None and want_dweight:
        dweight = torch.empty(cols, dtype=torch.float32, device=dev)
        bytes_ = L.mxq_add_rmsnorm_backward_workspace_size(rows, cols)
        workspace = _workspace(max(bytes_, 16), dev, stream)
    _check(L.mxq_add_rmsnorm_backward(
        dy.data_ptr(), dy.stride(0), saved[0][0].data_ptr(), saved[0][1].data_ptr(), saved[1].data_ptr(), _ptr(weight),
        _ptr(dhidden), dhidden.stride(0) if dhidden is not None else 0, rows, cols, dt, dx_out.data_ptr(), _ptr(dweight),
        _ptr(workspace), bytes_, _stream_ptr(stream)))
    return dx_out, dweight


def swiglu(gate: torch.Tensor, up: torch.Tensor, dense: bool = False, checkpoint: bool = False, stream=None):
    """mxq_swiglu: h = gate * sigmoid(gate) * up.  Returns (h, saved): h as Q8, or in gate's type if `dense`; saved =
    SavedSwiglu for swiglu_backward if `checkpoint`, else None.  gate and up may be halves of one projection's output."""
    if _calls is not None and stream is None:
        done = _calls.swiglu(gate, up, dense, checkpoint)
        if done is not None:
            return _done(done)
    _rows(gate, "gate")
    _rows(up, "up", gate)
    rows, cols = gate.shape
    dt, dev = _dtype_code(gate), gate.device
    h = torch.empty((rows, cols), dtype=gate.dtype, device=dev) if dense else _q8_like(rows, cols, dev)
    saved = SavedSwiglu(_q8_like(rows, cols, dev), _q8_like(rows, cols, dev)) if checkpoint else None
    _check(_layers().mxq_swiglu(
        gate.data_ptr(), gate.stride(0), up.data_ptr(), up.stride(0), rows, cols, dt, None if dense else h[0].data_ptr(),
        None if dense else h[1].data_ptr(), h.data_ptr() if dense else None, saved[0][0].data_ptr() if checkpoint else None,
        saved[0][1].data_ptr() if checkpoint else None, saved[1][0].data_ptr() if checkpoint else None,
        saved[1][1].data_ptr() if checkpoint else None, _stream_ptr(stream)))
    return h, saved


def swiglu_backward(dh: torch.Tensor, saved: SavedSwiglu, again: bool = False, stream=None):
    """mxq_swiglu_backward: (dgate, dup, h) in dh's type from the 8-bit checkpoint; h, the forward output computed again, if
    `again`, else None.  dgate and dup are the halves of one [rows, 2 * cols] tensor, as the gradient of a fused gate-and-up
    projection's output is."""
    if _calls is not None and stream is None:
        done = _calls.swiglu_backward(dh, saved, again)
        if done is not None:
            return _done(done)
    _rows(dh, "dh")
    rows, cols = dh.shape
    dt, dev = _dtype_code(dh), dh.device
    _check_q8(saved[0], "saved gate", (rows, cols), dev)
    _check_q8(saved[1], "saved up", (rows, cols), dev)
    both = torch.empty((rows, 2 * cols), dtype=dh.dtype, device=dev)
    dgate, dup = both[:, :cols], both[:, cols:]
    h = torch.empty((rows, cols), dtype=dh.dtype, device=dev) if again else None
    _check(_layers().mxq_swiglu_backward(
        dh.data_ptr(), dh.stride(0), saved[0][0].data_ptr(), saved[0][1].data_ptr(), saved[1][0].data_ptr(),
        saved[1][1].data_ptr(), rows, cols, dt, dgate.data_ptr(), 2 * cols, dup.data_ptr(), 2 * cols, _ptr(h),
        _stream_ptr(stream)))
    return dgate, dup, h


def linear(x, w: W4, adapters: Adapters | None = None, ids: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
           out: torch.Tensor | None = None, stream=None, sums: int = SUMS_F32) -> torch.Tensor:
    """mxq_linear: y = x W^T over packed FP4 weights, plus the low-rank adapter of each row.  x is Q8 or a bfloat16 tensor with
    contiguous rows; ids (int32, one a row) says which adapter a row has, values outside of 0 .. count-1 that it has none, and may
    be left out when there is one adapter for all.  y is bfloat16 or float32; `out` may have any row stride.  Sums are held in 32
    bits; SUMS_MX takes about 21 bits within each 128 of k for twice the rate, where x is Q8, y bfloat16 and the weights have E8M0
    scales of 32 elements or more."""
    if _calls is not None and stream is None and out is None:
        done = _calls.linear(x, w, adapters, ids, out_dtype, sums)
        if done is not None:
            return _done(done)
    codes, scales, block, scale_fmt, tensor_scale = w
    if isinstance(x, torch.Tensor):
        _rows(x, "x")
        if x.dtype != torch.bfloat16:
            raise TypeError("x must be bfloat16 or Q8")
        m, k = x.shape
        dev = x.device
    else:
        m, k = x[0].shape
        dev = x[0].device
        _check_q8(x, "x", (m, k), dev)
    n = codes.shape[0]
    _whole(codes, "w codes", (n, k // 2), torch.uint8, dev)
    if block <= 0:
        raise ValueError("block must be positive")
    _whole(scales, "w scales", (n, k // block), torch.uint8, dev)
    args = _Linear(m=m, n=n, k=k, w_codes=codes.data_ptr(), w_scales=scales.data_ptr(), block=block, scale_fmt=scale_fmt,
                   sums=sums)
    if isinstance(x, torch.Tensor):
        args.x, args.ld_x = x.data_ptr(), x.stride(0)
    else:
        args.x_codes, args.x_scales = x[0].data_ptr(), x[1].data_ptr()
    if isinstance(tensor_scale, torch.Tensor):
        _need(tensor_scale, 4, "tensor_scale", torch.float32)
        args.tensor_scale, args.tensor_scale_dev = 1.0, tensor_scale.data_ptr()
    else:
        args.tensor_scale = float(tensor_scale)
    if adapters is not None:
        a, b, scaling = adapters
        if a.dim() != 3:
            raise ValueError("adapters.a must have shape [count, rank, k]")
        count, rank = a.shape[0], a.shape[1]
        _whole(a, "adapters.a", (count, rank, k), torch.bfloat16, dev)
        _whole(b, "adapters.b", (count, n, rank), torch.bfloat16, dev)
        _whole(scaling, "adapters.scaling", (count,), torch.float32, dev)
        if ids is None and count != 1:
            raise ValueError("ids are needed with more than one adapter")
        if ids is not None:
            _whole(ids, "ids", (m,), torch.int32, dev)
            args.adapter_ids = ids.data_ptr()
        args.adapter_a, args.adapter_b, args.adapter_scaling = a.data_ptr(), b.data_ptr(), scaling.data_ptr()
        args.adapter_count, args.adapter_rank = count, rank
    elif ids is not None:
        raise ValueError("ids without adapters")
    if out is None:
        out = torch.empty((m, n), dtype=out_dtype, device=dev)
    else:
        _rows(out, "out")
        if tuple(out.shape) != (m, n) or out.device != dev:
            raise ValueError(f"out must have shape {(m, n)} on {dev}")
    args.y, args.ld_y, args.y_dtype = out.data_ptr(), out.stride(0), _dtype_code(out)
    L = _layers()
    need = L.mxq_linear_workspace_size(ctypes.byref(args))
    if need:
        workspace = _workspace(need, dev, stream)
        args.workspace, args.workspace_bytes = workspace.data_ptr(), need
    _check(L.mxq_linear(ctypes.byref(args), _stream_ptr(stream)))
    return out
