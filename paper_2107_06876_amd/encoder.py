"""ctypes binding of the operators of include/lcn.h that produce and train the points.  Same names as the C
entry points; argument marshalling only.

Tensors are contiguous device tensors of one type, float32 or bfloat16 (attention also takes views with strides);
work goes to torch's current stream on their device; `workspace`, where given, is a contiguous uint8 tensor."""
from __future__ import annotations

import ctypes

import torch

from .binding import BF16, F32, OK, LcnError, load_library

ACT_NONE, ACT_TANH, ACT_RELU, ACT_GELU, ACT_SILU = range(5)

_TYPES = {torch.float32: F32, torch.bfloat16: BF16}
_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        vp, i64, i32, sz, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
        out = ctypes.POINTER(sz)
        lib.lcn_linear_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, out]
        lib.lcn_linear.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.lcn_linear_backward.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        lib.lcn_cross_entropy_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, out]
        lib.lcn_cross_entropy.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, f32, vp, vp, vp, sz, vp]
        lib.lcn_cross_entropy_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, f32, vp, vp, vp, vp, sz, vp]
        for name in ("lcn_linear_workspace_bytes", "lcn_linear", "lcn_linear_backward", "lcn_cross_entropy_workspace_bytes",
                     "lcn_cross_entropy", "lcn_cross_entropy_backward"):
            getattr(lib, name).restype = i32
        _lib = lib
    return _lib


def _tensor(t, name, shape, dtype, device):
    """The address of a contiguous device tensor of this shape and type; None stays None."""
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or tuple(t.shape) != shape or t.device != device:
        raise ValueError("%s: expected a contiguous %s tensor of shape %s on %s, got %s %s on %s"
                         % (name, dtype, shape, device, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _matrix(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2 or t.dtype not in _TYPES or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous float32 or bfloat16 device matrix" % name)
    return t


def _space(call, sizes, workspace, device):
    need = ctypes.c_size_t(0)
    st = call(*sizes, ctypes.byref(need))
    if st != OK:
        raise LcnError(st, call.__name__)
    if workspace is None:
        workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
    elif not workspace.is_contiguous() or workspace.dtype != torch.uint8 or workspace.device != device:
        raise ValueError("workspace: expected a contiguous uint8 tensor on %s" % device)
    return workspace


def _linear_shapes(x, w):
    x, w = _matrix(x, "x"), _matrix(w, "w")
    if x.dtype != w.dtype or x.device != w.device or x.shape[1] != w.shape[1]:
        raise ValueError("x (rows, d_in) and w (d_out, d_in) must agree in type, device and d_in")
    return x.shape[0], x.shape[1], w.shape[0], _TYPES[x.dtype]


def lcn_linear(x, w, bias=None, residual=None, activation=ACT_NONE, keep_pre=False, out=None, workspace=None):
    """act(x W^T + bias) + residual as a (rows, d_out) tensor; with keep_pre also z = x W^T + bias in float32, which
    lcn_linear_backward takes."""
    lib = _library()
    rows, d_in, d_out, dtype = _linear_shapes(x, w)
    dev = x.device
    y = torch.empty((rows, d_out), dtype=x.dtype, device=dev) if out is None else out
    pre = torch.empty((rows, d_out), dtype=torch.float32, device=dev) if keep_pre else None
    ws = _space(lib.lcn_linear_workspace_bytes, (rows, d_in, d_out, dtype, 0), workspace, dev)
    with torch.cuda.device(dev):
        st = lib.lcn_linear(x.data_ptr(), w.data_ptr(), _tensor(bias, "bias", (d_out,), x.dtype, dev),
                            _tensor(residual, "residual", (rows, d_out), x.dtype, dev), rows, d_in, d_out, dtype,
                            int(activation), _tensor(y, "out", (rows, d_out), x.dtype, dev),
                            None if pre is None else pre.data_ptr(), ws.data_ptr(), ws.numel(),
                            torch.cuda.current_stream(dev).cuda_stream)
    if st != OK:
        raise LcnError(st, "lcn_linear")
    return (y, pre) if keep_pre else y


def lcn_linear_backward(x, w, pre, dy, activation=ACT_NONE, with_bias=True, with_x=True, with_w=True, workspace=None):
    """(dx, dw, dbias) for a given dy; pre: what lcn_linear kept (may be None without an activation).  Gradients that
    are not asked for are None."""
    lib = _library()
    rows, d_in, d_out, dtype = _linear_shapes(x, w)
    dev = x.device
    dx = torch.empty_like(x) if with_x else None
    dw = torch.empty_like(w) if with_w else None
    db = torch.empty(d_out, dtype=x.dtype, device=dev) if with_bias else None
    ws = _space(lib.lcn_linear_workspace_bytes, (rows, d_in, d_out, dtype, 1), workspace, dev)
    with torch.cuda.device(dev):
        st = lib.lcn_linear_backward(x.data_ptr(), w.data_ptr(), _tensor(pre, "pre", (rows, d_out), torch.float32, dev),
                                     _tensor(dy, "dy", (rows, d_out), x.dtype, dev), rows, d_in, d_out, dtype,
                                     int(activation), *[None if t is None else t.data_ptr() for t in (dx, dw, db)],
                                     ws.data_ptr(), ws.numel(), torch.cuda.current_stream(dev).cuda_stream)
    if st != OK:
        raise LcnError(st, "lcn_linear_backward")
    return dx, dw, db


def _entropy_shapes(x, w):
    x, w = _matrix(x, "x"), _matrix(w, "w")
    if x.dtype != w.dtype or x.device != w.device or x.shape[1] != w.shape[1]:
        raise ValueError("x (rows, dim) and w (vocab, dim) must agree in type, device and dim")
    return x.shape[0], w.shape[0], x.shape[1], _TYPES[x.dtype]


def lcn_cross_entropy(x, w, target, bias=None, scale=1.0, workspace=None):
    """(loss, lse), float32 per row, of the scores scale x W^T + bias; target: int64, negative where a row has none."""
    lib = _library()
    rows, vocab, dim, dtype = _entropy_shapes(x, w)
    dev = x.device
    loss = torch.empty(rows, dtype=torch.float32, device=dev)
    lse = torch.empty(rows, dtype=torch.float32, device=dev)
    ws = _space(lib.lcn_cross_entropy_workspace_bytes, (rows, vocab, dim, dtype, 0), workspace, dev)
    with torch.cuda.device(dev):
        st = lib.lcn_cross_entropy(x.data_ptr(), w.data_ptr(), _tensor(bias, "bias", (vocab,), torch.float32, dev),
                                   _tensor(target, "target", (rows,), torch.int64, dev), rows, vocab, dim, dtype,
                                   float(scale), loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                   torch.cuda.current_stream(dev).cuda_stream)
    if st != OK:
        raise LcnError(st, "lcn_cross_entropy")
    return loss, lse


def lcn_cross_entropy_backward(x, w, target, lse, grad_loss, bias=None, scale=1.0, with_x=True, with_w=True,
                               workspace=None):
    """(dx, dw, dbias) of sum(grad_loss * loss); lse as lcn_cross_entropy returned it.  dbias is None without a
    bias, dx and dw where they are not asked for."""
    lib = _library()
    rows, vocab, dim, dtype = _entropy_shapes(x, w)
    dev = x.device
    dx = torch.empty_like(x) if with_x else None
    dw = torch.empty_like(w) if with_w else None
    db = torch.empty(vocab, dtype=torch.float32, device=dev) if bias is not None else None
    ws = _space(lib.lcn_cross_entropy_workspace_bytes, (rows, vocab, dim, dtype, 1), workspace, dev)
    with torch.cuda.device(dev):
        st = lib.lcn_cross_entropy_backward(
            x.data_ptr(), w.data_ptr(), _tensor(bias, "bias", (vocab,), torch.float32, dev),
            _tensor(target, "target", (rows,), torch.int64, dev), _tensor(lse, "lse", (rows,), torch.float32, dev),
            _tensor(grad_loss, "grad_loss", (rows,), torch.float32, dev), rows, vocab, dim, dtype, float(scale),
            *[None if t is None else t.data_ptr() for t in (dx, dw, db)], ws.data_ptr(), ws.numel(),
            torch.cuda.current_stream(dev).cuda_stream)
    if st != OK:
        raise LcnError(st, "lcn_cross_entropy_backward")
    return dx, dw, db
