"""ctypes binding of the operators of include/lcn.h that produce and train the points.  Same names as the C
entry points; argument marshalling only.

Tensors are contiguous device tensors of one type, float32 or bfloat16 (attention also takes views with strides);
work goes to torch's current stream on their device; `workspace`, where given, is a contiguous uint8 tensor.  Results are
no part of automatic differentiation, also where an input requires a gradient: that is what the backward calls give."""
from __future__ import annotations

import ctypes

import torch

from .binding import BF16, F32, OK, LcnError, load_library

ACT_NONE, ACT_TANH, ACT_RELU, ACT_GELU, ACT_SILU = range(5)

_TYPES = {torch.float32: F32, torch.bfloat16: BF16}
_lib = None


class AttentionDesc(ctypes.Structure):
    _fields_ = [("num_sets", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float), ("cap", ctypes.c_float), ("total_q", ctypes.c_int64),
                ("total_k", ctypes.c_int64), ("max_q", ctypes.c_int64), ("q_off", ctypes.c_void_p),
                ("k_off", ctypes.c_void_p), ("prefix", ctypes.c_void_p), ("slopes", ctypes.c_void_p),
                ("q_token", ctypes.c_int64), ("q_head", ctypes.c_int64), ("k_token", ctypes.c_int64),
                ("k_head", ctypes.c_int64), ("v_token", ctypes.c_int64), ("v_head", ctypes.c_int64),
                ("clear", ctypes.c_int32)]


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
        desc = ctypes.POINTER(AttentionDesc)
        lib.lcn_attention_workspace_bytes.argtypes = [desc, i32, out]
        lib.lcn_attention.argtypes = [desc, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.lcn_attention_backward.argtypes = [desc, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        for name in ("lcn_attention_workspace_bytes", "lcn_attention", "lcn_attention_backward", "lcn_linear_workspace_bytes",
                     "lcn_linear", "lcn_linear_backward", "lcn_cross_entropy_workspace_bytes", "lcn_cross_entropy",
                     "lcn_cross_entropy_backward"):
            getattr(lib, name).restype = i32
        _lib = lib
    return _lib


def _tensor(t, name, shape, dtype, device):
    """The address of a contiguous device tensor of this shape and type; None stays None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous %s tensor of shape %s on %s, got %s %s on %s"
                         % (name, dtype, shape, device, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


_sizes = {}   # bytes of workspace by call and sizes


def _space(call, sizes, workspace, device):
    """The address and size of a workspace, and the tensor that holds it."""
    need = _sizes.get((call, sizes))
    if need is None:
        out = ctypes.c_size_t(0)
        st = getattr(_library(), call)(*sizes, ctypes.byref(out))
        if st != OK:
            raise LcnError(st, call)
        if len(_sizes) > 4096:
            _sizes.clear()
        need = _sizes[(call, sizes)] = out.value
    return _workspace(need, workspace, device)


def _workspace(need, workspace, device):
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace.data_ptr(), need, workspace
    if not workspace.is_contiguous() or workspace.dtype != torch.uint8 or workspace.device != device:
        raise ValueError("workspace: expected a contiguous uint8 tensor on %s" % device)
    return workspace.data_ptr(), workspace.numel(), workspace


def _raw_stream(index):
    return torch.cuda.current_stream(index).cuda_stream


# the same without the object around it, where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _call(name, device, *args):
    """Calls an entry point with torch's current stream of `device` as its last argument, on that device."""
    stream = _raw_stream(device.index)
    f = getattr(_library(), name)
    if device.index == torch.cuda.current_device():
        st = f(*args, stream)
    else:
        with torch.cuda.device(device):
            st = f(*args, stream)
    if st != OK:
        raise LcnError(st, name)


def _address(t):
    return None if t is None else t.data_ptr()


def _matrices(x, w, inner):
    """Rows of x and w, their common width and type: contiguous device matrices."""
    dtype = _TYPES.get(x.dtype)
    if (dtype is None or w.dtype is not x.dtype or x.dim() != 2 or w.dim() != 2 or not x.is_cuda or w.device != x.device
            or not x.is_contiguous() or not w.is_contiguous()):
        raise ValueError("x and w: expected contiguous float32 or bfloat16 matrices of one type on one device")
    rows, width = x.shape
    if w.shape[1] != width:
        raise ValueError("x and w must agree in %s" % inner)
    return rows, w.shape[0], width, dtype


def lcn_linear(x, w, bias=None, residual=None, activation=ACT_NONE, keep_pre=False, out=None, workspace=None):
    """act(x W^T + bias) + residual as a (rows, d_out) tensor; with keep_pre also z = x W^T + bias in float32, which
    lcn_linear_backward takes."""
    rows, d_out, d_in, dtype = _matrices(x, w, "d_in")
    dev = x.device
    y = torch.empty((rows, d_out), dtype=x.dtype, device=dev) if out is None else out
    pre = torch.empty((rows, d_out), dtype=torch.float32, device=dev) if keep_pre else None
    at, size, space = _space("lcn_linear_workspace_bytes", (rows, d_in, d_out, dtype, 0), workspace, dev)
    _call("lcn_linear", dev, x.data_ptr(), w.data_ptr(), _tensor(bias, "bias", (d_out,), x.dtype, dev),
          _tensor(residual, "residual", (rows, d_out), x.dtype, dev), rows, d_in, d_out, dtype, int(activation),
          _tensor(y, "out", (rows, d_out), x.dtype, dev), _address(pre), at, size)
    return (y, pre) if keep_pre else y


def lcn_linear_backward(x, w, pre, dy, activation=ACT_NONE, with_bias=True, with_x=True, with_w=True, workspace=None):
    """(dx, dw, dbias) for a given dy; pre: what lcn_linear kept (may be None without an activation).  Gradients that
    are not asked for are None."""
    rows, d_out, d_in, dtype = _matrices(x, w, "d_in")
    dev = x.device
    dx = torch.empty_like(x) if with_x else None
    dw = torch.empty_like(w) if with_w else None
    db = torch.empty(d_out, dtype=x.dtype, device=dev) if with_bias else None
    at, size, space = _space("lcn_linear_workspace_bytes", (rows, d_in, d_out, dtype, 1), workspace, dev)
    _call("lcn_linear_backward", dev, x.data_ptr(), w.data_ptr(), _tensor(pre, "pre", (rows, d_out), torch.float32, dev),
          _tensor(dy, "dy", (rows, d_out), x.dtype, dev), rows, d_in, d_out, dtype, int(activation), _address(dx),
          _address(dw), _address(db), at, size)
    return dx, dw, db


def lcn_cross_entropy(x, w, target, bias=None, scale=1.0, workspace=None):
    """(loss, lse), float32 per row, of the scores scale x W^T + bias; target: int64, negative where a row has none."""
    rows, vocab, dim, dtype = _matrices(x, w, "dim")
    dev = x.device
    loss, lse = torch.empty((2, rows), dtype=torch.float32, device=dev)
    at, size, space = _space("lcn_cross_entropy_workspace_bytes", (rows, vocab, dim, dtype, 0), workspace, dev)
    _call("lcn_cross_entropy", dev, x.data_ptr(), w.data_ptr(), _tensor(bias, "bias", (vocab,), torch.float32, dev),
          _tensor(target, "target", (rows,), torch.int64, dev), rows, vocab, dim, dtype, float(scale), loss.data_ptr(),
          lse.data_ptr(), at, size)
    return loss, lse


def lcn_cross_entropy_backward(x, w, target, lse, grad_loss, bias=None, scale=1.0, with_x=True, with_w=True,
                               workspace=None):
    """(dx, dw, dbias) of sum(grad_loss * loss); lse as lcn_cross_entropy returned it.  dbias is None without a
    bias, dx and dw where they are not asked for."""
    rows, vocab, dim, dtype = _matrices(x, w, "dim")
    dev = x.device
    dx = torch.empty_like(x) if with_x else None
    dw = torch.empty_like(w) if with_w else None
    db = torch.empty(vocab, dtype=torch.float32, device=dev) if bias is not None else None
    at, size, space = _space("lcn_cross_entropy_workspace_bytes", (rows, vocab, dim, dtype, 1), workspace, dev)
    _call("lcn_cross_entropy_backward", dev, x.data_ptr(), w.data_ptr(), _tensor(bias, "bias", (vocab,), torch.float32, dev),
          _tensor(target, "target", (rows,), torch.int64, dev), _tensor(lse, "lse", (rows,), torch.float32, dev),
          _tensor(grad_loss, "grad_loss", (rows,), torch.float32, dev), rows, vocab, dim, dtype, float(scale), _address(dx),
          _address(dw), _address(db), at, size)
    return dx, dw, db


def _heads(t, name, like=None):
    """Checks a (tokens, heads, dim) device tensor whose last dimension is contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 3 or t.dtype not in _TYPES:
        raise ValueError("%s: expected a float32 or bfloat16 device tensor (tokens, heads, dim)" % name)
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError("%s: the values of a head must be contiguous" % name)
    if like is not None and (t.dtype != like.dtype or t.device != like.device or t.shape[2] != like.shape[2]):
        raise ValueError("%s: q, k and v must agree in type, device and dim" % name)
    return t


def _attention_desc(q, k, v, q_off, k_off, scale, causal, prefix, slopes, cap, max_q):
    _heads(q, "q"), _heads(k, "k", q), _heads(v, "v", q)
    if k.shape != v.shape or k.shape[1] == 0 or q.shape[1] % k.shape[1]:
        raise ValueError("k and v must have one shape, and q a multiple of their heads")
    dev = q.device
    if q_off.dim() != 1 or q_off.shape[0] < 1:
        raise ValueError("q_off: expected num_sets + 1 offsets")
    sets = q_off.shape[0] - 1

    def strides(t):   # of a dimension with one entry: any
        dense = t.shape[1] * t.shape[2]
        token, head = t.stride(0), t.stride(1)
        if (t.shape[0] > 1 and token < 1) or (t.shape[1] > 1 and head < 1):
            raise ValueError("tensors that are broadcast over tokens or heads are not taken: make them whole")
        return token if t.shape[0] > 1 else dense, head if t.shape[1] > 1 else t.shape[2]

    return AttentionDesc(sets, q.shape[1], k.shape[1], q.shape[2], _TYPES[q.dtype], 1 if causal else 0,
                         float(q.shape[2] ** -0.5 if scale is None else scale), float(cap), q.shape[0], k.shape[0], int(max_q),
                         _tensor(q_off, "q_off", (sets + 1,), torch.int64, dev),
                         _tensor(k_off, "k_off", (sets + 1,), torch.int64, dev),
                         _tensor(prefix, "prefix", (sets,), torch.int32, dev),
                         _tensor(slopes, "slopes", (q.shape[1],), torch.float32, dev), *strides(q), *strides(k), *strides(v), 1)


def _attention_space(desc, backward, workspace, device):
    out = ctypes.c_size_t(0)
    st = _library().lcn_attention_workspace_bytes(ctypes.byref(desc), backward, ctypes.byref(out))
    if st != OK:
        raise LcnError(st, "lcn_attention_workspace_bytes")
    return _workspace(out.value, workspace, device)


def lcn_attention(q, k, v, q_off, k_off, scale=None, causal=False, prefix=None, slopes=None, cap=0.0, max_q=0,
                  workspace=None):
    """(o, lse): attention of the queries of every set to the keys of the same set.  q: (tokens, heads, dim), k and v:
    (tokens, key heads, dim), views with strides are taken; q_off, k_off: int64 offsets of the sets on the device; scale:
    1 / sqrt(dim) where None; prefix: int32 per set (read if causal); slopes: float32 per head; max_q: the largest number of
    queries of a set, where known.  o is dense like q, lse float32 (heads, tokens); queries in no set have 0 and -inf,
    those that a max_q below the truth leaves out NaN."""
    d = _attention_desc(q, k, v, q_off, k_off, scale, causal, prefix, slopes, cap, max_q)
    dev = q.device
    o = torch.empty(q.shape, dtype=q.dtype, device=dev)
    lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=dev)
    at, size, space = _attention_space(d, 0, workspace, dev)
    _call("lcn_attention", dev, ctypes.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), at, size)
    return o, lse


def lcn_attention_backward(q, k, v, o, lse, dy, q_off, k_off, scale=None, causal=False, prefix=None, slopes=None, cap=0.0,
                           max_q=0, with_q=True, with_kv=True, workspace=None):
    """(dq, dk, dv) for a given dy, the gradient of o; o and lse as lcn_attention returned them, the rest as it was
    given.  Gradients are dense, zero for tokens in no set; those that are not asked for are None."""
    d = _attention_desc(q, k, v, q_off, k_off, scale, causal, prefix, slopes, cap, max_q)
    dev = q.device
    shape = tuple(q.shape)
    dq = torch.empty(shape, dtype=q.dtype, device=dev) if with_q else None
    dk = torch.empty(k.shape, dtype=q.dtype, device=dev) if with_kv else None
    dv = torch.empty(k.shape, dtype=q.dtype, device=dev) if with_kv else None
    at, size, space = _attention_space(d, 1, workspace, dev)
    _call("lcn_attention_backward", dev, ctypes.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr(),
          _tensor(o, "o", shape, q.dtype, dev), _tensor(lse, "lse", (shape[1], shape[0]), torch.float32, dev),
          _tensor(dy, "dy", shape, q.dtype, dev), _address(dq), _address(dk), _address(dv), at, size)
    return dq, dk, dv
