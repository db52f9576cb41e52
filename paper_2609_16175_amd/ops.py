"""Operators of a query tower on device tensors: layer norm, softmax cross
entropy over the points of an index, products with 4-bit rows.

Argument marshalling for libboa.so (include/boa.h); every computation runs in
the library's HIP kernels. Tensors live on one GPU; calls are queued on its
current stream, or on `stream`, and return without waiting. With `stream`,
results belong to it, and its order after whatever makes the inputs is the
caller's.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import _check, lib

T_F32, T_BF16, T_F16 = 0, 1, 2
_DTYPES = {torch.float32: T_F32, torch.bfloat16: T_BF16, torch.float16: T_F16}
_REDUCE = {"none": 0, "sum": 1, "mean": 2}


class Xent(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("d", C.c_int32), ("B", C.c_int64), ("V", C.c_int64),
                ("h", C.c_void_p), ("h_stride", C.c_int64), ("points", C.c_void_p), ("points_stride", C.c_int64),
                ("labels", C.c_void_p), ("bias", C.c_void_p), ("scale", C.c_float), ("reduction", C.c_int32),
                ("loss", C.c_void_p), ("lse", C.c_void_p), ("dloss", C.c_void_p), ("dh", C.c_void_p),
                ("dpoints", C.c_void_p), ("dbias", C.c_void_p)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        P, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        L.boa_layer_norm.argtypes = [P, i64, i32, i64, i32, P, P, i32, f32, P, P, P, P]
        L.boa_layer_norm_backward.argtypes = [P, i64, P, i64, i64, i32, i32, P, i32, P, P, P, P, P, P, i64, P]
        L.boa_layer_norm_backward_workspace.argtypes = [i64, i32]
        L.boa_layer_norm_backward_workspace.restype = i64
        L.boa_softmax_xent_workspace.argtypes = [C.POINTER(Xent), i32]
        L.boa_softmax_xent_workspace.restype = i64
        for f in (L.boa_softmax_xent, L.boa_softmax_xent_grad):
            f.argtypes = [C.POINTER(Xent), P, i64, P]
        L.boa_matvec_fourbit.argtypes = [P, i64, i64, i32, P, i64, i32, i64, P, P, i64, i32, i32, P, i64, P]
        _ready = L
    return _ready


# The current device and stream as plain numbers: a call on one row is a few
# microseconds of kernel, and torch's stream objects cost as much again.
_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _at(x, stream, *inputs):
    """None where the call can go on: x lies on the current GPU and `stream` is
    its current stream. Else the context in which to make the call again, with
    the inputs kept for the other stream: what the call allocates and copies
    then belongs to it too."""
    dev = x.get_device()
    if stream is not None and stream.cuda_stream != _current_stream(dev):
        for t in inputs:
            if t is not None:
                t.record_stream(stream)
        return torch.cuda.stream(stream)
    return torch.cuda.device(dev) if dev != _current_device() else None


def _workspace(x, nbytes):
    return torch.empty((max(16, int(nbytes)),), dtype=torch.uint8, device=x.device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _device(name, *tensors):
    dev = None
    for t in tensors:
        if t is None:
            continue
        at = t.get_device() if isinstance(t, torch.Tensor) and t.is_cuda else -1
        if at < 0:
            raise ValueError(f"{name}: arguments must be device tensors")
        if dev is not None and at != dev:
            raise ValueError(f"{name}: tensors on different devices")
        dev = at


def _dtype(name, t, of=tuple(_DTYPES)):
    if t.dtype not in of:
        raise TypeError(f"{name}: {t.dtype} is not supported here")
    return _DTYPES[t.dtype]


def _rows(x):
    """x as a matrix whose last dimension is contiguous, without a copy where
    its strides allow."""
    if x.is_contiguous() and x.dim() == 2:
        return x
    m = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
    if m.shape[1] > 1 and m.stride(1) != 1 or m.shape[0] > 1 and m.stride(0) < m.shape[1]:
        m = m.contiguous()
    return m


def _stride(m):
    return m.stride(0) if m.shape[0] > 1 else m.shape[1]


# ---------------------------------------------------------------------------
# layer norm

def _norm_params(name, x, weight, bias):
    last = x.shape[-1:]
    if not last or last[0] < 1:
        raise ValueError(f"{name}: x needs a last dimension of at least 1")
    dtype = None
    for p in (weight, bias):
        if p is None:
            continue
        if p.shape != last or p.dtype != x.dtype and p.dtype != torch.float32:
            raise ValueError(f"{name}: weight and bias must be ({last[0]},) of x's type or float32")
        if dtype is not None and p.dtype != dtype:
            raise ValueError(f"{name}: weight and bias must have one type")
        dtype = p.dtype
    return _DTYPES[x.dtype if dtype is None else dtype]


def _dense(t):
    return t if t is None or t.is_contiguous() else t.contiguous()


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, stream=None):
    """(y, mean, rstd) of layer norm over the last dimension of x.

    x: float32, bfloat16 or float16, any leading dimensions; weight, bias: (d,)
    of x's type or float32. y has x's type; mean and rstd (float32, one per
    row) are what layer_norm_backward takes."""
    _device("layer_norm", x, weight, bias)
    dt = _dtype("layer_norm", x)
    pd = _norm_params("layer_norm", x, weight, bias)
    w, b = _dense(weight), _dense(bias)
    other = _at(x, stream, x, weight, bias)
    if other is not None:
        with other:
            return layer_norm_forward(x, weight, bias, eps)
    m = _rows(x)
    rows, d = m.shape
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    mean, rstd = torch.empty((2, rows), dtype=torch.float32, device=x.device).unbind(0)
    _check(_lib().boa_layer_norm(m.data_ptr(), rows, d, _stride(m), dt, _ptr(w), _ptr(b), pd, eps, y.data_ptr(),
                                 mean.data_ptr(), rstd.data_ptr(), _current_stream(x.get_device())))
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, need=(True, True, True), stream=None, param_dtype=None):
    """(dx, dweight, dbias) of layer_norm_forward; weight may be None. dweight
    and dbias have weight's type; without one, param_dtype (x's, the default,
    or float32). need: which of the three to compute."""
    _device("layer_norm_backward", dy, x, weight, mean, rstd)
    dt = _dtype("layer_norm_backward", x)
    pd = _norm_params("layer_norm_backward", x, weight, None)
    ptype = weight.dtype if weight is not None else x.dtype if param_dtype is None else param_dtype
    if param_dtype not in (None, ptype) or ptype not in (x.dtype, torch.float32):
        raise ValueError("layer_norm_backward: param_dtype must be weight's type, or without one x's or float32")
    pd = _DTYPES[ptype]
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("layer_norm_backward: dy must have x's shape and type")
    m, g = _rows(x), _rows(dy)
    rows, d = m.shape
    for s in (mean, rstd):
        if s.dtype != torch.float32 or s.numel() != rows or not s.is_contiguous():
            raise ValueError("layer_norm_backward: mean and rstd must be the float32 tensors of the forward pass")
    other = _at(x, stream, dy, x, weight, mean, rstd)
    if other is not None:
        with other:
            return layer_norm_backward(dy, x, weight, mean, rstd, need, param_dtype=param_dtype)
    w = _dense(weight)
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need[0] else None
    dw = db = None
    if need[1] and need[2]:
        dw, db = torch.empty((2, d), dtype=ptype, device=x.device).unbind(0)
    elif need[1]:
        dw = torch.empty((d,), dtype=ptype, device=x.device)
    elif need[2]:
        db = torch.empty((d,), dtype=ptype, device=x.device)
    ws = _workspace(x, _lib().boa_layer_norm_backward_workspace(rows, d)) if need[1] or need[2] else None
    _check(_lib().boa_layer_norm_backward(g.data_ptr(), _stride(g), m.data_ptr(), _stride(m), rows, d, dt, _ptr(w), pd,
                                          mean.data_ptr(), rstd.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db), _ptr(ws),
                                          0 if ws is None else ws.numel(),
                                          _current_stream(x.get_device())))
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias_type = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        return *layer_norm_backward(dy, x, weight, mean, rstd, ctx.needs_input_grad[:3], param_dtype=ctx.bias_type), None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension of x, for autograd."""
    return _LayerNorm.apply(x, weight, bias, eps)


# ---------------------------------------------------------------------------
# softmax cross entropy over the points

@dataclass
class XentResult:
    loss: "object"             # float32: a number, or one per query (reduction "none")
    lse: "object"              # float32 (B,): log of the sum of exponentials
    dh: "object" = None        # like h
    drows: "object" = None     # like rows
    dbias: "object" = None     # float32 (V,)


def _xent(name, h, rows, labels, bias, scale, reduction, stream, grad, dloss=None, h_grad=False, rows_grad=False,
          bias_grad=False):
    _device(name, h, rows, labels, bias, dloss)
    if h.dtype == torch.float16:
        dt = T_F16   # refused by the library, with its reason
    else:
        dt = _dtype(name, h, (torch.float32, torch.bfloat16))
    if h.dim() != 2 or rows.dim() != 2 or h.shape[1] != rows.shape[1] or h.dtype != rows.dtype:
        raise ValueError(f"{name}: h must be (B, d) and rows (V, d), of one type")
    (B, d), V = h.shape, rows.shape[0]
    if labels.dtype != torch.int64 or tuple(labels.shape) != (B,):
        raise ValueError(f"{name}: labels must be int64 of shape ({B},)")
    if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (V,)):
        raise ValueError(f"{name}: bias must be float32 of shape ({V},)")
    if reduction not in _REDUCE:
        raise ValueError(f"{name}: reduction must be one of {', '.join(_REDUCE)}")
    shape = (B,) if reduction == "none" else ()
    if dloss is not None and (dloss.dtype != torch.float32 or tuple(dloss.shape) != shape):
        raise ValueError(f"{name}: dloss must be float32 of the loss's shape")
    other = _at(h, stream, h, rows, labels, bias, dloss)
    if other is not None:
        with other:
            return _xent(name, h, rows, labels, bias, scale, reduction, None, grad, dloss, h_grad, rows_grad, bias_grad)
    dev = h.device
    hm, rm, lab, bm, gm = _rows(h), _rows(rows), _dense(labels), _dense(bias), _dense(dloss)
    r = XentResult(torch.empty(shape, dtype=torch.float32, device=dev), torch.empty((B,), dtype=torch.float32, device=dev))
    if h_grad:
        r.dh = torch.empty((B, d), dtype=h.dtype, device=dev)
    if rows_grad:
        r.drows = torch.empty((V, d), dtype=rows.dtype, device=dev)
    if bias_grad:
        r.dbias = torch.empty((V,), dtype=torch.float32, device=dev)
    a = Xent(dt, d, B, V, hm.data_ptr(), _stride(hm), rm.data_ptr(), _stride(rm), lab.data_ptr(), _ptr(bm), scale,
             _REDUCE[reduction], r.loss.data_ptr(), r.lse.data_ptr(), _ptr(gm), _ptr(r.dh), _ptr(r.drows), _ptr(r.dbias))
    nbytes = _lib().boa_softmax_xent_workspace(C.byref(a), int(grad))
    if nbytes < 0:
        _check(nbytes)
    ws = _workspace(h, nbytes)
    fn = _lib().boa_softmax_xent_grad if grad else _lib().boa_softmax_xent
    _check(fn(C.byref(a), ws.data_ptr(), ws.numel(),
              _current_stream(h.get_device())))
    return r


def softmax_xent_grad(h, rows, labels, bias=None, scale=1.0, reduction="mean", dloss=None, h_grad=True, rows_grad=True,
                      bias_grad=False, stream=None):
    """Softmax cross entropy of queries h (B, d) over points rows (V, d) as
    classes, and its gradients, in one call: an XentResult.

    logits = scale * h @ rows.T + bias, never stored. labels: int64 (B,), the
    point of each query; a negative one leaves its query out. bias: float32
    (V,), -inf leaves a point out. dloss: the gradient of the loss (default 1).
    h_grad, rows_grad, bias_grad: which gradients to compute. In bfloat16 the
    probabilities, but for the labels' own, are rounded to bfloat16 as operands
    of the gradients' products; the results are rounded once."""
    if bias_grad and bias is None:
        raise ValueError("softmax_xent: a gradient of bias without a bias")
    return _xent("softmax_xent", h, rows, labels, bias, scale, reduction, stream, True, dloss, h_grad, rows_grad, bias_grad)


class _SoftmaxXent(torch.autograd.Function):
    # The gradients are formed in the forward pass, where the points pass by
    # anyway; backward scales them, which rounds bfloat16 gradients a second
    # time where dloss is no power of two. Unreduced losses have a gradient per
    # query, which the points' gradient cannot be scaled by afterwards:
    # there, backward does the whole work.
    @staticmethod
    def forward(ctx, h, rows, labels, bias, scale, reduction):
        need = ctx.needs_input_grad
        ctx.args = scale, reduction
        if reduction == "none":
            ctx.save_for_backward(h, rows, labels, bias)
            return _xent("softmax_xent", h, rows, labels, bias, scale, reduction, None, False).loss
        r = _xent("softmax_xent", h, rows, labels, bias, scale, reduction, None, True, None, need[0], need[1], need[3])
        ctx.save_for_backward(r.dh, r.drows, r.dbias)
        return r.loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        scale, reduction = ctx.args
        need = ctx.needs_input_grad
        if reduction == "none":
            h, rows, labels, bias = ctx.saved_tensors
            r = _xent("softmax_xent", h, rows, labels, bias, scale, reduction, None, True, dloss.float(), need[0], need[1],
                      need[3])
            return r.dh, r.drows, None, r.dbias, None, None
        dh, drows, dbias = ctx.saved_tensors
        by = lambda t: None if t is None else (t * dloss).to(t.dtype)  # noqa: E731
        return by(dh), by(drows), None, by(dbias), None, None


def softmax_xent(h, rows, labels, bias=None, scale=1.0, reduction="mean"):
    """The loss of softmax_xent_grad, for autograd; without gradients to
    compute, the losses alone. A reduced loss' gradients are formed with it and
    multiplied by the gradient that arrives, in h's and rows' type: bfloat16
    ones are rounded a second time then. softmax_xent_grad with dloss rounds
    once."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (h, rows, bias)):
        return _SoftmaxXent.apply(h, rows, labels, bias, scale, reduction)
    return _xent("softmax_xent", h, rows, labels, bias, scale, reduction, None, False).loss


# ---------------------------------------------------------------------------
# products with 4-bit rows

def matvec_4bit(x, codes, scales, offsets=None, group=None, stream=None):
    """y = x @ w.T for rows w of 4-bit codes: w = scales * code + offsets, or
    scales * (code - 8) without offsets.

    x: (M, K) or (K,), float32, bfloat16 or float16. codes: uint8 (N, K / 2),
    value 2j in the low nibble of byte j. scales, offsets: (N, groups) of one
    floating type. group: values of k per scale (default K / groups). For
    serving: autograd does not see it."""
    _device("matvec_4bit", x, codes, scales, offsets)
    dt = _dtype("matvec_4bit", x)
    sd = _dtype("matvec_4bit", scales)
    if x.dim() not in (1, 2):
        raise ValueError("matvec_4bit: x must be (M, K) or (K,)")
    m = _rows(x if x.dim() == 2 else x[None])
    M, K = m.shape
    if codes.dtype != torch.uint8 or codes.dim() != 2 or codes.shape[1] != (K + 1) // 2:
        raise ValueError(f"matvec_4bit: codes must be uint8 (N, {(K + 1) // 2})")
    N = codes.shape[0]
    if scales.dim() != 2 or scales.shape[0] != N or scales.shape[1] < 1:
        raise ValueError("matvec_4bit: scales must be (N, groups)")
    G = scales.shape[1]
    if group is None:
        if K % G:
            raise ValueError("matvec_4bit: K is no multiple of the number of groups: pass group")
        group = K // G
    if group < 1 or -(-K // group) != G:
        raise ValueError(f"matvec_4bit: {G} groups of {group} do not cover K = {K}")
    if offsets is not None and (offsets.shape != scales.shape or offsets.dtype != scales.dtype):
        raise ValueError("matvec_4bit: offsets must have the scales' shape and type")
    other = _at(x, stream, x, codes, scales, offsets)
    if other is not None:
        with other:
            return matvec_4bit(x, codes, scales, offsets, group)
    c, s = _rows(codes), _rows(scales)
    o = None if offsets is None else _rows(offsets)
    if o is not None and _stride(o) != _stride(s):
        s, o = s.contiguous(), o.contiguous()
    y = torch.empty((M, N), dtype=x.dtype, device=x.device)
    _check(_lib().boa_matvec_fourbit(m.data_ptr(), M, _stride(m), dt, c.data_ptr(), N, K, _stride(c), s.data_ptr(), _ptr(o),
                                     _stride(s), sd, group, y.data_ptr(), N, _current_stream(x.get_device())))
    return y if x.dim() == 2 else y[0]
