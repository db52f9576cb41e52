"""Operators of a query tower on device tensors: layer norm, linear layers, the
norms around a residual block, softmax cross entropy over the points of an
index, products with 4-bit rows, orthogonalised updates of weights.

Argument marshalling for libboa.so (include/boa.h); every computation runs in
the library's HIP kernels. Tensors live on one GPU; calls are queued on its
current stream, or on `stream`, and return without waiting. With `stream`,
results belong to it, and its order after whatever makes the inputs is the
caller's.
"""
from __future__ import annotations

import ctypes as C
import struct
from array import array
from dataclasses import dataclass

import torch
from torch.autograd import forward_ad
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


class Dense(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("activation", C.c_int32), ("M", C.c_int64), ("N", C.c_int32), ("K", C.c_int32),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("w", C.c_void_p), ("w_stride", C.c_int64),
                ("bias", C.c_void_p), ("param_dtype", C.c_int32), ("residual", C.c_void_p), ("residual_stride", C.c_int64),
                ("y", C.c_void_p), ("pre", C.c_void_p), ("dy", C.c_void_p), ("dy_stride", C.c_int64), ("dx", C.c_void_p),
                ("dw", C.c_void_p), ("dbias", C.c_void_p)]


class Block(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("param_dtype", C.c_int32), ("rows", C.c_int64), ("d", C.c_int32), ("norm", C.c_int32),
                ("post", C.c_int32), ("pre", C.c_int32), ("gate_rows", C.c_int32), ("scale", C.c_float), ("eps", C.c_float),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("f", C.c_void_p), ("f_stride", C.c_int64), ("gate", C.c_void_p),
                ("gate_stride", C.c_int64), ("post_weight", C.c_void_p), ("post_bias", C.c_void_p), ("weight", C.c_void_p),
                ("bias", C.c_void_p), ("h", C.c_void_p), ("y", C.c_void_p), ("stats", C.c_void_p), ("dh", C.c_void_p),
                ("dh_stride", C.c_int64), ("dy", C.c_void_p), ("dy_stride", C.c_int64), ("dx", C.c_void_p), ("df", C.c_void_p),
                ("dgate", C.c_void_p), ("dpost_weight", C.c_void_p), ("dpost_bias", C.c_void_p), ("dweight", C.c_void_p),
                ("dbias", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class Orth(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("rows", C.c_int32), ("cols", C.c_int32), ("count", C.c_int64), ("update", C.c_void_p),
                ("update_stride", C.c_int64), ("update_batch", C.c_int64), ("steps", C.c_int32), ("coefficients", C.c_void_p),
                ("eps", C.c_float), ("out", C.c_void_p)]


def _packer(cls):
    """pack() of a struct's values as bytes, in the order of its fields: a third of the time that filling the struct takes."""
    code = {C.c_int32: "i", C.c_int64: "q", C.c_float: "f", C.c_void_p: "P"}
    return struct.Struct("@" + "".join(code[kind] for _, kind in cls._fields_)).pack


_pack_dense, _pack_block, _pack_orth = _packer(Dense), _packer(Block), _packer(Orth)
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
        # packed structs: bytes go as void pointers
        L.boa_linear_workspace.argtypes = [P, i32]
        L.boa_linear_workspace.restype = i64
        for f in (L.boa_linear, L.boa_linear_grad):
            f.argtypes = [P, P, i64, P]
        for f in (L.boa_block_norm, L.boa_block_norm_backward):
            f.argtypes = [P, P]
        L.boa_block_norm_backward_workspace.argtypes = [i64, i32]
        L.boa_block_norm_backward_workspace.restype = i64
        L.boa_orthogonalize_workspace.argtypes = [P]
        L.boa_orthogonalize_workspace.restype = i64
        L.boa_orthogonalize.argtypes = [P, P, i64, P]
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


def _address(t):   # for packed structs
    return 0 if t is None else t.data_ptr()


def _device(name, *tensors):
    dev = None
    for t in tensors:
        if t is None:
            continue
        at = t.get_device() if isinstance(t, torch.Tensor) else -1   # -1 for host tensors too
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
    once. Forward-mode tangents raise."""
    # past its function, which refuses them, a call would drop the tangents that there can be at a forward-mode level
    if forward_ad._current_level >= 0 or torch.is_grad_enabled() and any(
            t is not None and t.requires_grad for t in (h, rows, bias)):
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


# ---------------------------------------------------------------------------
# linear layers

_ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
LINEAR_FEW = 16   # rows up to which a forward pass takes no work memory


def _activation(name, activation):
    if activation not in _ACTIVATIONS:
        raise ValueError(f"{name}: activation must be one of {', '.join(_ACTIVATIONS)}")
    return _ACTIVATIONS[activation]


def _linear_shapes(name, x, weight, bias):
    if weight.dim() != 2 or weight.dtype != x.dtype or x.dim() < 1 or x.shape[-1] != weight.shape[1]:
        raise ValueError(f"{name}: x must be (..., K) and weight (N, K), of one type")
    if weight.shape[0] < 1 or weight.shape[1] < 1:
        raise ValueError(f"{name}: weight needs at least one row and one column")
    if bias is not None and (bias.shape != weight.shape[:1] or bias.dtype not in (x.dtype, torch.float32)):
        raise ValueError(f"{name}: bias must be ({weight.shape[0]},) of x's type or float32")


def linear_forward(x, weight, bias=None, residual=None, activation="none", keep=False, stream=None):
    """(y, pre) of a linear layer: y = activation(x @ weight.T + bias) + residual.

    x: (..., K), float32, bfloat16 or float16; weight: (N, K) of x's type; bias:
    (N,) of x's type or float32; residual: like y, (..., N). activation: "none",
    "relu", "silu", "gelu" (the error function's) or "gelu_tanh". pre is what
    linear_backward takes where there is an activation: x @ weight.T + bias in
    float16, infinite beyond its range and for relu never 0 where it is above 0
    (float32 for float32 layers); None without `keep` or without an activation."""
    _device("linear", x, weight, bias, residual)
    dt = _dtype("linear", x)
    act = _activation("linear", activation)
    _linear_shapes("linear", x, weight, bias)
    N, K = weight.shape
    shape = (*x.shape[:-1], N)
    if residual is not None and (residual.shape != shape or residual.dtype != x.dtype):
        raise ValueError(f"linear: residual must be {shape} of x's type")
    other = _at(x, stream, x, weight, bias, residual)
    if other is not None:
        with other:
            return linear_forward(x, weight, bias, residual, activation, keep)
    m, w, b = _rows(x), _rows(weight), _dense(bias)
    r = None if residual is None else _rows(residual)
    M = m.shape[0]
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    pre = torch.empty(shape, dtype=torch.float32 if dt == T_F32 else torch.float16, device=x.device) if keep and act else None
    a = _pack_dense(dt, act, M, N, K, m.data_ptr(), _stride(m), w.data_ptr(), _stride(w), _address(b),
                    dt if b is None else _DTYPES[b.dtype], _address(r), 0 if r is None else _stride(r), y.data_ptr(), _address(pre),
                    0, 0, 0, 0, 0)
    ws, n = _linear_workspace(x, a, 0) if M > LINEAR_FEW else (None, 0)
    rc = _lib().boa_linear(a, _ptr(ws), n, _current_stream(x.get_device()))
    if rc:
        _check(rc)
    return y, pre


def _linear_workspace(x, a, grad):
    n = _lib().boa_linear_workspace(a, grad)
    if n < 0:
        _check(n)
    return (_workspace(x, n), n) if n else (None, 0)


def linear_backward(dy, x, weight, pre=None, activation="none", need=(True, True, True), bias_dtype=None, stream=None):
    """(dx, dweight, dbias) of linear_forward; the residual's gradient is dy.
    pre: the forward pass's, where there is an activation. need: which of the
    three to compute. dbias has bias_dtype: x's type (the default) or float32.
    In bfloat16 and float16 the gradient before the activation is rounded to
    x's type as an operand of the products, not in dbias; results are rounded
    once."""
    _device("linear_backward", dy, x, weight, pre)
    dt = _dtype("linear_backward", x)
    act = _activation("linear_backward", activation)
    _linear_shapes("linear_backward", x, weight, None)
    N, K = weight.shape
    if tuple(dy.shape) != (*x.shape[:-1], N) or dy.dtype != x.dtype:
        raise ValueError("linear_backward: dy must be (..., N) of x's type")
    if act:
        want = torch.float32 if dt == T_F32 else torch.float16
        if pre is None or pre.shape != dy.shape or pre.dtype != want or not pre.is_contiguous():
            raise ValueError("linear_backward: pre must be the tensor that linear_forward gave with keep")
    ptype = x.dtype if bias_dtype is None else bias_dtype
    if ptype not in (x.dtype, torch.float32):
        raise ValueError("linear_backward: bias_dtype must be x's or float32")
    other = _at(x, stream, dy, x, weight, pre)
    if other is not None:
        with other:
            return linear_backward(dy, x, weight, pre, activation, need, bias_dtype)
    m, w, g = _rows(x), _rows(weight), _rows(dy)
    dev = x.device
    dx = torch.empty(x.shape, dtype=x.dtype, device=dev) if need[0] else None
    dw = torch.empty((N, K), dtype=x.dtype, device=dev) if need[1] else None
    db = torch.empty((N,), dtype=ptype, device=dev) if need[2] else None
    a = _pack_dense(dt, act, m.shape[0], N, K, m.data_ptr(), _stride(m), w.data_ptr(), _stride(w), 0, _DTYPES[ptype], 0, 0, 0,
                    _address(pre) if act else 0, g.data_ptr(), _stride(g), _address(dx), _address(dw), _address(db))
    ws, n = _linear_workspace(x, a, 1)
    _check(_lib().boa_linear_grad(a, _ptr(ws), n, _current_stream(dev.index)))
    return dx, dw, db


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, activation):
        need = ctx.needs_input_grad
        y, pre = linear_forward(x, weight, bias, residual, activation, keep=need[0] or need[1] or need[2])
        ctx.save_for_backward(x, weight, pre)
        ctx.activation, ctx.bias_dtype = activation, None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw = db = None
        if any(need[:3]):
            dx, dw, db = linear_backward(dy, x, weight, pre, ctx.activation, need[:3], ctx.bias_dtype)
        return dx, dw, db, dy if need[3] else None, None


def linear(x, weight, bias=None, residual=None, activation="none"):
    """linear_forward's y, for autograd. Forward-mode tangents raise."""
    # past its function, which refuses them, a call would drop the tangents that there can be at a forward-mode level
    if forward_ad._current_level >= 0 or torch.is_grad_enabled() and (
            x.requires_grad or weight.requires_grad or bias is not None and bias.requires_grad
            or residual is not None and residual.requires_grad):
        return _Linear.apply(x, weight, bias, residual, activation)
    return linear_forward(x, weight, bias, residual, activation)[0]


# ---------------------------------------------------------------------------
# the norms around a residual block

_NORMS = {"layer": 0, "rms": 1}
_NO_GRADIENTS = (0,) * 13   # the rest of a Block in the forward pass


@dataclass
class BlockNormGrads:
    dx: "object"
    df: "object"
    dgate: "object" = None          # like gate
    dpost_weight: "object" = None   # like the parameters, where there are some
    dpost_bias: "object" = None
    dweight: "object" = None
    dbias: "object" = None


def _block(name, x, f, gate, post, pre, post_weight, post_bias, weight, bias, norm, scale, eps):
    """The arguments that both passes share, and the parameters' type."""
    dt = _dtype(name, x)
    d = x.shape[-1] if x.dim() else 0
    if d < 1:
        raise ValueError(f"{name}: x needs a last dimension of at least 1")
    if f.shape != x.shape or f.dtype != x.dtype:
        raise ValueError(f"{name}: f must have x's shape and type")
    if norm not in _NORMS:
        raise ValueError(f"{name}: norm must be one of {', '.join(_NORMS)}")
    if not post and (post_weight is not None or post_bias is not None):
        raise ValueError(f"{name}: post_weight and post_bias belong to the norm after the block: pass post=True")
    if not pre and (weight is not None or bias is not None):
        raise ValueError(f"{name}: weight and bias belong to the norm before the next block: pass pre=True")
    gate_rows = gate is not None and x.dim() > 1 and gate.shape == x.shape
    if gate_rows and gate.dtype != x.dtype:
        raise ValueError(f"{name}: a gate of x's shape must have its type")
    ptype = None
    for p in (post_weight, post_bias, weight, bias, None if gate_rows else gate):
        if p is None:
            continue
        if p.shape != x.shape[-1:] or p.dtype not in (x.dtype, torch.float32):
            raise ValueError(f"{name}: parameters and a shared gate must be ({d},) of x's type or float32")
        if ptype not in (None, p.dtype):
            raise ValueError(f"{name}: parameters and a shared gate must have one type")
        ptype = p.dtype
    ptype = x.dtype if ptype is None else ptype
    xm, fm = _rows(x), _rows(f)
    gm = None if gate is None else _rows(gate) if gate_rows else _dense(gate)
    w = _dense(post_weight), _dense(post_bias), _dense(weight), _dense(bias)
    head = (dt, _DTYPES[ptype], xm.shape[0], d, _NORMS[norm], post, pre, gate_rows, scale, eps, xm.data_ptr(), _stride(xm),
            fm.data_ptr(), _stride(fm), _address(gm), _stride(gm) if gate_rows else 0, _address(w[0]), _address(w[1]), _address(w[2]),
            _address(w[3]))
    return head, (xm, fm, gm, w), ptype   # the tensors, which may be copies, have to live until the call


def block_norm_forward(x, f, gate=None, scale=1.0, post=False, post_weight=None, post_bias=None, pre=True, weight=None, bias=None,
                       norm="layer", eps=1e-5, stream=None):
    """(h, y, stats) of what stands between two blocks of a residual tower, for
    the residual stream x and a block's output f:

        u = norm(f) * post_weight + post_bias, or f without post
        h = scale * x + gate * u
        y = norm(h) * weight + bias, or None without pre

    x, f: (..., d), float32, bfloat16 or float16. gate: (d,), or of x's shape and
    type. post_weight, post_bias, weight, bias, a shared gate: (d,) of x's type
    or float32, all of one; any may be None. norm: "layer" or "rms". stats
    (float32, (4, rows)) is what block_norm_backward takes."""
    _device("block_norm", x, f, gate, post_weight, post_bias, weight, bias)
    other = _at(x, stream, x, f, gate, post_weight, post_bias, weight, bias)
    if other is not None:
        with other:
            return block_norm_forward(x, f, gate, scale, post, post_weight, post_bias, pre, weight, bias, norm, eps)
    head, keep, _ = _block("block_norm", x, f, gate, post, pre, post_weight, post_bias, weight, bias, norm, scale, eps)
    h = torch.empty_like(x, memory_format=torch.contiguous_format)
    y = torch.empty_like(h) if pre else None
    stats = torch.empty((4, head[2]), dtype=torch.float32, device=x.device)
    rc = _lib().boa_block_norm(_pack_block(*head, h.data_ptr(), _address(y), stats.data_ptr(), *_NO_GRADIENTS),
                               _current_stream(x.get_device()))
    if rc:
        _check(rc)
    return h, y, stats


def block_norm_backward(dh, dy, x, f, stats, gate=None, scale=1.0, post=False, post_weight=None, post_bias=None, pre=True,
                        weight=None, bias=None, norm="layer", need_gate=True, need_params=True, stream=None):
    """Gradients of block_norm_forward from those of h and y (either may be
    None): a BlockNormGrads with those of x and f, of the gate (need_gate) and of
    the parameters that there are (need_params)."""
    _device("block_norm_backward", x, f, stats, gate, post_weight, post_bias, weight, bias, dh, dy)
    if dh is None and dy is None:
        raise ValueError("block_norm_backward: neither dh nor dy")
    if dy is not None and not pre:
        raise ValueError("block_norm_backward: dy without pre")
    for g in (dh, dy):
        if g is not None and (g.shape != x.shape or g.dtype != x.dtype):
            raise ValueError("block_norm_backward: dh and dy must have x's shape and type")
    if stats.dtype != torch.float32 or stats.dim() != 2 or stats.shape[0] != 4 or not stats.is_contiguous() \
            or x.dim() and stats.shape[1] * x.shape[-1] != x.numel():
        raise ValueError("block_norm_backward: stats must be the tensor of the forward pass")
    other = _at(x, stream, dh, dy, x, f, stats, gate, post_weight, post_bias, weight, bias)
    if other is not None:
        with other:
            return block_norm_backward(dh, dy, x, f, stats, gate, scale, post, post_weight, post_bias, pre, weight, bias, norm,
                                       need_gate, need_params)
    head, keep, ptype = _block("block_norm_backward", x, f, gate, post, pre, post_weight, post_bias, weight, bias, norm, scale, 0.0)
    dhm, dym = None if dh is None else _rows(dh), None if dy is None else _rows(dy)
    dev, rows, d, gate_rows = x.device, head[2], head[3], head[7]
    r = BlockNormGrads(torch.empty(x.shape, dtype=x.dtype, device=dev), torch.empty(x.shape, dtype=x.dtype, device=dev))
    vector = lambda wanted: torch.empty((d,), dtype=ptype, device=dev) if wanted else None  # noqa: E731
    if gate is not None and need_gate:
        r.dgate = torch.empty(x.shape, dtype=x.dtype, device=dev) if gate_rows else vector(True)
    r.dpost_weight, r.dpost_bias, r.dweight, r.dbias = (vector(need_params and p is not None)
                                                        for p in (post_weight, post_bias, weight, bias))
    ws = None
    if any(t is not None for t in (r.dpost_weight, r.dpost_bias, r.dweight, r.dbias)) or r.dgate is not None and not gate_rows:
        ws = _workspace(x, _lib().boa_block_norm_backward_workspace(rows, d))
    a = _pack_block(*head, 0, 0, stats.data_ptr(), _address(dhm), 0 if dhm is None else _stride(dhm), _address(dym),
                    0 if dym is None else _stride(dym), r.dx.data_ptr(), r.df.data_ptr(), _address(r.dgate), _address(r.dpost_weight),
                    _address(r.dpost_bias), _address(r.dweight), _address(r.dbias), _address(ws), 0 if ws is None else ws.numel())
    _check(_lib().boa_block_norm_backward(a, _current_stream(dev.index)))
    return r


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, gate, post_weight, post_bias, weight, bias, scale, post, pre, norm, eps):
        h, y, stats = block_norm_forward(x, f, gate, scale, post, post_weight, post_bias, pre, weight, bias, norm, eps)
        ctx.save_for_backward(x, f, gate, post_weight, post_bias, weight, bias, stats)
        ctx.args = scale, post, pre, norm
        ctx.set_materialize_grads(False)
        return h, y

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dy):
        x, f, gate, post_weight, post_bias, weight, bias, stats = ctx.saved_tensors
        scale, post, pre, norm = ctx.args
        if dh is None and dy is None:
            return (None,) * 12
        need = ctx.needs_input_grad
        r = block_norm_backward(dh, dy, x, f, stats, gate, scale, post, post_weight, post_bias, pre, weight, bias, norm, need[2],
                                any(need[3:7]))
        return r.dx, r.df, r.dgate, r.dpost_weight, r.dpost_bias, r.dweight, r.dbias, None, None, None, None, None


def block_norm(x, f, gate=None, scale=1.0, post=False, post_weight=None, post_bias=None, pre=True, weight=None, bias=None,
               norm="layer", eps=1e-5):
    """(h, y) of block_norm_forward, for autograd."""
    return _BlockNorm.apply(x, f, gate, post_weight, post_bias, weight, bias, scale, post, pre, norm, eps)


# ---------------------------------------------------------------------------
# orthogonalised updates

def orthogonalize(update, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, stream=None):
    """Newton-Schulz orthogonalisation of the last two dimensions of update, as
    an optimiser of weight matrices applies it to a momentum: x = update /
    (|update| + eps), then `steps` times x = a x + (b x x' + c (x x')^2) x, which
    takes the singular values towards 1 and keeps the singular vectors.

    update: (..., rows, cols), float32, bfloat16 or float16; the result has its
    type. coefficients: (a, b, c) for every step, or one such triple a step
    (`steps` of them). Updates of one shape are best passed together. Not seen by
    autograd."""
    _device("orthogonalize", update)
    dt = _dtype("orthogonalize", update)
    if update.dim() < 2 or update.shape[-1] < 1 or update.shape[-2] < 1:
        raise ValueError("orthogonalize: update must be (..., rows, cols)")
    if not 1 <= steps <= 32:
        raise ValueError("orthogonalize: steps must be 1 to 32")
    each = list(coefficients)
    if len(each) == 3 and not hasattr(each[0], "__len__"):
        each = [each] * steps
    if len(each) != steps or any(len(c) != 3 for c in each):
        raise ValueError("orthogonalize: coefficients must be (a, b, c), or one such triple a step")
    other = _at(update, stream, update)
    if other is not None:
        with other:
            return orthogonalize(update, steps, coefficients, eps)
    rows, cols = update.shape[-2:]
    u = update if update.dim() == 3 else update.reshape(-1, rows, cols)
    if cols > 1 and u.stride(2) != 1 or rows > 1 and u.stride(1) < cols:
        u = u.contiguous()
    out = torch.empty(update.shape, dtype=update.dtype, device=update.device)
    flat = array("f", [v for c in each for v in c])
    a = _pack_orth(dt, rows, cols, u.shape[0], u.data_ptr(), u.stride(1) if rows > 1 else cols, u.stride(0), steps,
                   flat.buffer_info()[0], eps, out.data_ptr())
    n = _lib().boa_orthogonalize_workspace(a)
    if n < 0:
        _check(n)
    ws = _workspace(update, n) if n else None
    _check(_lib().boa_orthogonalize(a, _ptr(ws), n, _current_stream(update.get_device())))
    return out
