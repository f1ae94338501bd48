"""ctypes binding of include/dblp_layers.h: a worker's matrix products, their gradients, and the update of a mean gradient.

Same names and meanings as the C entry points, same conventions as the operators of `worker`: device tensors, outputs and
workspaces the caller's, `stream` a raw hipStream_t (default: torch's current stream of the tensors' device).  Shapes, types and
devices are checked here, everything else by the library.
"""
from __future__ import annotations

import ctypes

from . import worker
from .worker import _bad, _check, _matrix, _place, _shape, _space, _types, _vector

ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
EXPORTS = ["dblp_linear", "dblp_linear_grad_input", "dblp_linear_grad_weight", "dblp_linear_workspace", "dblp_activation_grad",
           "dblp_orthogonalize", "dblp_orthogonalize_workspace"]

_lib = None
_f32 = None


def _load():
    global _lib, _f32
    L = worker._lib or worker._load()
    vp, u64, u32, i32, f32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_float
    L.dblp_linear.argtypes = [i32, vp, u64, u32, u32, vp, u64, vp, u64, i32, vp, i32, i32, vp, u64, vp, u64, vp, u64, i32, vp, u64]
    L.dblp_linear_grad_input.argtypes = [i32, vp, u64, u32, u32, vp, u64, vp, u64, i32, vp, u64, i32, vp, u64, vp, u64, i32, vp, u64]
    L.dblp_linear_grad_weight.argtypes = [i32, vp, u64, u32, u32, vp, u64, vp, u64, i32, vp, u64, vp, u64, vp, vp, vp, u64]
    L.dblp_linear_workspace.argtypes = [u64, u32, u32]
    L.dblp_linear_workspace.restype = u64
    L.dblp_activation_grad.argtypes = [i32, vp, u64, u32, vp, u64, vp, u64, i32, vp, u64, i32]
    L.dblp_orthogonalize.argtypes = [i32, vp, u64, u32, u32, vp, u64, u64, i32, ctypes.POINTER(ctypes.c_double), u32, f32, vp, u64, u64, f32, vp, u64, u64, i32, vp, u64]
    L.dblp_orthogonalize_workspace.argtypes = [u64, u32, u32]
    L.dblp_orthogonalize_workspace.restype = u64
    _f32 = worker._torch.float32
    _lib = L
    return L


def _activation(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        _bad(f"activation: {name!r}, not one of {', '.join(repr(k) for k in ACTIVATIONS)}")


def _sizes(*sizes):
    """The library takes columns as 32-bit numbers: larger ones must not come to it as others."""
    if any(n >= 1 << 31 for n in sizes):
        _bad(f"size out of range: {sizes}")


def _type(name, t):
    if t.dtype not in _types:
        _bad(f"{name}: type {t.dtype}")
    return _types[t.dtype]


def linear_workspace(n_tokens, in_features, out_features) -> int:
    """Bytes of linear's, linear_grad_input's and linear_grad_weight's workspace."""
    _sizes(in_features, out_features)
    return (_lib or _load()).dblp_linear_workspace(n_tokens, in_features, out_features)


def linear(x, weight, out, workspace, bias=None, activation=None, residual=None, pre=None, stream=None):
    """out = act(x weight^T + bias) + residual; pre: a tensor for what the activation is taken of."""
    L = _lib or _load()
    (n, inner), dev = _shape("x", x)
    index, stream = _place(dev, stream)
    p, p_stride = _matrix("x", x, dev, n, inner)
    w, w_stride = _matrix("weight", weight, dev, None, inner, x.dtype)
    outer = weight.shape[0]
    _sizes(n, inner, outer)
    o, o_stride = _matrix("out", out, dev, n, outer)
    r, r_stride = (None, 0) if residual is None else _matrix("residual", residual, dev, n, outer, out.dtype)
    z, z_stride = (None, 0) if pre is None else _matrix("pre", pre, dev, n, outer, out.dtype)
    b, b_type = (None, 0) if bias is None else (_vector("bias", bias, dev, outer, bias.dtype), _type("bias", bias))
    _check(L.dblp_linear(index, stream, n, inner, outer, p, p_stride, w, w_stride, _types[x.dtype], b, b_type, _activation(activation), r, r_stride,
                         o, o_stride, z, z_stride, _types[out.dtype], *_space(workspace, dev)))


def linear_grad_input(dy, weight, dx, workspace, pre=None, activation=None, base=None, stream=None):
    """dx = (dy weight) act'(pre) + base; pre: that of the layer whose result x was (None: no factor)."""
    L = _lib or _load()
    (n, outer), dev = _shape("dy", dy)
    index, stream = _place(dev, stream)
    d, d_stride = _matrix("dy", dy, dev, n, outer)
    w, w_stride = _matrix("weight", weight, dev, outer, None, dy.dtype)
    inner = weight.shape[1]
    _sizes(n, inner, outer)
    o, o_stride = _matrix("dx", dx, dev, n, inner)
    z, z_stride = (None, 0) if pre is None else _matrix("pre", pre, dev, n, inner, dx.dtype)
    b, b_stride = (None, 0) if base is None else _matrix("base", base, dev, n, inner, dx.dtype)
    _check(L.dblp_linear_grad_input(index, stream, n, inner, outer, d, d_stride, w, w_stride, _types[dy.dtype], z, z_stride, _activation(activation),
                                    b, b_stride, o, o_stride, _types[dx.dtype], *_space(workspace, dev)))


def linear_grad_weight(dy, x, grad, workspace, base=None, bias_grad=None, bias_base=None, stream=None):
    """grad = base + dy^T x, bias_grad = bias_base + dy's sums over the tokens; no base: zeros, base grad: in place."""
    L = _lib or _load()
    (n, outer), dev = _shape("dy", dy)
    index, stream = _place(dev, stream)
    d, d_stride = _matrix("dy", dy, dev, n, outer)
    p, p_stride = _matrix("x", x, dev, n, None, dy.dtype)
    inner = x.shape[1]
    _sizes(n, inner, outer)
    g, g_stride = _matrix("grad", grad, dev, outer, inner, _f32)
    b, b_stride = (None, 0) if base is None else _matrix("base", base, dev, outer, inner, _f32)
    _check(L.dblp_linear_grad_weight(index, stream, n, inner, outer, d, d_stride, p, p_stride, _types[dy.dtype], b, b_stride, g, g_stride,
                                     _vector("bias_base", bias_base, dev, outer, _f32), _vector("bias_grad", bias_grad, dev, outer, _f32),
                                     *_space(workspace, dev)))


def activation_grad(dy, pre, dz, activation, stream=None):
    """dz = dy act'(pre)."""
    L = _lib or _load()
    (rows, cols), dev = _shape("dy", dy)
    index, stream = _place(dev, stream)
    d, d_stride = _matrix("dy", dy, dev, rows, cols)
    z, z_stride = _matrix("pre", pre, dev, rows, cols, dy.dtype)
    o, o_stride = _matrix("dz", dz, dev, rows, cols, dy.dtype)
    _sizes(rows, cols)
    _check(L.dblp_activation_grad(index, stream, rows, cols, d, d_stride, z, z_stride, _activation(activation), o, o_stride, _types[dy.dtype]))


def _matrices(name, t, dev, shape, dtype=None):
    """(address, row stride, step) of one matrix or of several."""
    if t.ndim not in (2, 3) or (shape is not None and tuple(t.shape) != shape):
        _bad(f"{name}: shape {tuple(t.shape)} where {shape or 'that of a matrix, or of several'} is expected")
    stride = t.stride()
    if stride[-1] != 1 and t.shape[-1] > 1:
        _bad(f"{name}: columns must be adjacent")
    if t.device != dev:
        _bad(f"{name}: on {t.device}, not {dev}")
    if dtype is not None and t.dtype != dtype:
        _bad(f"{name}: type {t.dtype}")
    _type(name, t)
    return t.data_ptr(), stride[-2], stride[0] if t.ndim == 3 else 0


def orthogonalize_workspace(count, rows, cols) -> int:
    """Bytes of orthogonalize's workspace."""
    _sizes(rows, cols)
    return (_lib or _load()).dblp_orthogonalize_workspace(count, rows, cols)


def orthogonalize(g, out, workspace, scale=1.0, base=None, base_scale=1.0, steps=5, coefficients=None, stream=None):
    """out = base_scale base + scale X, X the nearly orthogonal matrix of g's directions; g: a matrix, or [count, rows, cols].

    coefficients: (a, b, c) for every step, or one such triple a step; None: the library's."""
    L = _lib or _load()
    dev = g.device
    index, stream = _place(dev, stream)
    p, p_stride, p_step = _matrices("g", g, dev, None)
    shape = tuple(g.shape)
    o, o_stride, o_step = _matrices("out", out, dev, shape)
    b, b_stride, b_step = (None, 0, 0) if base is None else _matrices("base", base, dev, shape, out.dtype)
    _sizes(*shape)
    if not 0 <= steps <= 16:
        _bad(f"steps: {steps}, not in 0..16")
    table = None
    if coefficients is not None:
        rows = list(coefficients)
        if len(rows) == 3 and not hasattr(rows[0], "__len__"):
            rows = [rows] * steps
        if len(rows) != steps or any(len(r) != 3 for r in rows):
            _bad(f"coefficients: three numbers, or three for each of {steps} steps, are expected")
        table = (ctypes.c_double * (3 * steps))(*[v for r in rows for v in r])
    count = shape[0] if len(shape) == 3 else 1
    _check(L.dblp_orthogonalize(index, stream, count, shape[-2], shape[-1], p, p_stride, p_step, _types[g.dtype], table, steps, scale, b, b_stride, b_step, base_scale,
                                o, o_stride, o_step, _types[out.dtype], *_space(workspace, dev)))
