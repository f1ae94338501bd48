"""ctypes binding of include/dblp_worker.h: the two ends of a worker's training step.

Same names and meanings as the C entry points.  Tensors are device tensors, outputs and workspaces the
caller's; the calls enqueue on `stream` (a raw hipStream_t; default: torch's current stream of the
tensors' device).  Tensors used on another stream than the one they were allocated on need what torch
asks for there (`record_stream`, or the caller's own events).  Shapes, types and devices are checked
here, everything else by the library.  Matrices may have any row stride; columns must be adjacent.
"""
from __future__ import annotations

import ctypes

from .binding import EINVAL, OK, DblpError, lib

F32, BF16, F16 = 0, 1, 2
EXPORTS = ["dblp_embed", "dblp_embed_grad", "dblp_embed_grad_workspace", "dblp_dropout", "dblp_token_logprobs",
           "dblp_policy_loss", "dblp_logits_workspace", "dblp_worker_error"]


class Drop(ctypes.Structure):
    """dblp_drop: a dropout mask.  d_draw: a device tensor of one int64 that is added to `draw` when the kernel runs."""
    _fields_ = [("seed", ctypes.c_uint64), ("draw", ctypes.c_uint64), ("d_draw", ctypes.c_void_p), ("p", ctypes.c_double)]

    def __init__(self, seed, draw, p, d_draw=None):
        if d_draw is not None and not (d_draw.is_cuda and d_draw.numel() == 1 and d_draw.element_size() == 8 and not d_draw.is_floating_point()):
            _bad("d_draw: must be one 64-bit integer on the GPU")
        super().__init__(seed, draw, None if d_draw is None else d_draw.data_ptr(), p)
        self._draw = d_draw                      # kept alive with the mask


_lib = None
_torch = None
_raw_stream = None               # torch's current stream of a device as an address, without an object for it (2 us less a call)
_types = {}


def _load():
    global _lib, _torch, _raw_stream
    import torch
    L = lib()
    vp, u64, u32, i32, f32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_float
    drop = ctypes.POINTER(Drop)
    L.dblp_embed.argtypes = [i32, vp, vp, u64, u32, vp, u64, u64, i32, f32, vp, vp, u64, u64, drop, vp, u64, i32]
    L.dblp_embed_grad.argtypes = [i32, vp, vp, u64, u32, u64, f32, drop, vp, u64, i32, vp, u64, vp, u64, vp, u64]
    L.dblp_embed_grad_workspace.argtypes = [u64, u64, u32]
    L.dblp_embed_grad_workspace.restype = u64
    L.dblp_dropout.argtypes = [i32, vp, u64, u32, vp, u64, vp, u64, drop, vp, u64, i32]
    L.dblp_token_logprobs.argtypes = [i32, vp, u64, u32, vp, u64, i32, vp, vp, vp, vp, u64]
    L.dblp_policy_loss.argtypes = [i32, vp, u64, u32, vp, u64, i32, vp, vp, vp, vp, vp, f32, f32, f32, f32, vp, u64, vp, vp, vp, u64]
    L.dblp_logits_workspace.argtypes = [u64, u32]
    L.dblp_logits_workspace.restype = u64
    L.dblp_worker_error.restype = ctypes.c_char_p
    _types.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    _torch = torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _lib = L
    return L


def _bad(why):
    raise DblpError(EINVAL, why)


def _check(rc):
    if rc != OK:
        raise DblpError(rc, _lib.dblp_worker_error().decode())


def _matrix(name, t, dev, rows, cols, dtype=None):
    """(address, row stride) of a matrix; rows or cols None: any."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        _bad(f"{name}: shape {tuple(shape)} where ({rows}, {cols}) is expected")
    if stride[1] != 1 and shape[1] > 1:
        _bad(f"{name}: columns must be adjacent")
    if t.device != dev:
        _bad(f"{name}: on {t.device}, not {dev}")
    if t.dtype not in _types or (dtype is not None and t.dtype != dtype):
        _bad(f"{name}: type {t.dtype}")
    return t.data_ptr(), stride[0]


def _vector(name, t, dev, n, dtype):
    if t is None:
        return None
    shape = t.shape
    if len(shape) != 1 or shape[0] != n or t.dtype != dtype or t.device != dev or (n > 1 and not t.is_contiguous()):
        _bad(f"{name}: {tuple(shape)} {t.dtype} on {t.device} where {n} adjacent {dtype} on {dev} are expected")
    return t.data_ptr()


def _mask(drop, dev):
    if drop is not None and (type(drop) is not Drop or (drop._draw is not None and drop._draw.device != dev)):
        _bad(f"drop: must be a Drop, its d_draw on {dev}")
    return drop


def _shape(name, t):
    """(rows, columns), device."""
    if t.ndim != 2:
        _bad(f"{name}: shape {tuple(t.shape)}, not that of a matrix")
    return t.shape, t.device


def _space(t, dev):
    if t.device != dev or not t.is_contiguous():
        _bad(f"workspace: must be contiguous and on {dev}")
    return t.data_ptr(), t.nbytes


def _place(dev, stream):
    """(device ordinal, stream) of a call."""
    if dev.type != "cuda":
        _bad(f"tensors must be on the GPU, not on {dev}")
    if stream is None:
        stream = _raw_stream(dev.index) if _raw_stream else _torch.cuda.current_stream(dev).cuda_stream
    return dev.index, stream


def embed(tokens, table, out, scale=1.0, positions=None, pos_table=None, drop=None, stream=None):
    """out[t] = drop(scale * table[tokens[t]] + pos_table[positions[t]])."""
    L = _lib or _load()
    n, ((_, dim), dev) = tokens.numel(), _shape("table", table)
    index, stream = _place(dev, stream)
    p, p_stride = _matrix("table", table, dev, None, dim)
    o, o_stride = _matrix("out", out, dev, n, dim)
    q, q_stride, n_pos = None, 0, 0
    if pos_table is not None:
        q, q_stride = _matrix("pos_table", pos_table, dev, None, dim, table.dtype)
        n_pos = pos_table.shape[0]
    _check(L.dblp_embed(index, stream, _vector("tokens", tokens, dev, n, _torch.int64), n, dim, p, p_stride, table.shape[0], _types[table.dtype],
                        scale, _vector("positions", positions, dev, n, _torch.int64), q, q_stride, n_pos, _mask(drop, dev), o, o_stride, _types[out.dtype]))


def embed_grad_workspace(n_tokens, vocab, dim) -> int:
    """Bytes of embed_grad's workspace."""
    return (_lib or _load()).dblp_embed_grad_workspace(n_tokens, vocab, dim)


def embed_grad(tokens, dy, grad, workspace, scale=1.0, drop=None, base=None, stream=None):
    """grad[v] = base[v] + scale * sum of drop(dy[t]) over the tokens that are v; base None: zeros, base grad: in place."""
    L = _lib or _load()
    n, ((vocab, dim), dev) = tokens.numel(), _shape("grad", grad)
    index, stream = _place(dev, stream)
    g, g_stride = _matrix("grad", grad, dev, None, dim, _torch.float32)
    d, d_stride = _matrix("dy", dy, dev, n, dim)
    b, b_stride = (None, 0) if base is None else _matrix("base", base, dev, vocab, dim, _torch.float32)
    _check(L.dblp_embed_grad(index, stream, _vector("tokens", tokens, dev, n, _torch.int64), n, dim, vocab, scale, _mask(drop, dev), d, d_stride, _types[dy.dtype],
                             b, b_stride, g, g_stride, *_space(workspace, dev)))


def dropout(x, y, drop, residual=None, stream=None):
    """y = drop(x) + residual; on y's gradient, without a residual, it is the gradient of x."""
    L = _lib or _load()
    (rows, cols), dev = _shape("x", x)
    index, stream = _place(dev, stream)
    a, a_stride = _matrix("x", x, dev, rows, cols)
    o, o_stride = _matrix("y", y, dev, rows, cols, x.dtype)
    r, r_stride = (None, 0) if residual is None else _matrix("residual", residual, dev, rows, cols, x.dtype)
    _check(L.dblp_dropout(index, stream, rows, cols, a, a_stride, r, r_stride, _mask(drop, dev), o, o_stride, _types[x.dtype]))


def logits_workspace(n_tokens, vocab) -> int:
    """Bytes of token_logprobs' and policy_loss' workspace."""
    return (_lib or _load()).dblp_logits_workspace(n_tokens, vocab)


def token_logprobs(logits, targets, logp, workspace, lse=None, stream=None):
    """logp[t] = logits[t, targets[t]] - lse[t]; 0 where the target is none."""
    L = _lib or _load()
    ((n, vocab), dev), f32 = _shape("logits", logits), _torch.float32
    index, stream = _place(dev, stream)
    x, x_stride = _matrix("logits", logits, dev, n, vocab)
    _check(L.dblp_token_logprobs(index, stream, n, vocab, x, x_stride, _types[logits.dtype], _vector("targets", targets, dev, n, _torch.int64),
                                 _vector("logp", logp, dev, n, f32), _vector("lse", lse, dev, n, f32), *_space(workspace, dev)))


def policy_loss(logits, targets, advantages, weights, stats, workspace, old_logp=None, ref_logp=None, dlogits=None, logp=None,
                clip=(0.2, 0.2), kl_coef=0.0, grad_scale=1.0, stream=None):
    """stats = loss, its policy and KL sums, tokens clipped and counted; dlogits = grad_scale * d loss / d logits (in place: dlogits=logits)."""
    L = _lib or _load()
    ((n, vocab), dev), f32 = _shape("logits", logits), _torch.float32
    index, stream = _place(dev, stream)
    x, x_stride = _matrix("logits", logits, dev, n, vocab)
    d, d_stride = (None, 0) if dlogits is None else _matrix("dlogits", dlogits, dev, n, vocab, logits.dtype)
    _check(L.dblp_policy_loss(index, stream, n, vocab, x, x_stride, _types[logits.dtype], _vector("targets", targets, dev, n, _torch.int64),
                              _vector("advantages", advantages, dev, n, f32), _vector("weights", weights, dev, n, f32),
                              _vector("old_logp", old_logp, dev, n, f32), _vector("ref_logp", ref_logp, dev, n, f32), clip[0], clip[1], kl_coef,
                              grad_scale, d, d_stride, _vector("logp", logp, dev, n, f32), _vector("stats", stats, dev, 5, f32),
                              *_space(workspace, dev)))
