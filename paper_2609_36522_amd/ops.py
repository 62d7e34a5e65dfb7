"""Operators of a text-conditioned noise network (the C ABI in include/paraanya_ops.h): layer norm,
cross attention to a prompt encoder's states, a shared projection with the low-rank adapters of many
requests, group norm with an activation, a gated feed-forward block, a projection in 8-bit integers.

Argument marshalling only, as in :mod:`binding`: every product and sum runs in the library's HIP
kernels. Tensors lie on the current device; kernels run on torch's current stream, outputs and
workspaces come from torch's allocator on that stream. :func:`layer_norm`, :func:`cross_attention`,
:func:`group_norm` and :func:`feed_forward` take part in autograd, for first derivatives (a gradient's
gradient is refused); the ``*_forward`` and ``*_backward`` functions do not. All may be captured into a graph; while a
backward pass is captured, no graph of autograd that was built outside may hold the same leaves (torch would accumulate their
gradients on that graph's stream).
"""
from __future__ import annotations

import ctypes as C
import functools
import math
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

PA_F32, PA_BF16, PA_F16 = 0, 1, 2
PA_MASK_NONE, PA_MASK_BOOL, PA_MASK_ADD = 0, 1, 2
PA_NORM_MAX_COLS = 1 << 20
PA_LORA_MAX_RANK = 128
HEAD_DIM_MAX = 128
PA_ACT_NONE, PA_ACT_SILU, PA_ACT_GELU = 0, 1, 2
PA_GROUP_MAX_CHANNELS = 4096
PA_INT8_MAX_IN = (1 << 17) - 1

EXPORTED = ("paraanya_layer_norm", "paraanya_layer_norm_backward", "paraanya_layer_norm_backward_workspace",
            "paraanya_cross_attention", "paraanya_cross_attention_workspace",
            "paraanya_cross_attention_backward", "paraanya_cross_attention_backward_workspace",
            "paraanya_lora_linear", "paraanya_lora_linear_workspace",
            "paraanya_group_norm", "paraanya_group_norm_workspace",
            "paraanya_group_norm_backward", "paraanya_group_norm_backward_workspace",
            "paraanya_feed_forward", "paraanya_feed_forward_saved", "paraanya_feed_forward_workspace",
            "paraanya_feed_forward_backward", "paraanya_feed_forward_backward_workspace",
            "paraanya_quantize_rows", "paraanya_int8_linear")

_ACT = {None: PA_ACT_NONE, "silu": PA_ACT_SILU, "gelu": PA_ACT_GELU}
_DTYPE = {torch.float32: PA_F32, torch.bfloat16: PA_BF16, torch.float16: PA_F16}


class Norm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("dtype", C.c_int32), ("param_dtype", C.c_int32),
                ("eps", C.c_double), ("x_stride", C.c_int64), ("y_stride", C.c_int64), ("dx_stride", C.c_int64)]


class Cross(C.Structure):
    _fields_ = [("batch", C.c_int64), ("q_len", C.c_int64), ("kv_len", C.c_int64), ("q_heads", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_double),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("o_stride", C.c_int64 * 3), ("kv_lens", C.c_void_p), ("mask", C.c_void_p),
                ("mask_kind", C.c_int32), ("pad", C.c_int32), ("mask_stride", C.c_int64)]


class CrossGrad(C.Structure):
    _fields_ = [("do_stride", C.c_int64 * 3), ("dq_stride", C.c_int64 * 3), ("dk_stride", C.c_int64 * 3),
                ("dv_stride", C.c_int64 * 3)]


class Lora(C.Structure):
    _fields_ = [("rows", C.c_int64), ("in_features", C.c_int32), ("out_features", C.c_int32), ("rank", C.c_int32),
                ("adapters", C.c_int32), ("requests", C.c_int32), ("dtype", C.c_int32), ("x_stride", C.c_int64),
                ("w_stride", C.c_int64), ("y_stride", C.c_int64), ("offsets", C.c_void_p), ("ids", C.c_void_p),
                ("scales", C.c_void_p)]


class GroupNorm(C.Structure):
    _fields_ = [("batch", C.c_int64), ("pixels", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32),
                ("dtype", C.c_int32), ("param_dtype", C.c_int32), ("activation", C.c_int32), ("pad", C.c_int32),
                ("eps", C.c_double), ("x_stride", C.c_int64 * 2), ("y_stride", C.c_int64 * 2), ("dx_stride", C.c_int64 * 2)]


class Feed(C.Structure):
    _fields_ = [("rows", C.c_int64), ("in_features", C.c_int32), ("hidden_features", C.c_int32), ("out_features", C.c_int32),
                ("dtype", C.c_int32), ("activation", C.c_int32), ("alignment", C.c_int32), ("x_stride", C.c_int64),
                ("gate_stride", C.c_int64), ("up_stride", C.c_int64), ("down_stride", C.c_int64), ("y_stride", C.c_int64)]


class FeedGrad(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dx", "dgate", "dup", "ddown", "dgate_bias", "dup_bias", "ddown_bias")]


class Quantize(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("dtype", C.c_int32), ("pad", C.c_int32), ("x_stride", C.c_int64),
                ("q_stride", C.c_int64)]


class Int8Linear(C.Structure):
    _fields_ = [("rows", C.c_int64), ("in_features", C.c_int32), ("out_features", C.c_int32), ("dtype", C.c_int32),
                ("pad", C.c_int32), ("x_stride", C.c_int64), ("w_stride", C.c_int64), ("y_stride", C.c_int64)]


_LIB = None


def _library():
    global _LIB
    if _LIB is None:
        lib = B.load_library()
        P, Z = C.c_void_p, C.c_size_t
        lib.paraanya_layer_norm.argtypes = [P, P, P, P, P, P, P, P]
        lib.paraanya_layer_norm_backward.argtypes = [P, P, P, P, P, P, P, P, P, P, Z, P]
        lib.paraanya_cross_attention.argtypes = [P, P, P, P, P, P, P, Z, P]
        lib.paraanya_cross_attention_backward.argtypes = [P, P, P, P, P, P, P, P, P, P, P, P, Z, P]
        lib.paraanya_lora_linear.argtypes = [P, P, P, P, P, P, P, P, Z, P]
        lib.paraanya_group_norm.argtypes = [P, P, P, P, P, P, P, P, Z, P]
        lib.paraanya_group_norm_backward.argtypes = [P, P, P, P, P, P, P, P, P, P, P, Z, P]
        lib.paraanya_feed_forward.argtypes = [P, P, P, P, P, P, P, P, P, P, Z, P, Z, P]
        lib.paraanya_feed_forward_backward.argtypes = [P, P, P, P, P, P, P, P, Z, P, Z, P]
        lib.paraanya_quantize_rows.argtypes = [P, P, P, P, P]
        lib.paraanya_int8_linear.argtypes = [P, P, P, P, P, P, P, P]
        for name in EXPORTED:
            f = getattr(lib, name)
            f.restype = C.c_int
            if name.endswith(("_workspace", "_saved")):
                f.argtypes = [P, C.POINTER(Z)]
        lib.paraanya_feed_forward_workspace.argtypes = [P, C.c_int, C.POINTER(Z)]
        _LIB = lib
    return _LIB


def _on_device(*tensors):
    """The current stream's handle, once every tensor given is on the current device."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"expected tensors on the current CUDA device {dev}")
    return torch._C._cuda_getCurrentRawStream(dev)


def _size(query, p):
    n = C.c_size_t(0)
    B._check(query(C.byref(p), C.byref(n)))
    return n.value


def _workspace(n, like):
    return like.new_empty(n, dtype=torch.uint8) if n else None


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ layer norm
def _rows(t, N):
    """A [rows, N] view of t (a copy where its strides allow no view)."""
    if t.dim() != 2:
        t = t.reshape(-1, N)
    return t if t.stride(1) == 1 and (t.shape[0] < 2 or t.stride(0) >= N) else t.contiguous()


def _stride(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _norm_args(x, weight, bias):
    if x.dtype not in _DTYPE:
        raise ValueError(f"layer norm of {x.dtype} is not built")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("layer norm needs at least one column")
    pt = x.dtype
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        if t.shape != x.shape[-1:] or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous with {x.shape[-1]} elements")
        if t.dtype not in (x.dtype, torch.float32):
            raise ValueError(f"{name} must have x's type or float32")
        pt = t.dtype
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have one type")
    return pt


@functools.lru_cache(maxsize=256)
def _norm(M, N, dtype, param_dtype, eps, x_stride, y_stride):
    """The (constant) description of a norm and the workspace that its backward pass needs."""
    lib = _library()
    p = Norm(M, N, dtype, param_dtype, eps, x_stride, y_stride, N)
    return p, C.byref(p), _size(lib.paraanya_layer_norm_backward_workspace, p)


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of the norm over x's last dimension; mean and rstd are fp32, one per row."""
    pt = _norm_args(x, weight, bias)
    st = _on_device(x, weight, bias)
    N = x.shape[-1]
    x2 = _rows(x, N)
    M = x2.shape[0]
    _, ref, _ = _norm(M, N, _DTYPE[x.dtype], _DTYPE[pt], eps, _stride(x2), N)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = torch.empty(M, dtype=torch.float32, device=x.device)
    rstd = torch.empty(M, dtype=torch.float32, device=x.device)
    B._check(_LIB.paraanya_layer_norm(ref, x2.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), mean.data_ptr(),
                                      rstd.data_ptr(), st))
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, *, param_dtype=None):
    """(dx, dweight, dbias) from the forward pass's x, mean and rstd. dweight and dbias have
    weight's type (``param_dtype``, or x's, without a weight)."""
    if weight is not None:
        param_dtype = weight.dtype
    elif param_dtype is None:
        param_dtype = x.dtype
    _norm_args(x, weight, None)
    if param_dtype not in (x.dtype, torch.float32):
        raise ValueError("param_dtype must be x's type or float32")
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have x's shape and type")
    N = x.shape[-1]
    x2, dy2 = _rows(x, N), _rows(dy, N)
    M = x2.shape[0]
    for t in (mean, rstd):
        if t.dtype != torch.float32 or t.numel() != M or not t.is_contiguous():
            raise ValueError(f"mean and rstd must be contiguous float32 tensors of {M} elements")
    st = _on_device(x, dy, mean, rstd, weight)
    _, ref, n = _norm(M, N, _DTYPE[x.dtype], _DTYPE[param_dtype], 0.0, _stride(x2), _stride(dy2))
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty(N, dtype=param_dtype, device=x.device)
    db = torch.empty(N, dtype=param_dtype, device=x.device)
    ws = _workspace(n, x)
    B._check(_LIB.paraanya_layer_norm_backward(ref, dy2.data_ptr(), x2.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                               _ptr(weight), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), _ptr(ws), n, st))
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.param_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(dy, x, mean, rstd, weight, param_dtype=ctx.param_dtype)
        need = ctx.needs_input_grad
        return dx if need[0] else None, dw if need[1] else None, db if need[2] else None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """The norm over x's last dimension, differentiable (once) in x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


# ------------------------------------------------------------------ cross attention
def _heads(t, name):
    """t [batch, tokens, heads, head_dim] with consecutive head elements (a copy otherwise)."""
    if t.dim() != 4:
        raise ValueError(f"{name} must have the shape [batch, tokens, heads, head_dim]")
    return t if t.stride(3) == 1 or t.shape[3] == 1 else t.contiguous()


@functools.lru_cache(maxsize=256)
def _cross(q_shape, k_shape, dtype, scale, q_stride, k_stride, v_stride, o_stride, mask_kind, mask_stride):
    """The description of an attention without its kv_lens and mask (to be copied), and the workspaces of its
    forward and backward pass (which do not depend on them)."""
    (Bn, Lq, Hq, D), (_, Lk, Hk, _) = q_shape, k_shape
    p = Cross(Bn, Lq, Lk, Hq, Hk, D, dtype, 1.0 / math.sqrt(max(D, 1)) if scale is None else scale,
              q_stride[:3], k_stride[:3], v_stride[:3], o_stride[:3])
    p.mask_kind, p.mask_stride = mask_kind, mask_stride
    if mask_kind:
        p.mask = 256          # any address: only the sizes are asked for
    lib = _library()
    return p, _size(lib.paraanya_cross_attention_workspace, p), _size(lib.paraanya_cross_attention_backward_workspace, p)


def _cross_args(q, k, v, kv_lens, mask, scale, o):
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"cross attention of {q.dtype} is not built")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k and v must have one type")
    Bn, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    if k.shape != (Bn, Lk, Hk, D) or v.shape != k.shape:
        raise ValueError("k and v must have one shape, and q's batch and head_dim")
    if Hk < 1 or Hq % Hk:
        raise ValueError("q's heads must be a multiple of k's")
    if kv_lens is not None and (kv_lens.dtype != torch.int32 or kv_lens.shape != (Bn,) or not kv_lens.is_contiguous()):
        raise ValueError(f"kv_lens must be a contiguous int32 tensor of {Bn} elements")
    kind = PA_MASK_NONE
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8, torch.float32) or mask.shape != (Bn, Lk):
            raise ValueError(f"mask must be a bool, uint8 or float32 tensor of [{Bn}, {Lk}]")
        if mask.stride(1) != 1 and Lk > 1:
            raise ValueError("a mask row's elements must be consecutive")
        kind = PA_MASK_ADD if mask.dtype == torch.float32 else PA_MASK_BOOL
    p, forward, backward = _cross(q.shape, k.shape, _DTYPE[q.dtype], scale, q.stride(), k.stride(), v.stride(), o.stride(),
                                  kind, mask.stride(0) if kind else 0)
    if kv_lens is not None or kind:
        p = Cross.from_buffer_copy(p)
        p.kv_lens = None if kv_lens is None else kv_lens.data_ptr()
        p.mask = mask.data_ptr() if kind else None
    return p, forward, backward


def cross_attention_forward(q, k, v, *, kv_lens=None, mask=None, scale=None):
    """(o, stats): softmax(scale q k^T + mask) v per head.

    q [batch, q_len, q_heads, head_dim], k and v [batch, kv_len, kv_heads, head_dim] in bf16 or fp16, of
    any strides with consecutive head elements (a stride of 0 repeats); q_heads a multiple of kv_heads.
    ``kv_lens`` (int32, [batch]) is each sample's number of states; ``mask`` [batch, kv_len] admits keys
    (bool or uint8) or is added to their scores (float32, -inf hides a key). ``scale`` defaults to
    1 / sqrt(head_dim). stats [batch, q_heads, q_len, 2] is what the backward pass needs (a score near
    the row's largest and the logarithm of the sum of exponentials past it; their sum is the log-sum-exp)."""
    q, k, v = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    st = _on_device(q, k, v, kv_lens, mask)
    p, n, _ = _cross_args(q, k, v, kv_lens, mask, scale, o)
    stats = torch.empty((q.shape[0], q.shape[2], q.shape[1], 2), dtype=torch.float32, device=q.device)
    ws = _workspace(n, q)
    B._check(_LIB.paraanya_cross_attention(C.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                           stats.data_ptr(), _ptr(ws), n, st))
    return o, stats


def cross_attention_backward(do, q, k, v, o, stats, *, kv_lens=None, mask=None, scale=None):
    """(dq, dk, dv) from the forward pass's inputs and results. A gradient has its input's full shape,
    also where the input repeats memory (an expanded tensor)."""
    q, k, v, o, do = _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), _heads(o, "o"), _heads(do, "do")
    if o.shape != q.shape or do.shape != q.shape or o.dtype != q.dtype or do.dtype != q.dtype:
        raise ValueError("o and do must have q's shape and type")
    if stats.dtype != torch.float32 or stats.shape != (q.shape[0], q.shape[2], q.shape[1], 2) or not stats.is_contiguous():
        raise ValueError("stats must be the forward pass's")
    st = _on_device(q, k, v, o, do, stats, kv_lens, mask)
    p, _, n = _cross_args(q, k, v, kv_lens, mask, scale, o)
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    dv = torch.empty(v.shape, dtype=q.dtype, device=q.device)
    g = CrossGrad(do.stride()[:3], dq.stride()[:3], dk.stride()[:3], dv.stride()[:3])
    ws = _workspace(n, q)
    B._check(_LIB.paraanya_cross_attention_backward(C.byref(p), C.byref(g), do.data_ptr(), q.data_ptr(), k.data_ptr(),
                                                    v.data_ptr(), o.data_ptr(), stats.data_ptr(), dq.data_ptr(),
                                                    dk.data_ptr(), dv.data_ptr(), _ptr(ws), n, st))
    return dq, dk, dv


class _CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, kv_lens, mask, scale):
        o, stats = cross_attention_forward(q, k, v, kv_lens=kv_lens, mask=mask, scale=scale)
        ctx.save_for_backward(q, k, v, o, stats, kv_lens, mask)
        ctx.scale = scale
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        q, k, v, o, stats, kv_lens, mask = ctx.saved_tensors
        dq, dk, dv = cross_attention_backward(do, q, k, v, o, stats, kv_lens=kv_lens, mask=mask, scale=ctx.scale)
        return dq, dk, dv, None, None, None


def cross_attention(q, k, v, *, kv_lens=None, mask=None, scale=None):
    """:func:`cross_attention_forward`'s o, differentiable (once) in q, k and v. The mask gets no gradient: one that
    requires it is refused."""
    if mask is not None and mask.requires_grad and torch.is_grad_enabled():
        raise ValueError("cross attention has no gradient for its mask: pass mask.detach()")
    return _CrossAttention.apply(q, k, v, kv_lens, mask, scale)


# ------------------------------------------------------------------ projection with adapters
@functools.lru_cache(maxsize=256)
def _lora(M, K, N, R, E, n, dtype, x_stride, w_stride):
    """The description of a projection without its offsets, ids and scales (to be copied), and its workspace."""
    p = Lora(M, K, N, R, E, n, dtype, x_stride, w_stride, N, 256, 256, None)
    return p, _size(_library().paraanya_lora_linear_workspace, p)


def lora_linear(x, weight, a, b, offsets, ids, *, scales=None, bias=None):
    """x W^T + bias + scales[i] (x A_i^T) B_i^T with the adapter i of each row's request.

    x [rows, K], weight [N, K] (row strides of their own), bias [N], a [adapters, R, K] and
    b [adapters, N, R] in bf16 or fp16. Request r is rows offsets[r] .. offsets[r + 1] - 1 and uses
    adapter ids[r] (none if negative); offsets (requests + 1) and ids are int32 tensors on the
    device, scales float32 ([adapters], 1 if absent). No gradients: an inference operator."""
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"lora linear of {x.dtype} is not built")
    for t in (weight, a, b) + (() if bias is None else (bias,)):
        if t.dtype != x.dtype:
            raise ValueError("x, weight, a, b and bias must have one type")
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, a, b, bias, scales)):
        raise ValueError("lora linear has no gradients: call it under torch.no_grad()")
    if x.dim() != 2 or weight.dim() != 2 or a.dim() != 3 or b.dim() != 3:
        raise ValueError("expected x [rows, K], weight [N, K], a [adapters, R, K] and b [adapters, N, R]")
    (M, K), N, (E, R) = x.shape, weight.shape[0], a.shape[:2]
    if weight.shape[1] != K or a.shape[2] != K or b.shape != (E, N, R) or (bias is not None and bias.shape != (N,)):
        raise ValueError("x, weight, a, b and bias do not fit together")
    n = ids.numel()
    for t, count, name in ((offsets, n + 1, "offsets"), (ids, n, "ids")):
        if t.dtype != torch.int32 or t.dim() != 1 or t.numel() != count or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor of {count} elements")
    if scales is not None and (scales.dtype != torch.float32 or scales.shape != (E,) or not scales.is_contiguous()):
        raise ValueError(f"scales must be a contiguous float32 tensor of {E} elements")
    if not (a.is_contiguous() and b.is_contiguous() and (bias is None or bias.is_contiguous())):
        raise ValueError("a, b and bias must be contiguous")
    x, weight = (t if t.stride(1) == 1 and (t.shape[0] < 2 or t.stride(0) >= K) else t.contiguous() for t in (x, weight))
    st = _on_device(x, weight, a, b, offsets, ids, scales, bias)
    y = torch.empty((M, N), dtype=x.dtype, device=x.device)
    p, size = _lora(M, K, N, R, E, n, _DTYPE[x.dtype], _stride(x), _stride(weight))
    p = Lora.from_buffer_copy(p)
    p.offsets, p.ids, p.scales = offsets.data_ptr(), ids.data_ptr(), _ptr(scales)
    ws = _workspace(size, x)
    B._check(_LIB.paraanya_lora_linear(C.byref(p), x.data_ptr(), weight.data_ptr(), _ptr(bias), a.data_ptr(), b.data_ptr(),
                                       y.data_ptr(), _ptr(ws), size, st))
    return y


# ------------------------------------------------------------------ group norm
def _pixels(t):
    """A [batch, pixels, channels] view of t with consecutive channels (a copy where its strides allow no view)."""
    B, Ch = t.shape[0], t.shape[-1]
    if t.dim() != 3:
        t = t.reshape(B, math.prod(t.shape[1:-1]), Ch)
    return t if (t.stride(2) == 1 or Ch == 1) and (t.shape[1] < 2 or t.stride(1) >= Ch) else t.contiguous()


def _activation(name):
    if name not in _ACT:
        raise ValueError(f"activation must be None, 'silu' or 'gelu', not {name!r}")
    return _ACT[name]


def _group_args(x, groups, weight, bias):
    if x.dtype not in _DTYPE:
        raise ValueError(f"group norm of {x.dtype} is not built")
    if x.dim() < 2 or x.shape[-1] < 1:
        raise ValueError("group norm needs the shape [batch, ..., channels]")
    if groups < 1 or x.shape[-1] % groups:
        raise ValueError("channels must be a multiple of groups")
    return _norm_args(x, weight, bias)


@functools.lru_cache(maxsize=256)
def _group(B_, P, Ch, G, dtype, param_dtype, act, eps, x_stride, y_stride):
    """The (constant) description of a group norm and the workspaces of its forward and backward pass."""
    lib = _library()
    p = GroupNorm(B_, P, Ch, G, dtype, param_dtype, act, 0, eps, x_stride, y_stride, (P * Ch, Ch))
    return p, C.byref(p), _size(lib.paraanya_group_norm_workspace, p), _size(lib.paraanya_group_norm_backward_workspace, p)


def group_norm_forward(x, groups, weight=None, bias=None, eps=1e-5, *, activation=None):
    """(y, mean, rstd) of the norm over pixels and the channels of each group, followed by an activation.

    x [batch, ..., channels], channels last (of a channels-last image tensor: ``x.permute(0, 2, 3, 1)``, a view), in
    float32, bf16 or fp16; weight and bias [channels], of x's type or float32. ``activation`` is None, "silu" or
    "gelu". mean and rstd are fp32, [batch, groups]."""
    act = _activation(activation)
    pt = _group_args(x, groups, weight, bias)
    st = _on_device(x, weight, bias)
    x3 = _pixels(x)
    B_, P, Ch = x3.shape
    _, ref, n, _ = _group(B_, P, Ch, groups, _DTYPE[x.dtype], _DTYPE[pt], act, eps, x3.stride()[:2], (P * Ch, Ch))
    y = x.new_empty(x.shape)
    mean = x.new_empty((B_, groups), dtype=torch.float32)
    rstd = x.new_empty((B_, groups), dtype=torch.float32)
    if P == 0:
        mean.zero_(), rstd.zero_()
    ws = _workspace(n, x)
    B._check(_LIB.paraanya_group_norm(ref, x3.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                      _ptr(ws), n, st))
    return y, mean, rstd


def group_norm_backward(dy, x, mean, rstd, weight=None, bias=None, *, activation=None, param_dtype=None, need=(True,) * 3):
    """(dx, dweight, dbias) from the forward pass's x, weight, bias, mean and rstd. dweight and dbias have the
    parameters' type (``param_dtype``, or x's, where there are none). ``need`` says which of the three are computed (None in
    the others' place)."""
    act = _activation(activation)
    if mean.dim() != 2 or mean.shape[0] != x.shape[0]:
        raise ValueError("mean and rstd must be [batch, groups]")
    groups = mean.shape[1]
    pt = _group_args(x, groups, weight, bias)
    if weight is None and bias is None and param_dtype is not None:
        pt = param_dtype
    if pt not in (x.dtype, torch.float32):
        raise ValueError("param_dtype must be x's type or float32")
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have x's shape and type")
    for t in (mean, rstd):
        if t.dtype != torch.float32 or t.shape != mean.shape or not t.is_contiguous():
            raise ValueError("mean and rstd must be contiguous float32 tensors of one shape")
    st = _on_device(x, dy, mean, rstd, weight, bias)
    x3, dy3 = _pixels(x), _pixels(dy)
    B_, P, Ch = x3.shape
    p, _, _, n = _group(B_, P, Ch, groups, _DTYPE[x.dtype], _DTYPE[pt], act, 0.0, x3.stride()[:2], (P * Ch, Ch))
    p = GroupNorm.from_buffer_copy(p)
    p.y_stride[:] = dy3.stride()[:2]
    dx = x.new_empty(x.shape) if need[0] else None
    dw = x.new_empty(Ch, dtype=pt) if need[1] else None
    db = x.new_empty(Ch, dtype=pt) if need[2] else None
    ws = _workspace(n, x)
    B._check(_LIB.paraanya_group_norm_backward(C.byref(p), dy3.data_ptr(), x3.data_ptr(), _ptr(weight), _ptr(bias), mean.data_ptr(),
                                               rstd.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db), _ptr(ws), n, st))
    return dx, dw, db


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, groups, weight, bias, eps, activation):
        y, mean, rstd = group_norm_forward(x, groups, weight, bias, eps, activation=activation)
        ctx.save_for_backward(x, weight, bias, mean, rstd)
        ctx.activation = activation
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, bias, mean, rstd = ctx.saved_tensors
        need = tuple(ctx.needs_input_grad[i] for i in (0, 2, 3))
        some = {} if all(need) else {"need": need}
        dx, dw, db = group_norm_backward(dy, x, mean, rstd, weight, bias, activation=ctx.activation, **some)
        return dx, None, dw, db, None, None


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, *, activation=None):
    """:func:`group_norm_forward`'s y, differentiable (once) in x, weight and bias."""
    return _GroupNorm.apply(x, groups, weight, bias, eps, activation)


# ------------------------------------------------------------------ gated feed-forward block
class FeedGradients(NamedTuple):
    """Gradients of :func:`feed_forward`'s arguments, of their shapes (None where not asked for)."""
    x: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]
    up: Optional[torch.Tensor]
    down: Optional[torch.Tensor]
    gate_bias: Optional[torch.Tensor]
    up_bias: Optional[torch.Tensor]
    down_bias: Optional[torch.Tensor]


@functools.lru_cache(maxsize=256)
def _feed(M, K, H, N, dtype, act, alignment, strides):
    """The (constant) description of a block and the sizes of saved, of the forward pass's workspace without and with it,
    and of the backward pass's."""
    lib = _library()
    p = Feed(M, K, H, N, dtype, act, alignment, *strides)
    sizes = [_size(lib.paraanya_feed_forward_saved, p)]
    for with_saved in (0, 1):
        n = C.c_size_t(0)
        B._check(lib.paraanya_feed_forward_workspace(C.byref(p), with_saved, C.byref(n)))
        sizes.append(n.value)
    return (p, C.byref(p), *sizes, _size(lib.paraanya_feed_forward_backward_workspace, p))


def _feed_args(x, gate, up, down, biases, activation, y=None):
    """(description, x, gate, up, down, y as matrices of consecutive elements, stream)."""
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"feed forward of {x.dtype} is not built")
    act = _activation(activation)
    if x.dim() < 1 or gate.dim() != 2 or up.dim() != 2 or down.dim() != 2:
        raise ValueError("expected x [..., K], gate and up [H, K] and down [N, H]")
    K, (H, N) = x.shape[-1], (gate.shape[0], down.shape[0])
    if gate.shape != (H, K) or up.shape != (H, K) or down.shape != (N, H) or min(K, H, N) < 1:
        raise ValueError("x, gate, up and down do not fit together")
    dt = x.dtype
    for t, n in zip(biases, (H, H, N)):
        if t is not None and (t.shape != (n,) or not t.is_contiguous()):
            raise ValueError(f"a bias must be contiguous with {n} elements")
        if t is not None and t.dtype != dt:
            raise ValueError("x, the weights, the biases and dy must have one type")
    if gate.dtype != dt or up.dtype != dt or down.dtype != dt or (y is not None and y.dtype != dt):
        raise ValueError("x, the weights, the biases and dy must have one type")
    if y is not None and y.shape != (*x.shape[:-1], N):
        raise ValueError("dy must have y's shape")
    st = _on_device(x, gate, up, down, *biases, y)
    x, gate, up, down = _rows(x, K), _rows(gate, K), _rows(up, K), _rows(down, H)
    y = None if y is None else _rows(y, N)
    at = 16 | x.data_ptr() | gate.data_ptr() | up.data_ptr() | down.data_ptr() | (0 if y is None else y.data_ptr())
    d = _feed(x.shape[0], K, H, N, _DTYPE[x.dtype], act, at & -at,
              (_stride(x), _stride(gate), _stride(up), _stride(down), N if y is None else _stride(y)))
    return d, x, gate, up, down, y, st


def feed_forward_forward(x, gate, up, down, gate_bias=None, up_bias=None, down_bias=None, *, activation="silu", save=True):
    """(y, saved): (act(x gate^T + gate_bias) * (x up^T + up_bias)) down^T + down_bias.

    x [..., K], gate and up [H, K], down [N, H] (row strides of their own), biases [H], [H], [N], in bf16 or fp16.
    ``activation`` is "silu", "gelu" or None. saved (opaque; None without ``save``) is what the backward pass
    needs: the gated product and by what its gradient gives those of the two projections."""
    d, x2, g, u, dn, _, st = _feed_args(x, gate, up, down, (gate_bias, up_bias, down_bias), activation)
    _, ref, keep, plain, with_saved, _ = d
    y = x.new_empty((*x.shape[:-1], down.shape[0]))
    saved = x.new_empty(keep, dtype=torch.uint8) if save else None
    n = with_saved if save else plain
    ws = _workspace(n, x)
    B._check(_LIB.paraanya_feed_forward(ref, x2.data_ptr(), g.data_ptr(), _ptr(gate_bias), u.data_ptr(), _ptr(up_bias), dn.data_ptr(),
                                        _ptr(down_bias), y.data_ptr(), _ptr(saved), keep, _ptr(ws), n, st))
    return y, saved


def feed_forward_backward(dy, x, gate, up, down, saved, *, activation="silu", need=(True,) * 7):
    """:class:`FeedGradients` from dy, the forward pass's inputs and what it saved. ``need`` says which of them
    are computed (x, gate, up, down and the biases in that order; a bias's comes with its weight's)."""
    d, x2, g, u, dn, dy2, st = _feed_args(x, gate, up, down, (), activation, dy)
    p, ref, keep, _, _, n = d
    if saved.dtype != torch.uint8 or saved.numel() != keep or not saved.is_contiguous():
        raise ValueError("saved must be the forward pass's")
    _on_device(saved)
    H, N = gate.shape[0], down.shape[0]
    need = list(need)
    for i in (1, 2, 3):
        need[i] = need[i] or need[i + 3]
    shapes = (x.shape, gate.shape, up.shape, down.shape, (H,), (H,), (N,))
    out = FeedGradients(*(x.new_empty(s) if k else None for s, k in zip(shapes, need)))
    ws = _workspace(n, x)
    B._check(_LIB.paraanya_feed_forward_backward(ref, C.byref(FeedGrad(*map(_ptr, out))), dy2.data_ptr(), x2.data_ptr(), g.data_ptr(),
                                                 u.data_ptr(), dn.data_ptr(), _ptr(saved), keep, _ptr(ws), n, st))
    return out


class _FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, up, down, gate_bias, up_bias, down_bias, activation):
        y, saved = feed_forward_forward(x, gate, up, down, gate_bias, up_bias, down_bias, activation=activation,
                                        save=any(ctx.needs_input_grad))
        ctx.save_for_backward(x, gate, up, down, saved)
        ctx.activation = activation
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, gate, up, down, saved = ctx.saved_tensors
        need = ctx.needs_input_grad[:7]
        g = feed_forward_backward(dy, x, gate, up, down, saved, activation=ctx.activation, need=need)
        return (*(t if k else None for t, k in zip(g, need)), None)


def feed_forward(x, gate, up, down, gate_bias=None, up_bias=None, down_bias=None, *, activation="silu"):
    """:func:`feed_forward_forward`'s y, differentiable (once) in x, the weights and the biases. Under ``torch.no_grad()``
    nothing is saved."""
    if not torch.is_grad_enabled():          # (needs_input_grad tells of the tensors alone)
        return feed_forward_forward(x, gate, up, down, gate_bias, up_bias, down_bias, activation=activation, save=False)[0]
    return _FeedForward.apply(x, gate, up, down, gate_bias, up_bias, down_bias, activation)


# ------------------------------------------------------------------ projection in 8-bit integers
def _no_gradients(what, *tensors):
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{what} has no gradients: call it under torch.no_grad()")


@functools.lru_cache(maxsize=256)
def _quantize(M, K, dtype, x_stride, q_stride):
    _library()
    p = Quantize(M, K, dtype, 0, x_stride, q_stride)
    return p, C.byref(p)


def quantize_rows(x):
    """(q, scale): x's rows as 8-bit integers, scale = max |x| / 127 of each row (float32) and q = x / scale rounded to
    the nearest integer. x [..., K] in float32, bf16 or fp16. q's rows start at multiples of 16 bytes (so a matrix of
    weights is quantized by the same call). A row that holds an infinity or a NaN has scale NaN. No gradients."""
    if x.dtype not in _DTYPE:
        raise ValueError(f"quantize rows of {x.dtype} is not built")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("quantize rows needs at least one column")
    _no_gradients("quantize rows", x)
    st = _on_device(x)
    K = x.shape[-1]
    x2 = _rows(x, K)
    M, wide = x2.shape[0], (K + 15) // 16 * 16
    _, ref = _quantize(M, K, _DTYPE[x.dtype], _stride(x2), wide)
    q = x.new_empty((*x.shape[:-1], wide), dtype=torch.int8)
    scale = x.new_empty(x.shape[:-1], dtype=torch.float32)
    B._check(_LIB.paraanya_quantize_rows(ref, x2.data_ptr(), q.data_ptr(), scale.data_ptr(), st))
    return q if wide == K else q[..., :K], scale


def _int8_rows(t, K):
    """A [rows, K] view of t whose rows start at multiples of 16 bytes (a copy where it has none)."""
    if t.dim() != 2:
        t = t.reshape(-1, K)
    if (t.stride(1) == 1 or K == 1) and t.data_ptr() % 16 == 0 and (t.shape[0] < 2 or (t.stride(0) >= K and t.stride(0) % 16 == 0)):
        return t
    out = torch.empty((t.shape[0], (K + 15) // 16 * 16), dtype=torch.int8, device=t.device)[:, :K]
    return out.copy_(t)


def _int8_stride(t):
    return t.stride(0) if t.shape[0] > 1 else (t.shape[1] + 15) // 16 * 16


@functools.lru_cache(maxsize=256)
def _int8(M, K, N, dtype, x_stride, w_stride):
    _library()
    p = Int8Linear(M, K, N, dtype, 0, x_stride, w_stride, N)
    return p, C.byref(p)


def int8_linear(q, scale, weight, weight_scale, bias=None, *, dtype=torch.bfloat16):
    """(q weight^T) scale weight_scale + bias in ``dtype`` (bf16 or fp16).

    q [..., K] and weight [N, K] are int8 (as :func:`quantize_rows` gives them; rows that do not start at multiples
    of 16 bytes are copied), scale [...] and weight_scale [N] float32, bias [N] of ``dtype``. The product is summed in
    32-bit integers. No gradients."""
    if dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"int8 linear to {dtype} is not built")
    if q.dtype != torch.int8 or weight.dtype != torch.int8:
        raise ValueError("q and weight must be int8 tensors")
    if q.dim() < 1 or weight.dim() != 2 or weight.shape[1] != q.shape[-1] or min(weight.shape) < 1:
        raise ValueError("expected q [..., K] and weight [N, K]")
    K, N = q.shape[-1], weight.shape[0]
    if scale.dtype != torch.float32 or scale.shape != q.shape[:-1] or not scale.is_contiguous():
        raise ValueError(f"scale must be a contiguous float32 tensor of the shape {tuple(q.shape[:-1])}")
    if weight_scale.dtype != torch.float32 or weight_scale.shape != (N,) or not weight_scale.is_contiguous():
        raise ValueError(f"weight_scale must be a contiguous float32 tensor of {N} elements")
    if bias is not None and (bias.dtype != dtype or bias.shape != (N,) or not bias.is_contiguous()):
        raise ValueError(f"bias must be contiguous with {N} elements of {dtype}")
    _no_gradients("int8 linear", scale, weight_scale, bias)
    st = _on_device(q, scale, weight, weight_scale, bias)
    q2, w = _int8_rows(q, K), _int8_rows(weight, K)
    _, ref = _int8(q2.shape[0], K, N, _DTYPE[dtype], _int8_stride(q2), _int8_stride(w))
    y = q.new_empty((*q.shape[:-1], N), dtype=dtype)
    B._check(_LIB.paraanya_int8_linear(ref, q2.data_ptr(), scale.data_ptr(), w.data_ptr(), weight_scale.data_ptr(), _ptr(bias),
                                       y.data_ptr(), st))
    return y
