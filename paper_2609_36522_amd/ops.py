"""Operators of a text-conditioned noise network (the C ABI in include/paraanya_ops.h): layer norm,
cross attention to a prompt encoder's states, a shared projection with the low-rank adapters of many
requests.

Argument marshalling only, as in :mod:`binding`: every product and sum runs in the library's HIP
kernels. Tensors lie on the current device; kernels run on torch's current stream, outputs and
workspaces come from torch's allocator on that stream. :func:`layer_norm` and
:func:`cross_attention` take part in autograd, for first derivatives (a gradient's gradient is refused); the
``*_forward`` and ``*_backward`` functions do not.
"""
from __future__ import annotations

import ctypes as C
import functools
import math

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

PA_F32, PA_BF16, PA_F16 = 0, 1, 2
PA_MASK_NONE, PA_MASK_BOOL, PA_MASK_ADD = 0, 1, 2
PA_NORM_MAX_COLS = 1 << 20
PA_LORA_MAX_RANK = 128
HEAD_DIM_MAX = 128

EXPORTED = ("paraanya_layer_norm", "paraanya_layer_norm_backward", "paraanya_layer_norm_backward_workspace",
            "paraanya_cross_attention", "paraanya_cross_attention_workspace",
            "paraanya_cross_attention_backward", "paraanya_cross_attention_backward_workspace",
            "paraanya_lora_linear", "paraanya_lora_linear_workspace")

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
        for name in EXPORTED:
            f = getattr(lib, name)
            f.restype = C.c_int
            if name.endswith("_workspace"):
                f.argtypes = [P, C.POINTER(Z)]
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
    return torch.empty(n, dtype=torch.uint8, device=like.device) if n else None


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ layer norm
def _rows(t, N):
    """A [rows, N] view of t (a copy where its strides allow no view)."""
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
