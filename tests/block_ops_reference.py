"""Group norm, the gated feed-forward block and the 8-bit projection of include/paraanya_ops.h in 64 bits, with
bounds on how far the kernels may be from them: sums of rounding errors, as in ops_reference.py."""
import math

import torch

from ops_reference import TINY, U, U32

# Largest slopes of the activations and of their derivatives (silu 1.0999 and 0.5, gelu 1.1290 and 0.7979).
SLOPE, CURVE = 1.13, 0.8


def activation(name, z):
    """(value, derivative, bound of the value's evaluation in fp32, of the derivative's)."""
    if name is None:
        return z, torch.ones_like(z), torch.zeros_like(z), torch.zeros_like(z)
    if name == "silu":
        # The exponential's argument is rounded once (|z| 2^-24 of the result), then the exponential, the sum, the
        # reciprocal and the product, each by one or two units; 1 - p of a p near 1 is off by U32, times |z|.
        p = torch.sigmoid(z)
        v, d = z * p, p + z * p * torch.sigmoid(-z)
    else:
        # The polynomial's error is within 2e-7 max(1, |z|) (3.4 units), the density's argument z^2 / 2 is rounded
        # three times: z^2 phi |z| 3 units, at most 2.
        p = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        v, d = z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return v, d, (8 + 2 * z.abs()) * U32 * v.abs() + 4 * U32 * z.abs().clamp(min=1), (8 + 2 * z.abs()) * U32


def group_norm(x, groups, w, b, eps, act=None, dy=None):
    """{name: (value, bound)} of y (and dx, dw, db); x [batch, pixels, channels]."""
    dt, pt = x.dtype, next((t.dtype for t in (w, b) if t is not None), x.dtype)
    B, P, C = x.shape
    L = C // groups

    def split(t):
        return t.double().reshape(-1, P if t.dim() == 3 else 1, groups, L)

    def mean(t):
        return t.mean((1, 3), keepdim=True)

    x64 = split(x)
    w64 = torch.ones(1, 1, groups, L, dtype=torch.float64, device=x.device) if w is None else split(w.reshape(1, -1))
    b64 = torch.zeros_like(w64) if b is None else split(b.reshape(1, -1))
    mu = mean(x64)
    r = 1 / torch.sqrt(mean((x64 - mu).square()) + eps)
    xh = (x64 - mu) * r
    # A sum's longest chain: 16 pixels of a thread, up to 512 lanes of a channel, 64 channels of a lane, 6 levels,
    # 4 chunks of a lane and 6 levels. Its relative error is one of magnitudes, doubled for the squares.
    g = (16 + 512 + 64 + 16) * U32
    dxh = g * (mean(x64.abs()) * r + xh.abs() * 2) + 6 * U32 * (x64.abs() * r + xh.abs())
    z = xh * w64 + b64
    ez = dxh * w64.abs() + 4 * U32 * ((xh * w64).abs() + b64.abs())
    y, slope, ev, es = activation(act, z)
    out = {"y": (y, U[dt] * y.abs() + SLOPE * ez + ev + TINY[dt])}
    if dy is not None:
        dy64 = split(dy)
        dz = dy64 * slope
        edz = dy64.abs() * (CURVE * ez + es) * (act is not None) + U32 * dz.abs()
        gr, eg = dz * w64, edz * w64.abs()
        m1, m2 = mean(gr), mean(gr * xh)
        dx = r * (gr - m1 - xh * m2)
        mag = gr.abs() + mean(gr.abs()) + xh.abs() * mean((gr * xh).abs())
        # Sums over pixels of a channel: 8 of a thread (more in long samples: P / 256 chunks), 512 lanes, 256 chunks,
        # then over the group's channels.
        c = (8 + P / 256 + 512 + 256 + 64 + 16) * U32
        e = r * (mag * (c + g + 8 * U32) + dxh * (m2.abs() + mean((gr * xh).abs())) + xh.abs() * mean(gr.abs() * dxh)
                 + eg + mean(eg) + xh.abs() * mean(eg * xh.abs()))
        out["dx"] = (dx, U[dt] * dx.abs() + e + TINY[dt])
        s = c + B * U32
        dw, db = (dz * xh).sum((0, 1)), dz.sum((0, 1))
        out["dw"] = (dw, U[pt] * dw.abs() + s * (dz * xh).abs().sum((0, 1)) + (dz.abs() * dxh + edz * xh.abs()).sum((0, 1)) + TINY[pt])
        out["db"] = (db, U[pt] * db.abs() + s * dz.abs().sum((0, 1)) + edz.sum((0, 1)) + TINY[pt])
    return {n: (v.reshape((B, P, C) if n in ("y", "dx") else (C,)), e.expand_as(v).reshape((B, P, C) if n in ("y", "dx") else (C,)))
            for n, (v, e) in out.items()}


def feed_forward(x, gate, up, down, biases=(None, None, None), act="silu", dy=None):
    """{name: (value, bound)} of y (and x, gate, up, down, gate_bias, up_bias, down_bias: the gradients)."""
    dt = x.dtype
    u, tiny = U[dt], TINY[dt]
    (M, K), (H, N) = x.shape, (gate.shape[0], down.shape[0])
    X, G, Up, D = (t.double() for t in (x, gate, up, down))
    bg, bu, bd = (torch.zeros(n, dtype=torch.float64, device=x.device) if t is None else t.double() for t, n in zip(biases, (H, H, N)))
    p, q = X @ G.T + bg, X @ Up.T + bu
    ep, eq = ((K + 8) * U32 * (X.abs() @ t.abs().T + b.abs()) for t, b in ((G, bg), (Up, bu)))
    a, slope, ea, es = activation(act, p)
    h = a * q
    eh = (SLOPE * ep + ea) * (q.abs() + eq) + a.abs() * eq + (u + U32) * h.abs() + tiny
    y = h @ D.T + bd
    out = {"y": (y, eh @ D.abs().T + (H + 8) * U32 * (h.abs() @ D.abs().T + bd.abs()) + u * y.abs() + tiny)}
    if dy is None:
        return out
    Y = dy.double()
    ep, eq = ep + u * p.abs() + tiny, eq + u * q.abs() + tiny
    dh, edh = Y @ D, (N + 8) * U32 * (Y.abs() @ D.abs())
    dz, du = dh * q * slope, dh * a
    # In fp16 they are stored times a power of two s with s max |dy| >= 1/16: half of the least spacing over s is at most
    # 16 max |dy| times it.
    small = 16 * tiny * (float(Y.abs().max()) if dt == torch.float16 and Y.numel() else 1.0)
    edz = edh * ((q.abs() + eq) * (slope.abs() + CURVE * ep + es)) + dh.abs() * (eq * slope.abs() + (q.abs() + eq) * (CURVE * ep + es)) \
        + (u + 3 * U32) * dz.abs() + small
    edu = edh * (a.abs() + SLOPE * ep + ea) + dh.abs() * (SLOPE * ep + ea) + (u + 2 * U32) * du.abs() + small
    A = torch.Tensor.abs

    def put(name, v, e):
        out[name] = (v, 1.01 * e + u * v.abs() + tiny)

    put("x", dz @ G + du @ Up, edz @ A(G) + edu @ A(Up) + (2 * H + 8) * U32 * (A(dz) @ A(G) + A(du) @ A(Up)))
    m = (M + 16) * U32
    put("gate", dz.T @ X, edz.T @ A(X) + m * (A(dz).T @ A(X)))
    put("up", du.T @ X, edu.T @ A(X) + m * (A(du).T @ A(X)))
    put("down", Y.T @ h, A(Y).T @ eh + m * (A(Y).T @ A(h)))
    put("gate_bias", dz.sum(0), edz.sum(0) + m * A(dz).sum(0))
    put("up_bias", du.sum(0), edu.sum(0) + m * A(du).sum(0))
    put("down_bias", Y.sum(0), m * A(Y).sum(0))
    return out


def quantize_rows(x):
    """(q, scale) by fp32's own division and rounding, row by row: both are to be met exactly."""
    f = x.float()
    top = f.abs().amax(-1)
    # (By a plain number torch multiplies by its reciprocal.)
    scale = torch.where(torch.isfinite(top), top / torch.full_like(top, 127), math.nan)
    good = scale > 0
    q = torch.round(torch.where(good[..., None], f, 0.0) / torch.where(good, scale, 1.0)[..., None]).clamp(-127, 127)
    return q.to(torch.int8), scale


def int8_linear(q, scale, w, ws, bias, dt):
    """(y, bound): the whole number is rounded to fp32 once, multiplied twice, and the bias added."""
    v = (q.double() @ w.double().T) * scale.double()[:, None] * ws.double()
    y = v if bias is None else v + bias.double()
    return y, U[dt] * y.abs() + 4 * U32 * (v.abs() + y.abs()) + TINY[dt]
