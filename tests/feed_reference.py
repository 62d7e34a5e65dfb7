"""The gated feed-forward block in 64 bits with bounds for what its kernels keep: h, rounded to the element type, the two factors
by which dh gives the projections' gradients, cut to 24 bits, and those gradients, rounded to the element type."""
import math

import torch

from block_ops_reference import CURVE, SLOPE, activation
from ops_reference import TINY, U, U32

# Roundings to the element type on the way to a result, its own among them: of h; of dz or du; of h. (The factors' 2^-15 is a
# sixteenth of fp16's rounding.)
ROUNDINGS = {"y": 2, "x": 2, "gate": 2, "up": 2, "down": 2, "gate_bias": 2, "up_bias": 2, "down_bias": 1}
CUT = 2.0 ** -15
# Of normal numbers and of products of two, a rounding's root mean square over theirs: half a step is 2^e u for a value of
# 2^e to 2^(e + 1), a third of its square the mean, and 0.4245 u the root of its sum over that of the values' squares.
ROUNDING = 0.4245


def feed_forward(x, gate, up, down, biases, act, dy):
    """{name: (value, bound)} of y and the gradients x, gate, up, down, gate_bias, up_bias, down_bias."""
    dt = x.dtype
    u, tiny = U[dt], TINY[dt]
    (M, K), (H, N) = x.shape, (gate.shape[0], down.shape[0])
    A = torch.Tensor.abs
    X, G, Up, D, Y = (t.double() for t in (x, gate, up, down, dy))
    bg, bu, bd = (torch.zeros(n, dtype=torch.float64, device=x.device) if t is None else t.double() for t, n in zip(biases, (H, H, N)))
    p, q = X @ G.T + bg, X @ Up.T + bu
    ep, eq = ((K + 8) * U32 * (A(X) @ A(t).T + A(b)) for t, b in ((G, bg), (Up, bu)))
    a, slope, ea, es = activation(act, p)
    if act == "gelu":
        es = es + 4e-6                       # the polynomial for results of 16 bits
    ea, es = SLOPE * ep + ea, CURVE * ep + es
    h = a * q
    eh = ea * (A(q) + eq) + A(a) * eq + (u + U32) * A(h) + tiny
    out = {}

    def put(name, v, e):
        out[name] = (v, 1.01 * e + u * A(v) + tiny)

    put("y", h @ D.T + bd, eh @ A(D).T + (H + 8) * U32 * (A(h) @ A(D).T + A(bd)))
    # The factors, cut; dz = dh f and du = dh a, rounded. In fp16 both times a power of two s with s max |dy| >= 1/16: half
    # of the least spacing over s is at most 16 max |dy| times it.
    f = q * slope
    ef = A(q) * es + eq * (A(slope) + es) + (CUT + U32) * A(f)
    ea = ea + CUT * A(a)
    small = 16 * tiny * (float(A(Y).max()) if dt == torch.float16 and Y.numel() else 1.0)
    dh, edh = Y @ D, (N + 8) * U32 * (A(Y) @ A(D))
    dz, du = dh * f, dh * a
    edz = edh * (A(f) + ef) + A(dh) * ef + (u + 3 * U32) * A(dz) + small
    edu = edh * (A(a) + ea) + A(dh) * ea + (u + 3 * U32) * A(du) + small
    put("x", dz @ G + du @ Up, edz @ A(G) + edu @ A(Up) + (2 * H + 8) * U32 * (A(dz) @ A(G) + A(du) @ A(Up)))
    m = (M + 16) * U32
    put("gate", dz.T @ X, edz.T @ A(X) + m * (A(dz).T @ A(X)))
    put("up", du.T @ X, edu.T @ A(X) + m * (A(du).T @ A(X)))
    put("down", Y.T @ h, A(Y).T @ eh + m * (A(Y).T @ A(h)))
    put("gate_bias", dz.sum(0), edz.sum(0) + m * A(dz).sum(0))
    put("up_bias", du.sum(0), edu.sum(0) + m * A(du).sum(0))
    put("down_bias", Y.sum(0), m * A(Y).sum(0))
    return out


def norm_limit(name, want, dt, kept):
    """What the root of the squared errors' sum may be: of independent roundings, with room for their number and for the spread
    of sums of their squares; a result below the type's normal numbers is off by half of their least spacing.

    `kept`: the number of values that h, dz or du has; each is rounded once, however many results it goes into (one
    row's go into an outer product), so that a result has no more independent errors than that. The squares summed are of
    products of up to three normal numbers, whose fourth moment is 27 times their second's square, times a rounding's square,
    whose own is 9/5: the sum's deviation is sqrt(27 * 9 / 5 / kept), the root's half of that, 3.5 / sqrt(kept), three times
    which leaves 10.5 / sqrt(kept)."""
    n = want.numel()
    room = 1.04 + 10.5 / math.sqrt(min(n, kept))
    return ROUNDING * math.sqrt(ROUNDINGS[name]) * room * U[dt] * float(want.norm()) + TINY[dt] * math.sqrt(n)
