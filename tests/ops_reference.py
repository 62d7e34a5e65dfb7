"""The operators of include/paraanya_ops.h in 64 bits, with bounds on how far 16- and 32-bit kernels may
be from them. Bounds are sums of rounding errors: u is the unit roundoff of the element type, every
product of a matrix core is exact and added in fp32, and P, dS and t are rounded to the element type."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# Half of the spacing of the type's subnormal numbers: the least rounding error of a small value.
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U32 = 2.0 ** -24
# A weight below fp32's least normal number comes out of the exponential unit as 0.
FLUSH = 2.0 ** -126


def layer_norm(x, w, b, eps, dy=None):
    """{name: (value, bound)} of y (and dx, dw, db); x [M, N], w and b [N] or None."""
    dt, pt = x.dtype, x.dtype if w is None else w.dtype
    M, N = x.shape
    x64 = x.double()
    w64 = torch.ones(N, dtype=torch.float64, device=x.device) if w is None else w.double()
    b64 = torch.zeros_like(w64) if b is None else b.double()
    mu = x64.mean(1, keepdim=True)
    r = 1 / torch.sqrt((x64 - mu).square().mean(1, keepdim=True) + eps)
    xh = (x64 - mu) * r
    # Sums run over at most 32 terms of a lane and 8 levels across lanes (three passes for long rows:
    # N / 256 terms): relative error of a sum of magnitudes, doubled for the squares.
    g = (32 + N / 256 + 16) * U32
    dxh = g * (x64.abs().mean(1, keepdim=True) * r + xh.abs() * 2) + 4 * U32 * (x64.abs() * r + xh.abs())
    y = xh * w64 + b64
    out = {"y": (y, U[dt] * y.abs() + dxh * w64.abs() + 4 * U32 * ((xh * w64).abs() + b64.abs()) + TINY[dt])}
    if dy is not None:
        dy64 = dy.double()
        gr = dy64 * w64
        m1, m2 = gr.mean(1, keepdim=True), (gr * xh).mean(1, keepdim=True)
        dx = r * (gr - m1 - xh * m2)
        mag = gr.abs() + gr.abs().mean(1, keepdim=True) + xh.abs() * (gr * xh).abs().mean(1, keepdim=True)
        e = r * (mag * (g + 8 * U32) + dxh * (m2.abs() + (gr.abs() * xh.abs()).mean(1, keepdim=True))
                 + xh.abs() * (gr.abs() * dxh).mean(1, keepdim=True))
        out["dx"] = (dx, U[dt] * dx.abs() + e + TINY[dt])
        # A column's sum: M terms in at most 512 partial sums and two levels.
        c = (M / 128 + 600) * U32
        dw, db = (dy64 * xh).sum(0), dy64.sum(0)
        out["dw"] = (dw, U[pt] * dw.abs() + c * (dy64 * xh).abs().sum(0) + (dy64.abs() * dxh).sum(0) + TINY[pt])
        out["db"] = (db, U[pt] * db.abs() + c * dy64.abs().sum(0) + TINY[pt])
    return out


def key_bias(B, Lk, device, kv_lens=None, mask=None):
    """Additive bias [B, Lk] in 64 bits, -inf where a key is not visible."""
    bias = torch.zeros(B, Lk, dtype=torch.float64, device=device)
    if kv_lens is not None:
        n = kv_lens.clamp(0, Lk)
        bias.masked_fill_(torch.arange(Lk, device=device)[None] >= n[:, None], -math.inf)
    if mask is not None:
        bias = bias + mask.double() if mask.dtype == torch.float32 else bias.masked_fill(mask == 0, -math.inf)
    return bias


def cross_attention(q, k, v, do=None, *, kv_lens=None, mask=None, scale=None):
    """{name: (value, bound)} of o, lse (and dq, dk, dv). Invisible keys take part nowhere."""
    dt = q.dtype
    u, tiny = U[dt], TINY[dt]
    B, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1:3]
    G = Hq // Hk
    scale = 1 / math.sqrt(D) if scale is None else scale
    bias = key_bias(B, Lk, q.device, kv_lens, mask)
    z = dict(dtype=torch.float64, device=q.device)
    out = {n: (torch.zeros(s, **z), torch.zeros(s, **z)) for n, s in
           (("o", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    out["lse"] = (torch.full((B, Hq, Lq), -math.inf, **z), torch.zeros((B, Hq, Lq), **z))
    for b in range(B):
        seen = torch.nonzero(bias[b] > -math.inf)[:, 0]
        if seen.numel() == 0 or Lq == 0:
            continue
        add = bias[b, seen]
        for h in range(Hq):
            Q, K, V = q[b, :, h].double(), k[b, seen, h // G].double(), v[b, seen, h // G].double()
            S = scale * (Q @ K.T) + add
            P = torch.softmax(S, 1)
            o = P @ V
            # Scores: D products in fp32, the scaling and the bias; their error moves a weight by as much,
            # and so do the exponential's and the running sum's (2^-14 takes both with room).
            top = S.max(1, keepdim=True).values
            es = 2 * abs(scale) * D * U32 * (Q.abs() @ K.T.abs()).max(1, keepdim=True).values
            es = es + 4 * U32 * (S - top).abs().clamp(max=200).max(1, keepdim=True).values + 2.0 ** -14 * (u > 2.0 ** -12) \
                + 2.0 ** -16
            eo = (u + es) * (P @ V.abs()) + (tiny + FLUSH) * V.abs().sum(0)
            out["o"][0][b, :, h], out["o"][1][b, :, h] = o, eo + u * o.abs() + tiny
            out["lse"][0][b, h] = torch.logsumexp(S, 1)
            out["lse"][1][b, h] = (es[:, 0] + 4 * U32 * (torch.logsumexp(S, 1).abs() + top[:, 0].abs()))
            if do is None:
                continue
            dO = do[b, :, h].double()
            dP = dO @ V.T
            d = (P * dP).sum(1, keepdim=True)
            dS = P * (dP - d)
            # The row's sum d comes from the rounded o or from rounded products.
            ed = (dO.abs() * (eo + u * o.abs() + tiny)).sum(1, keepdim=True) + D * U32 * (dO.abs() @ V.T.abs()).max(1, keepdim=True).values
            eS = P * (ed + (2 * es) * (dP.abs() + d.abs()) + D * U32 * (dO.abs() @ V.T.abs())) + u * dS.abs() + tiny \
                + FLUSH * (dP.abs() + d.abs())
            eP = (u + 2 * es) * P + tiny + FLUSH
            a = abs(scale)
            dq = scale * (dS @ K)
            out["dq"][0][b, :, h], out["dq"][1][b, :, h] = dq, a * (eS @ K.abs()) * 1.01 + u * dq.abs() + tiny
            out["dk"][0][b, seen, h // G] += scale * (dS.T @ Q)
            out["dk"][1][b, seen, h // G] += a * (eS.T @ Q.abs()) * 1.01 + a * Lq * U32 * (dS.abs().T @ Q.abs())
            out["dv"][0][b, seen, h // G] += P.T @ dO
            out["dv"][1][b, seen, h // G] += (eP.T @ dO.abs()) * 1.01 + Lq * U32 * (P.T @ dO.abs())
    for n in ("dk", "dv"):
        out[n] = (out[n][0], out[n][1] + u * out[n][0].abs() + tiny)
    return out


def lora_linear(x, w, a, b, offsets, ids, scales=None, bias=None):
    """(y, bound); offsets and ids are lists."""
    dt = x.dtype
    u, tiny = U[dt], TINY[dt]
    K, E, R = x.shape[1], a.shape[0], a.shape[1]
    X, W = x.double(), w.double()
    y = X @ W.T
    e = (K + 8) * U32 * (X.abs() @ W.T.abs())
    if bias is not None:
        y = y + bias.double()
    for i, ad in enumerate(ids):
        lo, hi = (min(max(o, 0), x.shape[0]) for o in offsets[i:i + 2])
        if not 0 <= ad < E or hi <= lo:
            continue
        s = 1.0 if scales is None else float(scales[ad])
        A, Bm, Xi = a[ad].double(), b[ad].double(), X[lo:hi]
        t = s * (Xi @ A.T)
        et = u * t.abs() + (K + 8) * U32 * abs(s) * (Xi.abs() @ A.T.abs()) + tiny
        y[lo:hi] += t @ Bm.T
        e[lo:hi] += et @ Bm.T.abs() + (R + K) * U32 * (t.abs() @ Bm.T.abs())
    return y, e + u * y.abs() + tiny


def check(got, want, bound, what):
    assert got.shape == want.shape, what
    err = (got.double() - want).abs()
    same = (got.double() == want) | (torch.isnan(got.double()) & torch.isnan(want))
    bad = ~same & ~(err <= bound)
    if bool(bad.any()):
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; at {i} got {got[i].item()!r}, "
                             f"want {want[i].item()!r}, bound {bound[i].item():.3g}")
