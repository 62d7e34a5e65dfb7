"""Timed cases of the operators around attention in a conditioned noise network: group norm with an
activation over channels-last latents (forward and backward), a gated feed-forward block (forward and
backward) and a projection in 8-bit integers with scales for each token and channel.

``run`` computes a case in elementary torch operations in 32 bits, or, where ``own`` is true, with the
library's operators (``paper_2609_36522_amd.ops``). ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------ cases
def _gn(name, B, P, C, G, dtype, act, *, step):
    return _named(name, {"op": "group", "B": B, "P": P, "C": C, "G": G, "dtype": dtype, "act": act, "step": step})


def _ff(name, M, K, H, dtype, act, *, step, bias=True):
    return _named(name, {"op": "feed", "M": M, "K": K, "H": H, "dtype": dtype, "act": act, "step": step, "bias": bias})


def _i8(name, M, K, N, dtype, *, bias=True):
    return _named(name, {"op": "int8", "M": M, "K": K, "N": N, "dtype": dtype, "bias": bias})


def _named(name, case):
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # One 8 x 8 latent of 320 channels: launches and the host.
        _gn("group_small_1x64x320_bf16", 1, 64, 320, 32, "bf16", "silu", step=False),
        # Serving: a window of 32 latents of 64 x 64 pixels.
        _gn("group_window_32x4096x320_bf16", 32, 4096, 320, 32, "bf16", "silu", step=False),
        # Training on eight such latents with twice the channels.
        _gn("group_step_8x4096x640_bf16", 8, 4096, 640, 32, "bf16", "silu", step=True),
        # A 37 x 53 latent in 32 bits, groups of 30 channels.
        _gn("group_step_3x1961x330_f32", 3, 1961, 330, 11, "f32", "gelu", step=True),
        # One token: the weights are read, little is computed.
        _ff("feed_token_1x1024x4096_bf16", 1, 1024, 4096, "bf16", "silu", step=False, bias=False),
        # Serving eight latents of 1024 tokens at the network width 1024.
        _ff("feed_rows_8192x1024x4096_bf16", 8192, 1024, 4096, "bf16", "gelu", step=False),
        # Training on them.
        _ff("feed_step_8192x1024x4096_bf16", 8192, 1024, 4096, "bf16", "gelu", step=True),
        # A ragged batch, widths that divide nothing.
        _ff("feed_step_1999x1100x2731_f16", 1999, 1100, 2731, "f16", "silu", step=True),
        # A window of 32 latents through the widest network: the matrix cores' case.
        _ff("feed_window_32768x2048x8192_bf16", 32768, 2048, 8192, "bf16", "silu", step=False, bias=False),
        # One token each of eight requests.
        _i8("int8_token_8x1024x4096_bf16", 8, 1024, 4096, "bf16", bias=False),
        # Odd sizes everywhere.
        _i8("int8_odd_1999x1100x1347_f16", 1999, 1100, 1347, "f16"),
        # The window of 32 latents through one projection of the widest network.
        _i8("int8_window_32768x2048x8192_bf16", 32768, 2048, 8192, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["flops"] / 1e15, w["bytes"] / 4e12)


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("group", "feed", "int8")}
    kind = rng.choice(("group", "feed", "feed", "int8"))
    while True:
        dt = rng.choice(("bf16", "bf16", "f16"))
        if kind == "group":
            G = rng.choice((1, 8, 11, 16, 32))
            # Groups of few values have no gradient but rounding: 16 pixels at least.
            c = _gn(None, _log_int(rng, 1, 32), _log_int(rng, 16, 9216), G * _log_int(rng, 2, 60), G,
                    rng.choice((dt, dt, "f32")), rng.choice(("none", "silu", "silu", "gelu")), step=rng.random() < 0.5)
        elif kind == "feed":
            c = _ff(None, _log_int(rng, 1, 32768), _log_int(rng, 320, 2048), _log_int(rng, 320, 8192), dt,
                    rng.choice(("silu", "gelu")), step=rng.random() < 0.5, bias=rng.random() < 0.5)
        else:
            c = _i8(None, _log_int(rng, 1, 32768), _log_int(rng, 320, 2048), _log_int(rng, 320, 8192), dt, bias=rng.random() < 0.5)
        if _cost(c) <= most[kind]:
            return c


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _padded(q):
    """q with rows that start at multiples of 16 bytes, as a program keeps 8-bit weights."""
    N, K = q.shape
    out = torch.zeros((N, (K + 15) // 16 * 16), dtype=torch.int8, device=q.device)[:, :K]
    out.copy_(q)
    return out


def prepare(case, seed):
    """What a program holds before the call: activations, weights and gradients as they come in a network
    (channels of different size and offset; a few channels far larger than the others)."""
    g, dt = _generator(seed), DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "group":
        B, P, C = case["B"], case["P"], case["C"]
        s["x"] = (_randn(g, B, P, C) * (0.5 + torch.rand(C, generator=g, device="cuda")) + 0.5 * _randn(g, C) + 0.3 * _randn(g, B, 1, C)).to(dt)
        s["w"], s["b"] = (1 + 0.2 * _randn(g, C)).to(dt), (0.2 * _randn(g, C)).to(dt)
        s["dy"] = _randn(g, B, P, C).to(dt) if case["step"] else None
    elif case["op"] == "feed":
        M, K, H = case["M"], case["K"], case["H"]
        s["x"] = (_randn(g, M, K) * (0.5 + torch.rand(K, generator=g, device="cuda"))).to(dt)
        s["gate"], s["up"] = (_randn(g, H, K) / math.sqrt(K)).to(dt), (_randn(g, H, K) / math.sqrt(K)).to(dt)
        s["down"] = (_randn(g, K, H) / math.sqrt(H)).to(dt)
        s["biases"] = tuple((0.1 * _randn(g, n)).to(dt) if case["bias"] else None for n in (H, H, K))
        s["dy"] = _randn(g, M, K).to(dt) if case["step"] else None
    else:
        M, K, N = case["M"], case["K"], case["N"]
        size = torch.exp(0.7 * _randn(g, K))
        s["x"] = (_randn(g, M, K) * size).to(dt)
        w = _randn(g, N, K) / (math.sqrt(K) * size)
        s["ws"] = w.abs().amax(1) / 127
        s["wq"] = _padded(torch.round(w / s["ws"][:, None]).to(torch.int8))
        s["bias"] = (0.1 * _randn(g, N)).to(dt) if case["bias"] else None
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"group": _own_group, "feed": _own_feed, "int8": _own_int8}[op](s)
    return {"group": _plain_group, "feed": _plain_feed, "int8": _plain_int8}[op](s)


def _name(act):
    return None if act == "none" else act


def _own_group(s):
    from paper_2609_36522_amd import ops
    act = _name(s["case"]["act"])
    y, mean, rstd = ops.group_norm_forward(s["x"], s["case"]["G"], s["w"], s["b"], EPS, activation=act)
    if s["dy"] is None:
        return {"y": y}
    dx, dw, db = ops.group_norm_backward(s["dy"], s["x"], mean, rstd, s["w"], s["b"], activation=act)
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _own_feed(s):
    from paper_2609_36522_amd import ops
    act = s["case"]["act"]
    y, saved = ops.feed_forward_forward(s["x"], s["gate"], s["up"], s["down"], *s["biases"], activation=act, save=s["dy"] is not None)
    if s["dy"] is None:
        return {"y": y}
    g = ops.feed_forward_backward(s["dy"], s["x"], s["gate"], s["up"], s["down"], saved, activation=act)
    out = {"y": y, "dx": g.x, "dgate": g.gate, "dup": g.up, "ddown": g.down}
    if s["case"]["bias"]:
        out.update(dbgate=g.gate_bias, dbup=g.up_bias, dbdown=g.down_bias)
    return out


def _own_int8(s):
    from paper_2609_36522_amd import ops
    q, scale = ops.quantize_rows(s["x"])
    return {"y": ops.int8_linear(q, scale, s["wq"], s["ws"], s["bias"], dtype=s["x"].dtype), "q": q, "scale": scale}


def _activate(z, act):
    """(act(z), act'(z)) from the exponential and the error function."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    p = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * p, p + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def _plain_group(s):
    c, dt = s["case"], s["x"].dtype
    B, P, C, G = c["B"], c["P"], c["C"], c["G"]
    x, w, b = s["x"].float().reshape(B, P, G, C // G), s["w"].float().reshape(G, -1), s["b"].float().reshape(G, -1)
    d = x - x.mean((1, 3), keepdim=True)
    r = torch.rsqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    xh = d * r
    y, slope = _activate(xh * w + b, c["act"])
    out = {"y": y.reshape(B, P, C).to(dt)}
    if s["dy"] is None:
        return out
    dz = s["dy"].float().reshape(x.shape) * slope
    g = dz * w
    dx = r * (g - g.mean((1, 3), keepdim=True) - xh * (g * xh).mean((1, 3), keepdim=True))
    return {**out, "dx": dx.reshape(B, P, C).to(dt), "dw": (dz * xh).sum((0, 1)).reshape(C).to(dt), "db": dz.sum((0, 1)).reshape(C).to(dt)}


def _plain_feed(s):
    dt = s["x"].dtype
    x, wg, wu, wd = (s[n].float() for n in ("x", "gate", "up", "down"))
    bg, bu, bd = (0.0 if t is None else t.float() for t in s["biases"])
    act, slope = _activate(torch.matmul(x, wg.t()) + bg, s["case"]["act"])
    u = torch.matmul(x, wu.t()) + bu
    h = act * u
    out = {"y": (torch.matmul(h, wd.t()) + bd).to(dt)}
    if s["dy"] is None:
        return out
    dy = s["dy"].float()
    dh = torch.matmul(dy, wd)
    dg, du = dh * u * slope, dh * act
    out["dx"] = (torch.matmul(dg, wg) + torch.matmul(du, wu)).to(dt)
    out["dgate"], out["dup"] = torch.matmul(dg.t(), x).to(dt), torch.matmul(du.t(), x).to(dt)
    out["ddown"] = torch.matmul(dy.t(), h).to(dt)
    if s["case"]["bias"]:
        out["dbgate"], out["dbup"], out["dbdown"] = dg.sum(0).to(dt), du.sum(0).to(dt), dy.sum(0).to(dt)
    return out


def _plain_int8(s):
    x = s["x"].float()
    largest = x.abs().amax(1)
    scale = largest / torch.full_like(largest, 127)        # a quotient: by a number, torch multiplies by its reciprocal
    q = torch.round(x / torch.where(scale == 0, 1.0, scale)[:, None]).clamp(-127, 127)
    y = torch.matmul(q, s["wq"].float().t()) * scale[:, None] * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return {"y": y.to(s["x"].dtype), "q": q.to(torch.int8), "scale": scale}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    z = SIZE[case["dtype"]]
    if case["op"] == "group":
        n, C, step = case["B"] * case["P"] * case["C"], case["C"], case["step"]
        # x in and y out; with the gradients also dy in and dx out, and the parameters'.
        return {"bytes": z * (n + C) * (4 if step else 2), "flops": n * (40 if step else 15)}
    if case["op"] == "feed":
        M, K, H, step = case["M"], case["K"], case["H"], case["step"]
        weights = 3 * K * H + ((2 * H + K) if case["bias"] else 0)
        return {"bytes": z * (M * K * (4 if step else 2) + weights * (2 if step else 1)), "flops": (18 if step else 6) * M * K * H}
    M, K, N = case["M"], case["K"], case["N"]
    # 16-bit activations in, their 8-bit form and scales out; 8-bit weights in, 16-bit results out.
    return {"bytes": (z + 1) * M * K + 4 * M + N * K + 4 * N + z * M * N + (z * N if case["bias"] else 0), "flops": 2 * M * N * K}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"group": _exact_group, "feed": _exact_feed, "int8": _exact_int8}[case["op"]](s)


def _slope(act, z):
    """The activation's value and derivative, each from its closed form."""
    if act == "none":
        return z, torch.full_like(z, 1.0)
    if act == "silu":
        t = torch.sigmoid(z)
        return z * t, t + z * t * torch.sigmoid(-z)
    half = torch.special.erfc(-z / math.sqrt(2)) / 2
    return z * half, half + z * torch.exp(-z.square() / 2 - math.log(2 * math.pi) / 2)


def _exact_group(s):
    c = s["case"]
    B, P, C, G = c["B"], c["P"], c["C"], c["G"]
    out = {"y": torch.empty(B, P, C, dtype=torch.float64, device="cuda")}
    if s["dy"] is not None:
        out["dx"] = torch.empty_like(out["y"])
        out["dw"], out["db"] = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in "wb")
    for b in range(B):
        # One sample, a group's values in a row: [G, P L].
        rows = s["x"][b].double().reshape(P, G, C // G).transpose(0, 1).reshape(G, -1)
        sd = torch.sqrt(rows.var(1, correction=0) + EPS)
        xh = ((rows - rows.mean(1)[:, None]) / sd[:, None]).reshape(G, P, -1).transpose(0, 1).reshape(P, C)
        w = s["w"].double()
        y, slope = _slope(c["act"], torch.addcmul(s["b"].double(), xh, w))
        out["y"][b] = y
        if s["dy"] is None:
            continue
        dz = s["dy"][b].double() * slope
        out["dw"] += torch.linalg.vecdot(dz, xh, dim=0)
        out["db"] += dz.sum(0)

        def of_group(t):        # the mean over a pixel's group, for each channel
            return (t.sum(0).reshape(G, -1).sum(1) / (P * (C // G))).repeat_interleave(C // G)

        out["dx"][b] = (dz * w - of_group(dz * w) - xh * of_group(dz * w * xh)) / sd.repeat_interleave(C // G)
    return out


def _exact_feed(s):
    """Rows in pieces: what a row gives of y and dx is its own, what it adds to a weight's gradient is summed."""
    x64, wg, wu, wd = (s[n].double() for n in ("x", "gate", "up", "down"))
    bg, bu, bd = (None if t is None else t.double() for t in s["biases"])
    step, bias = s["dy"] is not None, s["case"]["bias"]
    out = {"y": torch.empty_like(x64)}
    if step:
        out.update(dx=torch.empty_like(x64), dgate=torch.zeros_like(wg), dup=torch.zeros_like(wu), ddown=torch.zeros_like(wd))
        if bias:
            out.update(dbgate=torch.zeros_like(bg), dbup=torch.zeros_like(bu), dbdown=torch.zeros_like(bd))
    for at in range(0, x64.shape[0], 4096):
        r = slice(at, at + 4096)
        x = x64[r]
        a, slope = _slope(s["case"]["act"], torch.nn.functional.linear(x, wg, bg))
        u = torch.nn.functional.linear(x, wu, bu)
        out["y"][r] = torch.nn.functional.linear(a * u, wd, bd)
        if not step:
            continue
        dy = s["dy"][r].double()
        dh = dy @ wd
        dz, du = dh * slope * u, dh * a
        out["dx"][r] = dz @ wg + du @ wu
        out["dgate"] += dz.T @ x
        out["dup"] += du.T @ x
        out["ddown"] += dy.T @ (a * u)
        if bias:
            out["dbgate"] += dz.sum(0)
            out["dbup"] += du.sum(0)
            out["dbdown"] += dy.sum(0)
    return out


def _exact_int8(s):
    """The integers' product is a whole number; q itself is compared as such."""
    x = s["x"].double()
    scale = x.abs().amax(1) / 127
    q = torch.round(x / scale.clamp(min=1e-300)[:, None]).clamp(-127, 127)
    y = (q @ s["wq"].double().T) * torch.outer(scale, s["ws"].double())
    return {"y": y if s["bias"] is None else y + s["bias"].double(), "q": None, "scale": scale}
