"""Timed cases of the operators of a text-conditioned noise network: layer norm (forward and
backward), cross attention to a prompt encoder's states (forward and backward) and a shared
projection with the low-rank adapters of many requests.

``run`` computes a case in elementary torch operations in 32 bits, or, where ``own`` is true,
with the library's operators (``paper_2609_36522_amd.ops``). ``exact`` is the definition in
64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
KEEP = 0.875                    # share of the keys that a drawn key mask leaves visible


# ------------------------------------------------------------------ cases
def _ln(name, M, N, dtype, *, step):
    return _named(name, {"op": "norm", "M": M, "N": N, "dtype": dtype, "step": step})


def _ca(name, B, Lq, Hq, Hk, Lk, D, dtype, *, step, mask="none"):
    return _named(name, {"op": "cross", "B": B, "Lq": Lq, "Hq": Hq, "Hk": Hk, "Lk": Lk, "D": D, "dtype": dtype,
                         "step": step, "mask": mask})


def _lora(name, M, K, N, R, adapters, requests, dtype):
    return _named(name, {"op": "lora", "M": M, "K": K, "N": N, "R": R, "adapters": adapters, "requests": requests,
                         "dtype": dtype})


def _named(name, case):
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # One token's norm at the network width 1024: launches and the host.
        _ln("norm_token_1x1024_bf16", 1, 1024, "bf16", step=False),
        # Training on a window of 32 latents of 1024 tokens (a 4x64x64 latent in 2x2 patches).
        _ln("norm_step_32768x1024_bf16", 32768, 1024, "bf16", step=True),
        # A ragged batch in 32 bits, a width that divides nothing.
        _ln("norm_step_5003x1333_f32", 5003, 1333, "f32", step=True),
        # One new token of four requests over long encoder states, shared key/value heads.
        _ca("cross_token_B4_Lk16381_D128_f16", 4, 1, 32, 8, 16381, 128, "f16", step=False),
        # Serving: a window of 32 latents over prompts of 1 to 77 tokens.
        _ca("cross_text_B32_1024x77_D64_bf16", 32, 1024, 16, 16, 77, 64, "bf16", step=False, mask="lens"),
        # A 4x96x96 latent (2304 tokens) over long encoder states: the matrix cores' case.
        _ca("cross_long_B2_2304x4096_D128_bf16", 2, 2304, 16, 16, 4096, 128, "bf16", step=False),
        # Training on eight latents over padded prompts, the padding given as truth values.
        _ca("cross_step_B8_1024x77_D64_bf16", 8, 1024, 16, 16, 77, 64, "bf16", step=True, mask="bool"),
        # Training over longer states of odd sizes, a head width of 80, shared heads, and an
        # additive mask that holds the type's lowest value, infinities and an empty row.
        _ca("cross_step_B2_2309x1541_D80_f16", 2, 2309, 16, 4, 1541, 80, "f16", step=True, mask="add"),
        # One token each of eight requests with adapters of their own.
        _lora("lora_token_8x1024x1024_R16_bf16", 8, 1024, 1024, 16, 8, 8, "bf16"),
        # A batch of eight latents of 1024 tokens in all lengths, some without an adapter.
        _lora("lora_rows_8192x1024x1024_R16_bf16", 8192, 1024, 1024, 16, 8, 11, "bf16"),
        # Odd sizes everywhere.
        _lora("lora_odd_1999x1100x1347_R24_f16", 1999, 1100, 1347, 24, 5, 13, "f16"),
        # A window of 32 latents through the widest network.
        _lora("lora_window_32768x2048x2048_R64_bf16", 32768, 2048, 2048, 64, 8, 32, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["flops"] / 1e15, w["bytes"] / 6e12)


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("norm", "cross", "lora")}
    kind = rng.choice(("norm", "cross", "cross", "lora"))
    while True:
        if kind == "norm":
            c = _ln(None, _log_int(rng, 1, 32768), _log_int(rng, 64, 4096), rng.choice(("bf16", "bf16", "f16", "f32")),
                    step=rng.random() < 0.6)
        elif kind == "cross":
            Hk, G = rng.choice((4, 8, 16)), rng.choice((1, 1, 2, 4))
            # A softmax over one key has no gradient but rounding: steps have more keys.
            step = rng.random() < 0.5
            c = _ca(None, _log_int(rng, 1, 32), rng.choice((1, _log_int(rng, 2, 2309), _log_int(rng, 64, 2309))), Hk * G, Hk,
                    _log_int(rng, 16 if step else 1, 16384), rng.choice((32, 40, 64, 72, 80, 96, 128)),
                    rng.choice(("bf16", "bf16", "f16")), step=step, mask=rng.choice(("none", "lens", "bool", "add")))
            # The plain form holds the scores of all heads in 32 bits.
            if c["B"] * c["Hq"] * c["Lq"] * c["Lk"] > 4e8:
                continue
        else:
            c = _lora(None, _log_int(rng, 1, 32768), _log_int(rng, 320, 2048), _log_int(rng, 320, 2048),
                      rng.choice((4, 8, 16, 24, 32, 64)), rng.randint(1, 16), rng.randint(1, 48), rng.choice(("bf16", "bf16", "f16")))
        if _cost(c) <= most[kind]:
            return c


def _lens(case):
    """Lengths of the samples' encoder states, 1 to Lk, spread over the batch."""
    B, Lk = case["B"], case["Lk"]
    return [1 + (Lk - 1) * ((i * 7 + 3) % B + 1) // B for i in range(B)]


def _requests(case):
    """(row offsets of the requests, adapter of each or -1): uneven, one empty, some without adapter."""
    M, n, E = case["M"], case["requests"], case["adapters"]
    if M == n:
        return list(range(M + 1)), [i % E for i in range(n)]
    parts = [1 + (i * 5) % 7 for i in range(n)]
    if n > 2:
        parts[n // 2] = 0
    total, off, at = sum(parts), [0], 0
    for p in parts:
        at += p
        off.append(M * at // total)
    return off, [-1 if i % 6 == 4 else (i * 3) % E for i in range(n)]


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def prepare(case, seed):
    """What a program holds before the call: activations, weights and gradients as they come in a
    network (channels of different size and offset, scores of a few units, a few padded keys)."""
    g, dt = _generator(seed), DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "norm":
        M, N = case["M"], case["N"]
        s["x"] = (_randn(g, M, N) * (0.5 + torch.rand(N, generator=g, device="cuda")) + 0.3 * _randn(g, N) + 0.2).to(dt)
        s["w"], s["b"] = (1 + 0.2 * _randn(g, N)).to(dt), (0.1 * _randn(g, N)).to(dt)
        s["dy"] = _randn(g, M, N).to(dt) if case["step"] else None
    elif case["op"] == "cross":
        B, Lq, Hq, Hk, Lk, D = (case[k] for k in ("B", "Lq", "Hq", "Hk", "Lk", "D"))
        s["q"] = (1.5 * _randn(g, B, Lq, Hq, D)).to(dt)
        s["k"], s["v"] = _randn(g, B, Lk, Hk, D).to(dt), _randn(g, B, Lk, Hk, D).to(dt)
        s["do"] = _randn(g, B, Lq, Hq, D).to(dt) if case["step"] else None
        s["lens"] = s["mask"] = None
        if case["mask"] == "lens":
            s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
        elif case["mask"] == "bool":
            s["mask"] = torch.rand((B, Lk), generator=g, device="cuda") < KEEP
            s["mask"][:, 0] = True
        elif case["mask"] == "add":
            r = torch.rand((B, Lk), generator=g, device="cuda")
            m = 0.5 * _randn(g, B, Lk)
            m = torch.where(r < (1 - KEEP) / 2, torch.full_like(m, torch.finfo(torch.float32).min), m)
            s["mask"] = torch.where(r > 1 - (1 - KEEP) / 2, torch.full_like(m, -math.inf), m)
            if B > 1:
                s["mask"][B - 1] = -math.inf
    else:
        M, K, N, R, E = (case[k] for k in ("M", "K", "N", "R", "adapters"))
        off, ids = _requests(case)
        s["x"] = _randn(g, M, K).to(dt)
        s["w"], s["bias"] = (_randn(g, N, K) / math.sqrt(K)).to(dt), (0.1 * _randn(g, N)).to(dt)
        s["a"], s["b"] = (_randn(g, E, R, K) / math.sqrt(K)).to(dt), (0.3 * _randn(g, E, N, R) / math.sqrt(R)).to(dt)
        s["scales"] = 0.5 + torch.rand(E, generator=g, device="cuda")
        s["offsets"] = torch.tensor(off, dtype=torch.int32, device="cuda")
        s["ids"] = torch.tensor(ids, dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _own_norm, "cross": _own_cross, "lora": _own_lora}[op](s)
    return {"norm": _plain_norm, "cross": _plain_cross, "lora": _plain_lora}[op](s)


def _own_norm(s):
    from paper_2609_36522_amd import ops
    y, mean, rstd = ops.layer_norm_forward(s["x"], s["w"], s["b"], EPS)
    if s["dy"] is None:
        return {"y": y}
    dx, dw, db = ops.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["w"])
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _own_cross(s):
    from paper_2609_36522_amd import ops
    o, lse = ops.cross_attention_forward(s["q"], s["k"], s["v"], kv_lens=s["lens"], mask=s["mask"])
    if s["do"] is None:
        return {"o": o}
    dq, dk, dv = ops.cross_attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, kv_lens=s["lens"], mask=s["mask"])
    return {"o": o, "dq": dq, "dk": dk, "dv": dv}


def _own_lora(s):
    from paper_2609_36522_amd import ops
    return {"y": ops.lora_linear(s["x"], s["w"], s["a"], s["b"], s["offsets"], s["ids"], scales=s["scales"], bias=s["bias"])}


def _plain_norm(s):
    dt = s["x"].dtype
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    d = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    xh = d * r
    y = (xh * w + b).to(dt)
    if s["dy"] is None:
        return {"y": y}
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return {"y": y, "dx": dx.to(dt), "dw": (dy * xh).sum(0).to(dt), "db": dy.sum(0).to(dt)}


def _visible(s, Lk):
    """Additive key mask [B, 1, 1, 1, Lk] in 32 bits, or None."""
    if s["lens"] is not None:
        keep = torch.arange(Lk, device="cuda")[None] < s["lens"][:, None]
    elif s["mask"] is None:
        return None
    elif s["mask"].dtype != torch.bool:
        return s["mask"][:, None, None, None]
    else:
        keep = s["mask"]
    return torch.where(keep, 0.0, -math.inf)[:, None, None, None]


def _plain_cross(s):
    dt = s["q"].dtype
    B, Lq, Hq, D = s["q"].shape
    Lk, Hk = s["k"].shape[1:3]
    scale = 1 / math.sqrt(D)

    def heads(t, G):    # [B, Hk, G, L, D] in 32 bits
        return t.float().reshape(B, t.shape[1], Hk, G, D).permute(0, 2, 3, 1, 4).contiguous()

    q, k, v = heads(s["q"], Hq // Hk), heads(s["k"], 1), heads(s["v"], 1)
    S = torch.matmul(q, k.transpose(-1, -2)) * scale
    bias = _visible(s, Lk)
    if bias is not None:
        S = S + bias
    top = S.amax(-1, keepdim=True)
    e = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    l = e.sum(-1, keepdim=True)
    P = e / torch.where(l == 0, 1.0, l)
    o = torch.matmul(P, v)

    def tokens(t):      # back to [B, L, H, D]
        return t.permute(0, 3, 1, 2, 4).reshape(B, t.shape[3], -1, D).to(dt)

    if s["do"] is None:
        return {"o": tokens(o)}
    do = heads(s["do"], Hq // Hk)
    dP = torch.matmul(do, v.transpose(-1, -2))
    dS = P * (dP - (do * o).sum(-1, keepdim=True)) * scale
    dq = torch.matmul(dS, k)
    dk = torch.matmul(dS.transpose(-1, -2), q).sum(2, keepdim=True)
    dv = torch.matmul(P.transpose(-1, -2), do).sum(2, keepdim=True)
    return {"o": tokens(o), "dq": tokens(dq), "dk": tokens(dk), "dv": tokens(dv)}


def _plain_lora(s):
    """All adapters' products at once; a row keeps the columns of its own."""
    x, (E, R, K) = s["x"].float(), s["a"].shape
    rows = torch.arange(x.shape[0], dtype=torch.int32, device="cuda")
    own_id = s["ids"][torch.searchsorted(s["offsets"][1:], rows, right=True)]
    keep = (own_id[:, None] == torch.arange(E, device="cuda")[None]) * s["scales"][None]
    t = torch.matmul(x, s["a"].float().reshape(E * R, K).t()).reshape(-1, E, R) * keep[:, :, None]
    b = s["b"].float().permute(0, 2, 1).reshape(E * R, -1)
    y = torch.matmul(x, s["w"].float().t()) + s["bias"].float() + torch.matmul(t.reshape(-1, E * R), b)
    return {"y": y.to(s["x"].dtype)}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    z = SIZE[case["dtype"]]
    if case["op"] == "norm":
        M, N, step = case["M"], case["N"], case["step"]
        # x in and y out; with the gradients also dy in and dx out, and the weights'.
        return {"bytes": z * (M * N * (4 if step else 2) + N * (4 if step else 2)), "flops": M * N * (22 if step else 8)}
    if case["op"] == "cross":
        B, Lq, Hq, Hk, D, step = (case[k] for k in ("B", "Lq", "Hq", "Hk", "D", "step"))
        keys = sum(_lens(case)) if case["mask"] == "lens" else B * case["Lk"]
        if case["mask"] in ("bool", "add"):
            keys = keys * KEEP
        if case["mask"] == "add" and B > 1:
            keys = keys * (B - 1) / B
        q, kv = B * Lq * Hq * D, 2 * keys * Hk * D
        return {"bytes": z * ((4 * q + 2 * kv) if step else (2 * q + kv)),
                "flops": (14 if step else 4) * Lq * Hq * D * keys}
    M, K, N, R = (case[k] for k in ("M", "K", "N", "R"))
    off, ids = _requests(case)
    used = {a for i, a in enumerate(ids) if a >= 0 and off[i + 1] > off[i]}
    rows = sum(off[i + 1] - off[i] for i, a in enumerate(ids) if a >= 0)
    return {"bytes": z * (M * K + N * K + M * N + N + len(used) * R * (K + N)), "flops": 2 * M * N * K + 2 * rows * R * (K + N)}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "cross": _exact_cross, "lora": _exact_lora}[case["op"]](s)


def _exact_norm(s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    N = x.shape[1]
    mu = x.sum(1) / N
    sd = torch.sqrt((x - mu[:, None]).square().sum(1) / N + EPS)
    xh = (x - mu[:, None]) / sd[:, None]
    out = {"y": torch.addcmul(b, xh, w)}
    if s["dy"] is not None:
        dy = s["dy"].double()
        # The Jacobian of xh against the row: (1 - 1/N - xh xh^T / N) / sd.
        g = dy * w
        out["dx"] = (g - g.sum(1)[:, None] / N - xh * (torch.linalg.vecdot(g, xh)[:, None] / N)) / sd[:, None]
        out["dw"], out["db"] = torch.linalg.vecdot(dy, xh, dim=0), torch.sum(dy, 0)
    return out


def _exact_cross(s):
    B, Lq, Hq, D = s["q"].shape
    Lk, Hk = s["k"].shape[1:3]
    G = Hq // Hk
    o = torch.zeros(B, Lq, Hq, D, dtype=torch.float64, device="cuda")
    dq, dk = torch.zeros_like(o), torch.zeros(B, Lk, Hk, D, dtype=torch.float64, device="cuda")
    dv = torch.zeros_like(dk)
    for b in range(B):
        if s["lens"] is not None:
            seen = torch.arange(Lk, device="cuda") < s["lens"][b]
            add = torch.zeros(Lk, dtype=torch.float64, device="cuda")
        elif s["mask"] is None or s["mask"].dtype == torch.bool:
            seen = torch.ones(Lk, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][b]
            add = torch.zeros(Lk, dtype=torch.float64, device="cuda")
        else:
            seen, add = s["mask"][b] > -math.inf, s["mask"][b].double()
        if not bool(seen.any()):
            continue
        add = add[seen]
        for h in range(Hq):
            q, k, v = s["q"][b, :, h].double(), s["k"][b, seen, h // G].double(), s["v"][b, seen, h // G].double()
            P = torch.softmax(q @ k.T / math.sqrt(D) + add, 1)
            o[b, :, h] = P @ v
            if s["do"] is not None:
                do = s["do"][b, :, h].double()
                dP = do @ v.T
                dS = P * (dP - torch.linalg.vecdot(P, dP)[:, None]) / math.sqrt(D)
                dq[b, :, h] = dS @ k
                dk[b, seen, h // G] += dS.T @ q
                dv[b, seen, h // G] += P.T @ do
    return {"o": o} if s["do"] is None else {"o": o, "dq": dq, "dk": dk, "dv": dv}


def _exact_lora(s):
    x = s["x"].double()
    y = x @ s["w"].double().T + s["bias"].double()
    off, ids, scales = s["offsets"].tolist(), s["ids"].tolist(), s["scales"].double()
    for i, a in enumerate(ids):
        if a >= 0 and off[i + 1] > off[i]:
            r = slice(off[i], off[i + 1])
            y[r] += scales[a] * (x[r] @ s["a"][a].double().T) @ s["b"][a].double().T
    return {"y": y}
