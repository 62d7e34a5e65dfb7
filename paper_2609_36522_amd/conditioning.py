"""Text-conditioned blocks of a noise network over the operators of :mod:`ops`.

    ConditionedBlock:  y = h + O(attend(Q(norm h), K(context), V(context)))
    FeedForwardBlock:  y = h + D(act(G(norm h)) * U(norm h))
    LatentBlock:       y = x + Out(FeedForwardBlock(ConditionedBlock(In(silu(group norm x)), context)))

h holds the tokens of a batch of latents ([batch, tokens, hidden], e.g. the 2 x 2 patches of the sampler's
latents, batch x tokens rows of one matrix), context the states of a prompt encoder ([batch, states,
context]), of which the first ``lengths[b]`` belong to sample b's prompt. Each request of a batch may bring
its own low-rank adapters for the four projections.

:meth:`ConditionedBlock.serve` runs a batch whose requests have adapters of their own (no gradients).
:meth:`ConditionedBlock.__call__` is the same block without adapters, differentiable (once) in its inputs and
weights: norm and attention and their backward passes run in the library's kernels, the plain projections
in torch's.

:class:`FeedForwardBlock` runs on tokens alone. :class:`LatentBlock` puts the two around a channels-last latent
([batch, height, width, channels], whose pixels are the tokens); its ``serve`` takes the projections into and out of the
block in 8-bit integers (:meth:`LatentBlock.quantize`).
"""
from __future__ import annotations

import math

import torch

from . import ops

PROJECTIONS = ("q", "k", "v", "o")


class Adapters:
    """``count`` adapters of one rank for each projection: a[p] [count, rank, in], b[p] [count, out, rank],
    and their scales [count]."""

    def __init__(self, a, b, scales):
        self.a, self.b, self.scales = a, b, scales


class ConditionedBlock:
    """Weights of one block, as tensors of ``dtype`` on the current device: norm's ``weight`` and ``bias``
    [hidden] and the projections ``w`` [out, in] (q: hidden from hidden; k, v: kv_heads x head_dim from
    context; o: hidden from hidden)."""

    def __init__(self, hidden, context, heads, kv_heads=None, *, dtype=torch.bfloat16, seed=0, eps=1e-5):
        if hidden % heads:
            raise ValueError("hidden must be a multiple of heads")
        self.hidden, self.context, self.heads, self.eps = hidden, context, heads, eps
        self.kv_heads = heads if kv_heads is None else kv_heads
        self.head_dim = hidden // heads
        g = torch.Generator(device="cuda").manual_seed(seed)
        kv = self.kv_heads * self.head_dim
        self.shapes = {"q": (hidden, hidden), "k": (kv, context), "v": (kv, context), "o": (hidden, hidden)}
        self.w = {p: (torch.randn(s, generator=g, device="cuda") / math.sqrt(s[1])).to(dtype) for p, s in self.shapes.items()}
        self.weight = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).to(dtype)
        self.bias = (0.1 * torch.randn(hidden, generator=g, device="cuda")).to(dtype)

    def adapters(self, count, rank, *, seed=1) -> Adapters:
        """Seeded adapters for this block's projections."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = self.weight.dtype
        a = {p: (torch.randn((count, rank, s[1]), generator=g, device="cuda") / math.sqrt(s[1])).to(dt) for p, s in self.shapes.items()}
        b = {p: (torch.randn((count, s[0], rank), generator=g, device="cuda") / math.sqrt(rank)).to(dt) for p, s in self.shapes.items()}
        return Adapters(a, b, 0.5 + torch.rand(count, generator=g, device="cuda"))

    def parameters(self):
        return [self.weight, self.bias, *(self.w[p] for p in PROJECTIONS)]

    def _split(self, t, heads):
        return t.reshape(*t.shape[:2], heads, self.head_dim)

    @torch.no_grad()
    def serve(self, h, context, adapters: Adapters, ids, *, lengths=None):
        """One pass for a batch of requests; request b (a sample) uses adapter ids[b] (int32, none if
        negative). lengths: int32 [batch], the prompts' states (all of them if None)."""

        def offsets(x):
            batch, rows = x.shape[:2]
            if rows == 0:
                return torch.zeros(batch + 1, dtype=torch.int32, device=x.device)
            return torch.arange(0, batch * rows + 1, rows, dtype=torch.int32, device=x.device)

        tokens, states = offsets(h), offsets(context)

        def project(p, x, off):
            y = ops.lora_linear(x.reshape(x.shape[0] * x.shape[1], x.shape[2]), self.w[p], adapters.a[p], adapters.b[p], off, ids,
                                scales=adapters.scales)
            return y.reshape(*x.shape[:2], y.shape[1])

        x, _, _ = ops.layer_norm_forward(h, self.weight, self.bias, self.eps)
        q = self._split(project("q", x, tokens), self.heads)
        k = self._split(project("k", context, states), self.kv_heads)
        v = self._split(project("v", context, states), self.kv_heads)
        o, _ = ops.cross_attention_forward(q, k, v, kv_lens=lengths)
        return h + project("o", o.reshape(h.shape), tokens)

    def __call__(self, h, context, *, lengths=None):
        """The block without adapters, differentiable."""
        x = ops.layer_norm(h, self.weight, self.bias, self.eps)
        q = self._split(torch.nn.functional.linear(x, self.w["q"]), self.heads)
        k = self._split(torch.nn.functional.linear(context, self.w["k"]), self.kv_heads)
        v = self._split(torch.nn.functional.linear(context, self.w["v"]), self.kv_heads)
        o = ops.cross_attention(q, k, v, kv_lens=lengths).reshape(h.shape)
        return h + torch.nn.functional.linear(o, self.w["o"])


class FeedForwardBlock:
    """Weights of one block, as tensors of ``dtype`` on the current device: norm's ``weight`` and ``bias`` [hidden],
    ``gate`` and ``up`` [inner, hidden], ``down`` [hidden, inner] and their biases."""

    def __init__(self, hidden, inner=None, *, activation="gelu", dtype=torch.bfloat16, seed=2, eps=1e-5):
        inner = 4 * hidden if inner is None else inner
        self.hidden, self.inner, self.activation, self.eps = hidden, inner, activation, eps
        g = torch.Generator(device="cuda").manual_seed(seed)

        def draw(*shape, scale=1.0, offset=0.0):
            return (offset + scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)

        self.weight, self.bias = draw(hidden, scale=0.1, offset=1.0), draw(hidden, scale=0.1)
        self.gate, self.up = (draw(inner, hidden, scale=1 / math.sqrt(hidden)) for _ in range(2))
        self.down = draw(hidden, inner, scale=1 / math.sqrt(inner))
        self.gate_bias, self.up_bias, self.down_bias = draw(inner, scale=0.1), draw(inner, scale=0.1), draw(hidden, scale=0.1)

    def parameters(self):
        return [self.weight, self.bias, self.gate, self.up, self.down, self.gate_bias, self.up_bias, self.down_bias]

    @torch.no_grad()
    def serve(self, h):
        x, _, _ = ops.layer_norm_forward(h, self.weight, self.bias, self.eps)
        y, _ = ops.feed_forward_forward(x, self.gate, self.up, self.down, self.gate_bias, self.up_bias, self.down_bias,
                                        activation=self.activation, save=False)
        return h + y

    def __call__(self, h):
        """Differentiable, like :meth:`ConditionedBlock.__call__`."""
        x = ops.layer_norm(h, self.weight, self.bias, self.eps)
        return h + ops.feed_forward(x, self.gate, self.up, self.down, self.gate_bias, self.up_bias, self.down_bias,
                                    activation=self.activation)


class Int8Weights:
    """8-bit forms of a block's projections: (weight, scale) for each name."""

    def __init__(self, weights):
        self.weights = {name: ops.quantize_rows(w) for name, w in weights.items()}

    def project(self, name, x, bias):
        q, scale = ops.quantize_rows(x)
        return ops.int8_linear(q, scale, *self.weights[name], bias, dtype=x.dtype)


class LatentBlock:
    """A latent's group norm, the projection of its pixels to tokens, a :class:`ConditionedBlock` (``attention``), a
    :class:`FeedForwardBlock` (``feed``) and the projection back, added to the latent. Weights: the norm's ``weight``
    and ``bias`` [channels], ``w_in`` [hidden, channels], ``w_out`` [channels, hidden] and their biases."""

    def __init__(self, channels, groups, hidden, context, heads, kv_heads=None, *, inner=None, dtype=torch.bfloat16, seed=0, eps=1e-5):
        if channels % groups:
            raise ValueError("channels must be a multiple of groups")
        self.channels, self.groups, self.hidden, self.eps = channels, groups, hidden, eps
        self.attention = ConditionedBlock(hidden, context, heads, kv_heads, dtype=dtype, seed=seed, eps=eps)
        self.feed = FeedForwardBlock(hidden, inner, dtype=dtype, seed=seed + 2, eps=eps)
        g = torch.Generator(device="cuda").manual_seed(seed + 3)

        def draw(*shape, scale=1.0, offset=0.0):
            return (offset + scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)

        self.weight, self.bias = draw(channels, scale=0.1, offset=1.0), draw(channels, scale=0.1)
        self.w_in, self.b_in = draw(hidden, channels, scale=1 / math.sqrt(channels)), draw(hidden, scale=0.1)
        self.w_out, self.b_out = draw(channels, hidden, scale=1 / math.sqrt(hidden)), draw(channels, scale=0.1)

    def parameters(self):
        return [self.weight, self.bias, self.w_in, self.b_in, self.w_out, self.b_out, *self.attention.parameters(), *self.feed.parameters()]

    def quantize(self) -> Int8Weights:
        """The projections into and out of the block in 8 bits, for :meth:`serve`; to be called again when they change."""
        with torch.no_grad():
            return Int8Weights({"in": self.w_in, "out": self.w_out})

    def _tokens(self, t):
        return t.reshape(t.shape[0], t.shape[1] * t.shape[2], t.shape[3])

    @torch.no_grad()
    def serve(self, x, context, adapters: Adapters, ids, int8: Int8Weights, *, lengths=None):
        """One pass for a batch of requests, each with an adapter of its own for the attention's projections
        (:meth:`ConditionedBlock.serve`)."""
        t, _, _ = ops.group_norm_forward(x, self.groups, self.weight, self.bias, self.eps, activation="silu")
        t = int8.project("in", self._tokens(t), self.b_in)
        t = self.feed.serve(self.attention.serve(t, context, adapters, ids, lengths=lengths))
        return x + int8.project("out", t, self.b_out).reshape(x.shape)

    def __call__(self, x, context, *, lengths=None):
        """The block without adapters, differentiable, in 16 bits."""
        t = self._tokens(ops.group_norm(x, self.groups, self.weight, self.bias, self.eps, activation="silu"))
        t = torch.nn.functional.linear(t, self.w_in, self.b_in)
        t = self.feed(self.attention(t, context, lengths=lengths))
        return x + torch.nn.functional.linear(t, self.w_out, self.b_out).reshape(x.shape)
