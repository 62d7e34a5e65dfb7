"""A text-conditioned block of a noise network over the operators of :mod:`ops`.

    y = h + O(attend(Q(norm h), K(context), V(context)))

h holds the tokens of a batch of latents ([batch, tokens, hidden], e.g. the 2 x 2 patches of the sampler's
latents, batch x tokens rows of one matrix), context the states of a prompt encoder ([batch, states,
context]), of which the first ``lengths[b]`` belong to sample b's prompt. Each request of a batch may bring
its own low-rank adapters for the four projections.

:meth:`ConditionedBlock.serve` runs a batch whose requests have adapters of their own (no gradients).
:meth:`ConditionedBlock.__call__` is the same block without adapters, differentiable (once) in its inputs and
weights: norm and attention and their backward passes run in the library's kernels, the plain projections
in torch's.
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
