"""What the differentiable operators of paper_2609_36522_amd.ops keep and compute, on formulas in the kernels' place (CPU)."""
import pytest
import torch

import block_ops_reference as R
from paper_2609_36522_amd import ops as O


@pytest.fixture
def leaves(monkeypatch):
    for t in (R.U, R.TINY):
        monkeypatch.setitem(t, torch.float64, 0.0)
    g = torch.Generator().manual_seed(3)
    shapes = (4, 5), (7, 5), (7, 5), (3, 7), (7,), (7,), (3,)
    return [torch.randn(s, generator=g, dtype=torch.float64).requires_grad_(i > 0) for i, s in enumerate(shapes)]


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_feed_forward_saves_nothing_without_gradients(leaves, monkeypatch, mode):
    """A validation pass over trainable weights: their flags say that they need gradients, the mode that nothing does."""
    saves = []

    def forward(x, gate, up, down, *biases, activation, save):
        saves.append(save)
        return R.feed_forward(x.detach(), *(t.detach() for t in (gate, up, down)), tuple(b.detach() for b in biases), activation)["y"][0], torch.zeros(1)

    monkeypatch.setattr(O, "feed_forward_forward", forward)
    want = O.feed_forward(*leaves)
    assert want.requires_grad and saves == [True]
    with mode():
        y = O.feed_forward(*leaves)
    assert saves == [True, False] and not y.requires_grad and torch.equal(y, want.detach())
    y = O.feed_forward(*(t.detach() for t in leaves))
    assert saves == [True, False, False] and not y.requires_grad


@pytest.mark.parametrize("trained", [(0,), (1,), (2,), (0, 2), (0, 1, 2)])
def test_group_norm_computes_the_gradients_that_are_needed(monkeypatch, trained):
    for t in (R.U, R.TINY):
        monkeypatch.setitem(t, torch.float64, 0.0)
    asked = []
    monkeypatch.setattr(O, "group_norm_forward", lambda x, n, w, b, eps, activation:
                        (R.group_norm(x.detach(), n, w.detach(), b.detach(), eps, activation)["y"][0], torch.zeros(2, n), None))

    def backward(dy, x, mean, rstd, w, b, *, activation, need=(True,) * 3):
        asked.append(need)
        ref = R.group_norm(x.detach(), mean.shape[1], w.detach(), b.detach(), 1e-5, activation, dy)
        return tuple(ref[n][0] if k else None for n, k in zip(("dx", "dw", "db"), need))

    monkeypatch.setattr(O, "group_norm_backward", backward)
    g = torch.Generator().manual_seed(4)
    leaves = [torch.randn(s, generator=g, dtype=torch.float64).requires_grad_(i in trained) for i, s in enumerate(((2, 5, 6), (6,), (6,)))]
    dy = torch.randn((2, 5, 6), generator=g, dtype=torch.float64)
    O.group_norm(leaves[0], 3, *leaves[1:], activation="silu").backward(dy)
    assert asked == [tuple(i in trained for i in range(3))]
    ref = R.group_norm(*(leaves[0].detach(), 3), leaves[1].detach(), leaves[2].detach(), 1e-5, "silu", dy)
    for i, name in enumerate(("dx", "dw", "db")):
        assert torch.equal(leaves[i].grad, ref[name][0]) if i in trained else leaves[i].grad is None
