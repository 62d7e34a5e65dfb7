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
