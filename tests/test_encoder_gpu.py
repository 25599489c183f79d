"""The per-bird encoder's differentiable functions and its example."""

import os
import sys

import pytest
import torch

from paper_2512_07009_amd import RotaryAxes, encoder

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_block_gradients_follow_the_loss():
    """A small step against the gradient lowers the loss by the gradient's
    square, to first order (bfloat16 features: within a quarter)."""
    torch.manual_seed(1)
    n = 300
    off = torch.tensor([0, 100, 100, 180, 300], dtype=torch.int32, device="cuda")
    xy = torch.randint(0, 16 * 300, (n, 2), dtype=torch.int32, device="cuda")
    block = encoder.EncoderBlock(64, q_heads=4, kv_heads=2, head_dim=32, axes=RotaryAxes(y=[0.1] * 8, x=[0.05] * 8),
                                 cap=20.0).cuda()
    x = torch.randn(n, 64, device="cuda").to(torch.bfloat16)
    goal = torch.randn(n, 64, device="cuda")

    def loss():
        return ((block(x, off, xy).float() - goal) ** 2).mean()

    first = loss()
    first.backward()
    moved = [block.norm_weight, block.norm_bias, block.log_slopes]
    square = sum((p.grad ** 2).sum() for p in moved)
    assert square > 0 and all(torch.isfinite(p.grad).all() for p in block.parameters())
    step = 0.02 * first.item() / square.item()
    with torch.no_grad():
        for p in moved:
            p -= step * p.grad
    drop = (first - loss()).item()
    assert 0.75 * step * square.item() <= drop <= 1.25 * step * square.item()


def test_frames_do_not_see_each_other():
    torch.manual_seed(2)
    off = torch.tensor([0, 70, 200], dtype=torch.int32, device="cuda")
    xy = torch.randint(0, 16 * 300, (200, 2), dtype=torch.int32, device="cuda")
    block = encoder.EncoderBlock(64, q_heads=2, head_dim=32, axes=RotaryAxes(y=[0.1] * 8, x=[0.05] * 8)).cuda()
    x = torch.randn(200, 64, device="cuda").to(torch.bfloat16)
    with torch.no_grad():
        a = block(x, off, xy)
        x[70:] = 0
        xy[70:] = 0
        b = block(x, off, xy)
    assert torch.equal(a[:70], b[:70])


def test_example_learns():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import bird_encoder
    losses, right = bird_encoder.main(steps=40, frames=4, height=240, width=320, n_birds=150, quiet=True)
    assert torch.isfinite(losses).all()
    assert losses[-5:].mean() < 0.7 * losses[:5].mean()
