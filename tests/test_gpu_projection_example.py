"""The example that runs the 8-bit projection, the heads and their gradients together: against autograd of the same in fp32, and that it learns.

Tolerance of the comparison: E4M3 keeps 4 bits of a value, an error of at most 2^-4 (rms 2^-4 / sqrt(3) / 1.5) of it; products of two such
operands are off by about sqrt(2) times that rms, and sums of many independent ones in proportion, 3.5 % of their norm.  Forwards and backwards pass
three such products in a row (the gradient of the norm sees the projection's result): 15 % is beyond them and far below what a wrong term would give."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def distance(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_gradients_follow_those_of_fp32(dtype):
    import projection_8bit as example
    gen = torch.Generator(device="cuda").manual_seed(5)
    p = example.Projection(384, 6, 64, "cuda", 3)
    p.q_weight.add_(torch.randn(64, generator=gen, device="cuda") * 0.1)
    x = torch.randn((320, 384), generator=gen, device="cuda").to(dtype)
    positions = torch.arange(64, device="cuda").repeat(5)
    p.quantise()
    out, saved = p.forward(x, positions)
    grads = [torch.randn(o.shape, generator=gen, device="cuda").to(dtype) for o in out]
    dx, dp = p.backward(*grads, saved)
    leaf = x.float().requires_grad_()
    for t in p.parameters():
        t.requires_grad_()
    want = p.plain(leaf, positions)
    torch.autograd.backward(want, [g.float() for g in grads])
    for a, b in zip(out, want):
        assert distance(a, b.detach()) < 0.15
    for a, b in zip((dx,) + dp, (leaf.grad,) + tuple(t.grad for t in p.parameters())):
        assert a.shape == b.shape and distance(a, b) < 0.15


def test_the_example_learns():
    import projection_8bit as example
    losses = example.train(steps=30, tokens=512, channels=192, heads=3, images=8)
    assert losses[-1] < 0.7 * losses[0]
