"""The operators together: the example's training step against the same step in 32-bit torch operations, and its loss over some steps."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("finetune_block", os.path.join(ROOT, "examples", "finetune_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_block(b, w, x, scale, shift, radius):
    """Block.__call__ on fp32 CPU tensors with elementary operations."""
    B, N, width = x.shape

    def norm(t, s, o):
        c = t - t.mean(-1, keepdim=True)
        return c / torch.sqrt(c.square().mean(-1, keepdim=True) + 1e-6) * s + o
    angle = (b.places.cpu().double().unsqueeze(-1) * b.freqs.cpu().unsqueeze(1)).sum(0)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turn(t):  # [B, H, N, d]
        e, o = t[..., 0::2], t[..., 1::2]
        return torch.stack([e * cos - o * sin, e * sin + o * cos], -1).flatten(-2)
    h = norm(x, 1 + scale.unsqueeze(1), shift.unsqueeze(1))
    q, k, v = ((h @ w["qkv"].t()).view(B, N, 3, b.heads, -1).unbind(2))
    q, k, v = turn(q.transpose(1, 2)), turn(k.transpose(1, 2)), v.transpose(1, 2)
    place = torch.arange(b.grid * b.grid)
    row, col = place // b.grid, place % b.grid
    near = (row[:, None] - row) ** 2 + (col[:, None] - col) ** 2 < radius * radius
    mask = torch.ones(N, N, dtype=torch.bool)
    mask[b.n_text:, b.n_text:] = near
    scores = (q @ k.transpose(-1, -2) / q.shape[-1] ** 0.5).masked_fill(~mask, float("-inf"))
    a = torch.softmax(scores, -1) @ v
    x = x + a.transpose(1, 2).reshape(B, N, width) @ w["out"].t()
    h = norm(x, w["scale"], w["shift"])
    g = h @ w["gate"].t()
    return x + (g / (1 + torch.exp(-g)) * (h @ w["up"].t())) @ w["down"].t()


def test_a_training_step_against_plain_operations(example):
    # every bf16 tensor on the way adds 2^-9 of itself; a dozen of them in a row, added as independent errors, stay under 2^-9 * sqrt(12) = 0.7 % of a
    # result's norm forward; the way back has as many again and the products of both: 2 % allowed
    b = example.Block(n_text=9, grid=12, heads=3, seed=4)
    g = torch.Generator().manual_seed(2)
    x, scale, shift = (torch.randn(2, 9 + 144, 192, generator=g).bfloat16(), (0.1 * torch.randn(2, 192, generator=g)).bfloat16(), (0.1 * torch.randn(2, 192, generator=g)).bfloat16())
    dy = torch.randn(2, 9 + 144, 192, generator=g).bfloat16()
    mine = [t.cuda().requires_grad_() for t in (x, scale, shift)]
    names = list(b.weights)
    for n in names:
        b.weights[n].requires_grad_()
    y = b(*mine, radius=4)
    y.backward(dy.cuda())
    w = {n: b.weights[n].detach().float().cpu().requires_grad_() for n in names}
    plain = [t.float().requires_grad_() for t in (x, scale, shift)]
    want = plain_block(b, w, *plain, radius=4)
    want.backward(dy.float())
    off = lambda got, ref: float((got.float().cpu() - ref).norm() / ref.norm())
    assert off(y.detach(), want.detach()) < 0.007
    for got, ref in list(zip(mine, plain)) + [(b.weights[n], w[n]) for n in names]:
        assert got.grad.shape == ref.grad.shape and off(got.grad, ref.grad) < 0.02


@pytest.mark.parametrize("bits", [8, 32])
def test_the_example_learns(example, bits):
    losses = example.finetune(n_text=16, grid=16, heads=2, radius=4, steps=30, state_bits=bits, say=None)
    assert all(v == v for v in losses) and sum(losses[-5:]) < 0.9 * sum(losses[:5])
