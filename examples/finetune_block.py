"""Fine-tunes one transformer block with CLEAR local attention towards the same block with full attention, as the distillation of the paper does for every
block of its model (arXiv 2412.16112, Sec. 3.3), with every operator of this library that a training step of it meets:

    adaptive layer norm -> projections (torch) -> rotary positions of two image axes -> CLEAR local attention
    -> residual with the next layer norm -> gated feed-forward projection -> projection (torch) -> loss -> backward -> AdamW, gradients clipped, states in 8 bits

    python examples/finetune_block.py [--grid 32] [--heads 8] [--steps 20] [--radius 4]

Weights and data are random; the loss is the mean square of the difference over that of the teacher's change to its input."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2412_16112_amd import clear_block as cb  # noqa: E402
from paper_2412_16112_amd.autograd import clear_attention, gated_ff, layer_norm, residual_norm, rotary  # noqa: E402
from paper_2412_16112_amd.optim import AdamW  # noqa: E402

HEAD_DIM = 64


class Block:
    """One block over n_text text tokens and a grid x grid image, in bf16; `radius` of its attention."""

    def __init__(self, n_text, grid, heads, seed=0, device="cuda"):
        self.n_text, self.grid, self.heads = n_text, grid, heads
        width, hidden = heads * HEAD_DIM, 8 * (heads * HEAD_DIM // 3)
        g = torch.Generator().manual_seed(seed)
        weight = lambda rows, cols: (torch.randn(rows, cols, generator=g) / cols ** 0.5).to(device, torch.bfloat16)
        self.weights = {"qkv": weight(3 * width, width), "out": weight(width, width), "scale": torch.ones(width, device=device, dtype=torch.bfloat16),
                        "shift": torch.zeros(width, device=device, dtype=torch.bfloat16), "gate": weight(hidden, width), "up": weight(hidden, width), "down": weight(width, hidden)}
        # two position axes, half of the pairs each; the text tokens stand at the origin
        axis = cb.rotary_frequencies(HEAD_DIM // 2)
        self.freqs = torch.zeros(2, HEAD_DIM // 2, dtype=torch.float64)
        self.freqs[0, :HEAD_DIM // 4], self.freqs[1, HEAD_DIM // 4:] = axis, axis
        self.freqs = self.freqs.to(device)
        image = torch.arange(grid * grid)
        text = torch.zeros(n_text, dtype=torch.int64)
        self.places = torch.stack([torch.cat([text, image // grid]), torch.cat([text, image % grid])]).to(device)  # [2, N]

    def __call__(self, x, scale, shift, radius):
        """x [B, N, width]; scale, shift [B, width] from the conditioning of each item."""
        w, (B, N, width) = self.weights, x.shape
        linear = lambda t, name: (t.reshape(-1, t.shape[-1]) @ w[name].t()).view(B, N, -1)
        h = layer_norm(x, scale, shift, weight_offset=1.0)
        q, k, v = (t.transpose(1, 2) for t in linear(h, "qkv").view(B, N, 3, self.heads, HEAD_DIM).unbind(2))  # [B, H, N, d], as the projection stored them
        q, k = rotary(q, k, self.places[:, None].expand(2, B, N), self.freqs)
        a = clear_attention(q, k, v, self.n_text, self.grid, self.grid, radius)
        x, h = residual_norm(x, linear(a.transpose(1, 2).reshape(B, N, width), "out"), weight=w["scale"], bias=w["shift"])
        return x + linear(gated_ff(h, w["gate"], w["up"]), "down")


def finetune(n_text=32, grid=32, heads=8, radius=4, steps=20, lr=1e-3, seed=0, state_bits=8, say=print):
    """The losses of the steps."""
    teacher, student = Block(n_text, grid, heads, seed), Block(n_text, grid, heads, seed)
    params = [w.requires_grad_() for w in student.weights.values()]
    opt = AdamW(params, lr=lr, weight_decay=0.0, state_bits=state_bits, masters=True)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    draw = lambda *shape, k=1.0: (k * torch.randn(*shape, generator=g, device="cuda")).to(torch.bfloat16)
    losses = []
    for step in range(steps):
        x, scale, shift = draw(2, n_text + grid * grid, heads * HEAD_DIM), draw(2, heads * HEAD_DIM, k=0.1), draw(2, heads * HEAD_DIM, k=0.1)
        with torch.no_grad():
            want = teacher(x, scale, shift, 2 * grid)  # a radius beyond the diagonal: full attention
        off = (student(x, scale, shift, radius) - want).float()
        loss = off.square().mean() / (want - x).float().square().mean()
        loss.backward()
        opt.step(max_norm=1.0)  # gradients clipped to a norm of 1, without waiting for it
        opt.zero_grad()
        losses.append(loss.detach())
        if say and (step % 5 == 0 or step + 1 == steps):
            say("step %3d  loss %.5f" % (step, float(loss.detach())))
    return [float(v) for v in losses]


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--grid", type=int, default=32)
    p.add_argument("--heads", type=int, default=8)
    p.add_argument("--radius", type=int, default=4)
    p.add_argument("--steps", type=int, default=40)
    a = p.parse_args()
    finetune(grid=a.grid, heads=a.heads, radius=a.radius, steps=a.steps)
