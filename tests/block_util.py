"""Plain definitions of the operators around the attention in 64 bits, written out on CPU tensors."""
import math

import torch


def rotary(x, positions, freqs, interleaved, scale=1.0, inverse=False):
    """x [B, H, N, d]; positions [axes, B, N]; freqs [axes, rot / 2]: fp64 result."""
    x = x.double().cpu()
    positions, freqs = positions.double().cpu(), freqs.double().cpu()
    half = freqs.shape[1]
    angle = sum(positions[a].unsqueeze(-1) * freqs[a] for a in range(freqs.shape[0])).unsqueeze(1)
    c, s = torch.cos(angle) * scale, torch.sin(angle) * scale * (-1 if inverse else 1)
    y = x.clone()
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def layer_norm(x, weight, bias, eps, offset):
    """x [B, N, C] fp64 (CPU); weight, bias [C], [B, C] or None."""
    mean = x.mean(-1, keepdim=True)
    xhat = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    wide = lambda t: t.unsqueeze(1) if t.dim() == 2 else t
    y = xhat if weight is None else xhat * (offset + wide(weight))
    return y if bias is None else y + wide(bias)


def activation(g, name):
    if name == "silu":
        return g / (1 + torch.exp(-g))
    if name == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    return 0.5 * g * (1 + torch.erf(g / math.sqrt(2)))


def activation_slope(g, name):
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
    return 0.5 * (1 + torch.erf(g / math.sqrt(2))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
