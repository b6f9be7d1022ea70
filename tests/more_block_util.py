"""Plain definitions in 64 bits of the gated residual with its norms, the gradients' norm and the operands in 4 bits, written out on CPU tensors, and how far results may be off."""
import torch

FP32 = 2.0 ** -24  # half a step of fp32, relative
MX_VALUES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def unit(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)


def wide(v):
    return v.unsqueeze(1) if v.dim() == 2 else v


def residual_norm(x, y, gate, weight, bias, post_weight, kind, post, eps, scale, offset, post_offset):
    """(r, h) for fp64 tensors [B, N, C]; gate, weight, bias [C] or [B, C]; any of the vectors None."""
    z = y
    if post is not None:
        z = unit(y, post, eps)
        if post_weight is not None:
            z = z * (post_offset + post_weight)
    r = scale * x + (z if gate is None else wide(gate) * z)
    h = unit(r, kind, eps)
    if weight is not None:
        h = h * (offset + wide(weight))
    return r, h if bias is None else h + wide(bias)


def exponents(x):
    """Stored exponents of the blocks of fp32 or bf16 x [rows, C]: int64 [rows, C / 32]."""
    top = x.float().abs().view(x.shape[0], -1, 32)
    bits = top.view(torch.int32).amax(2).long()
    # the exponent field, of which 2 are taken off; subnormal and tiny blocks have 2^-127; NaN and infinity 255
    return torch.where(bits >= 0x7f800000, 255, (bits.div(1 << 23, rounding_mode="floor") - 2).clamp(min=0))


def quantized(x):
    """(values, exponents) that the 4-bit form of x [rows, C] stands for: fp64."""
    e = exponents(x)
    blocks = x.double().view(x.shape[0], -1, 32)
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - 127).double()).unsqueeze(2)
    share = blocks / scale
    distance = (share.abs().unsqueeze(-1) - MX_VALUES[:8]).abs()
    nearest = distance.amin(-1, keepdim=True)
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])  # even codes first: they win where two are as near
    code = order[(distance[..., order] == nearest).int().argmax(-1)]
    values = torch.copysign(MX_VALUES[code], share) * scale
    return torch.where(e.unsqueeze(2) == 255, torch.nan, values).view(x.shape), e


def scale_bytes(scales, channels):
    """Row-major exponents [rows, C / 32] of scales [groups, rows, 8]."""
    return scales.permute(1, 0, 2).reshape(scales.shape[1], -1)[:, :channels // 32].long()


def decoded(codes, scales):
    """Values [rows, C] of CPU codes and scales: fp64."""
    rows, C = codes.shape[0], 2 * codes.shape[1]
    nibbles = torch.stack([codes.long() & 15, codes.long() >> 4], -1).view(rows, C)
    e = scale_bytes(scales, C)
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - 127).double())
    return MX_VALUES[nibbles] * torch.where(e == 255, torch.nan, scale).repeat_interleave(32, 1)


def check(got, want, off, what):
    """|got - want| <= off element by element; NaN only where NaN is wanted."""
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape, what
    assert torch.equal(got.isnan(), want.isnan()), what
    off = torch.as_tensor(off, dtype=torch.float64).cpu().expand_as(want)
    fine = ~want.isnan() & (got != want)
    over = ((got - want).abs() / off.clamp(min=1e-300))[fine]
    assert over.numel() == 0 or float(over.max()) <= 1, "%s: %.3g times what it may be off" % (what, float(over.max()))
