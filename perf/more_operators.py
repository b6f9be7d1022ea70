"""Timings of three more groups of operators of a transformer block and its training step, each in its plain form (elementary
torch operations in 32 bits) and through this library: what lies between two sublayers, the norm of all gradients with clipping,
and products of operands held in 4 bits.

`listed()` names twelve cases, `draw(rng)` gives another of the same ranges, `prepare` makes what a program holds before the
call, `run` is one pass as such a program calls it, `work` the bytes and operations that a pass cannot do without, `exact` the
outputs from the operators' definitions in 64 bits.

A case's "op" is one of
  residual  r = a x + gate * post(y), h = norm(r) * weight + bias: the gated residual of a sublayer's output y (which may have a norm of
            its own first) and the next sublayer's norm; with "train" its backward pass too;
  clip      the norm of all gradients and the factor that clips it; with "in_place" the gradients are scaled too;
  quantize  rows of numbers to 4 bits with a scale for every 32 of them, and back to the numbers that these stand for;
  linear    x W^T + bias with W held in 4 bits and x taken to 4 bits."""
import itertools
import math

import torch

own = False


# ---- cases ------------------------------------------------------------------------------------------------------------

def _residual(B, N, C, dtype, stream, weight, kind, post, gate, per_item, scale, train):
    """dtype: of y and h; stream: of x and r; weight: of the vectors; post: the norm of y, or ""; gate: "item", "shared" or "";
    per_item: weight and bias per batch item, the weight's distance from 1 then; scale: a."""
    return dict(op="residual", B=B, N=N, C=C, dtype=dtype, stream=stream, weight=weight, kind=kind, post=post, gate=gate, per_item=per_item, scale=scale, train=train)


def _clip(blocks, width, hidden, matrices, vectors, norm, in_place):
    return dict(op="clip", blocks=blocks, width=width, hidden=hidden, matrices=matrices, vectors=vectors, norm=norm, in_place=in_place)


def _quantize(M, C, dtype, out):
    return dict(op="quantize", M=M, C=C, dtype=dtype, out=out)


def _linear(M, C, F, dtype, out, bias):
    return dict(op="linear", M=M, C=C, F=F, dtype=dtype, out=out, bias=bias)


def listed():
    return [
        # a short prompt's rows between attention and feed-forward layer, inference: a fraction of the chip, launch bound
        dict(_residual(1, 77, 2432, "bf16", "bf16", "bf16", "layer", "", "item", True, 1.0, False), name="residual-prompt"),
        # a training step of an adaptive block at 1024 x 1024 pixels: gate, scale and shift from the conditioning of each batch item
        dict(_residual(2, 512 + 64 * 64, 2432, "bf16", "bf16", "bf16", "layer", "", "item", True, 1.0, True), name="residual-adaptive-train"),
        # inference at 2048 x 2048 pixels: root mean square norms before and after the sublayer, the residual stream in fp32
        dict(_residual(1, 512 + 128 * 128, 4096, "bf16", "f32", "f32", "rms", "rms", "item", False, 1.0, False), name="residual-sandwich-2048"),
        # an odd width in fp32 with a damped residual, both norms and a gate with learned weights, ragged rows, training
        dict(_residual(1, 333 + 128 * 128, 1111, "f32", "f32", "f32", "layer", "rms", "shared", False, 0.75, True), name="residual-odd-f32-train"),
        # the norms and adapters of a small model: many tensors of a few hundred elements, clipped in place, launch bound
        dict(_clip(2, 96, 250, "f32", "f32", 2, True), name="clip-small"),
        # the gradients of four blocks in bf16, whose factor goes to the optimizer
        dict(_clip(4, 1536, 4096, "bf16", "bf16", 2, False), name="clip-factor-bf16"),
        # matrices in bf16 beside vectors in fp32, odd sizes, of a scaled loss; clipped in place
        dict(_clip(3, 1001, 4099, "bf16", "f32", 2, True), name="clip-mixed-in-place"),
        # the activations of a short prompt in fp32, a width that ends inside a group of scales
        dict(_quantize(77, 2400, "f32", "f32"), name="quantize-prompt-f32"),
        # the activations of a block at 2048 x 2048 pixels with a short prompt
        dict(_quantize(333 + 128 * 128, 2432, "bf16", "bf16"), name="quantize-image-2048"),
        # a single token, such as the conditioning that gates and shifts are made from: the weight is read once
        dict(_linear(1, 4096, 11264, "bf16", "bf16", True), name="linear-single-token"),
        # a short prompt through a projection to an odd number of outputs, in fp32
        dict(_linear(333, 2432, 7297, "f32", "f32", True), name="linear-prompt-ragged"),
        # the feed-forward layer's first projection at 2048 x 2048 pixels with a short prompt
        dict(_linear(333 + 128 * 128, 2432, 9728, "bf16", "bf16", False), name="linear-image-2048"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw_once(rng):
    op = rng.choice(["residual", "clip", "quantize", "linear"])
    if op == "residual":
        dtype, stream = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        C = rng.choice([1536, 2432, 4096]) if rng.random() < 0.4 else _log_int(rng, 64, 8192)
        post = rng.choice(["", "", "rms", "layer"])
        return _residual(rng.choice([1, 1, 2, 4]), _log_int(rng, 1, 16896), C, dtype, stream, "f32" if dtype == "f32" else rng.choice(["bf16", "f32"]),
                         rng.choice(["layer", "rms"]), post, rng.choice(["item", "item", "shared", ""]), rng.random() < 0.5, rng.choice([1.0, 1.0, 0.75]), rng.random() < 0.6)
    if op == "clip":
        matrices = rng.choice(["f32", "bf16"])
        return _clip(rng.randint(1, 8), _log_int(rng, 64, 2432), _log_int(rng, 100, 6528), matrices, rng.choice([matrices, "f32"]), rng.choice([2, 2, 0]), rng.random() < 0.5)
    if op == "quantize":
        return _quantize(_log_int(rng, 1, 16896), 32 * _log_int(rng, 2, 256), *rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]))
    M = rng.choice([1, rng.randint(2, 64)]) if rng.random() < 0.3 else _log_int(rng, 64, 16896)
    return _linear(M, 32 * _log_int(rng, 8, 352), _log_int(rng, 64, 11264), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5)


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        for k in w:
            most[c["op"], k] = max(most.get((c["op"], k), 0), w[k])
    while True:
        c = _draw_once(rng)
        w = work(c)
        if all(w[k] <= most[c["op"], k] for k in w):
            return c


# ---- inputs -----------------------------------------------------------------------------------------------------------

class State:
    """What run() gets: the case's plain values and the tensors made for it."""

    def __init__(self, **have):
        self.__dict__.update(have)


TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}
EPS = 1e-6


def _normal(gen, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _activations(gen, shape, dtype):
    """Rows whose channels differ in size, a few of them by a lot."""
    C = shape[-1]
    size = torch.exp(0.5 * torch.randn(C, generator=gen, device="cuda"))
    size = torch.where(torch.rand(C, generator=gen, device="cuda") < 0.005, 20 * size, size)
    return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)


def _shapes(case):
    """(matrices, vectors) of the gradients of some blocks: attention projections with biases, norms, the feed-forward layer's matrices."""
    w, h = case["width"], case["hidden"]
    return [(w, w), (w, w), (w, w), (w, w), (h, w), (h, w), (w, h)] * case["blocks"], [(w,)] * (6 * case["blocks"])


def _flat(gen, shapes, dtype):
    """Gradients of these shapes in one buffer (some from odd places on), and the views of it."""
    ends = list(itertools.accumulate(math.prod(s) for s in shapes))
    flat = _normal(gen, (ends[-1],), scale=0.01)
    for at in range(0, ends[-1], 1 << 24):  # gradients of weights differ in size
        flat[at:at + (1 << 24)] *= torch.exp(1.5 * torch.randn(min(1 << 24, ends[-1] - at), generator=gen, device="cuda"))
    flat = flat.to(dtype)
    return flat, [flat[e - math.prod(s):e].view(s) for s, e in zip(shapes, ends)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    if op == "residual":
        B, N, C, t, ts, tw = case["B"], case["N"], case["C"], TYPES[case["dtype"]], TYPES[case["stream"]], TYPES[case["weight"]]
        x = _normal(gen, (B, N, C), scale=1.5)
        s = State(case=case, x=(x + 0.5 * torch.randn((C,), generator=gen, device="cuda")).to(ts), y=_activations(gen, (B, N, C), t))
        shape = (B, C) if case["per_item"] else (C,)
        s.weight = (_normal(gen, shape, scale=0.1) + (0 if case["per_item"] else 1)).to(tw)
        s.bias = _normal(gen, shape, tw, 0.1) if case["kind"] == "layer" else None
        s.gate = _normal(gen, (B, C) if case["gate"] == "item" else (C,), tw, 0.4) if case["gate"] else None
        s.post_weight = (1 + _normal(gen, (C,), scale=0.1)).to(tw) if case["post"] else None
        s.dr, s.dh = (_normal(gen, (B, N, C), ts), _normal(gen, (B, N, C), t)) if case["train"] else (None, None)
        return s
    if op == "clip":
        (g, matrices), (v, vectors) = (_flat(gen, shapes, TYPES[case[k]]) for shapes, k in zip(_shapes(case), ("matrices", "vectors")))
        # a loss that was scaled down by 4; the bound changes from pass to pass, so that a pass has work whatever the one before it left
        return State(case=case, g=g, v=v, grads=matrices + vectors, unscale=torch.full((), 4.0, device="cuda"), t=0)
    if op == "quantize":
        return State(case=case, x=_activations(gen, (case["M"], case["C"]), TYPES[case["dtype"]]))
    M, C, F = case["M"], case["C"], case["F"]
    w_codes, w_scales = _encode(_normal(gen, (F, C), scale=1 / math.sqrt(C)))
    return State(case=case, x=_activations(gen, (M, C), TYPES[case["dtype"]]), w_codes=w_codes, w_scales=w_scales,
                 bias=_normal(gen, (F,), scale=0.1) if case["bias"] else None)


# ---- plain forms --------------------------------------------------------------------------------------------------------

def _unit(x, kind):
    """(x without its size, 1 / size) of each row."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _unit_gradient(d, unit, r, kind):
    """The gradient of a row from that of its unit form."""
    d = d - unit * (d * unit).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - d.mean(-1, keepdim=True)  # (the unit rows have a mean of 0)
    return d * r


def _wide(v, case):
    return v.float()[:, None] if v.dim() == 2 else v.float()


def _plain_residual(s):
    case = s.case
    x, y = s.x.float(), s.y.float()
    w = _wide(s.weight, case)
    if case["per_item"]:
        w = 1 + w
    z = y
    if case["post"]:
        unit_y, r_y = _unit(y, case["post"])
        z = unit_y * s.post_weight.float()
    gate = _wide(s.gate, case) if case["gate"] else None
    r = case["scale"] * x + (z if gate is None else gate * z)
    unit, r_r = _unit(r, case["kind"])
    h = unit * w
    if s.bias is not None:
        h = h + _wide(s.bias, case)
    out = [r.to(s.x.dtype), h.to(s.y.dtype)]
    if not case["train"]:
        return out
    dr, dh = s.dr.float(), s.dh.float()

    def over_rows(d, like):
        # (sums over thousands of rows, in 64 bits)
        return d.double().sum((1,) if like.dim() == 2 else (0, 1)).to(like.dtype)
    d = dr + _unit_gradient(dh * w, unit, r_r, case["kind"])
    dz = d if gate is None else d * gate
    dy = _unit_gradient(dz * s.post_weight.float(), unit_y, r_y, case["post"]) if case["post"] else dz
    out += [(case["scale"] * d).to(s.x.dtype), dy.to(s.y.dtype), over_rows(dh * unit, s.weight)]
    if s.bias is not None:
        out.append(over_rows(dh, s.bias))
    if gate is not None:
        out.append(over_rows(d * z, s.gate))
    if case["post"]:
        out.append(over_rows(dz * unit_y, s.post_weight))
    return out


def _bound(s):
    """The bound of the norm in this pass, far below the norm of gradients as they are made and then in turn twice and half of what it was."""
    s.t += 1
    return 0.5 if s.t % 2 else 1.0


def _plain_clip(s):
    # (squares are added in 64 bits: there are up to 10^8 of them, of any size)
    if s.case["norm"] == 2:
        norm = torch.sqrt(s.g.double().square().sum() + s.v.double().square().sum())
    else:
        norm = torch.maximum(s.g.abs().max().double(), s.v.abs().max().double())
    if not s.case["in_place"]:
        return [norm.float(), torch.clamp(_bound(s) / norm, max=1.0).float()]
    norm = norm * s.unscale.double()
    scale = (torch.clamp(_bound(s) / norm, max=1.0) * s.unscale.double()).float()
    s.g.copy_((s.g.float() * scale).to(s.g.dtype))
    s.v.copy_((s.v.float() * scale).to(s.v.dtype))
    return [norm.float(), s.g, s.v]


# Numbers of 4 bits: a sign, two bits of exponent and one of fraction, 0, 0.5, 1, 1.5, 2, 3, 4, 6.  32 channels of a row share a scale, the power of two at which the largest of
# them lies between 4 and 8 (what is over 6 becomes 6), stored as its exponent + 127.  The first channel of a pair is in the low half of its byte; scales lie in
# groups of 8 (256 channels), [groups, rows, 8], 0 where there are no channels.

def _encode(x):
    rows, C = x.shape
    blocks = x.float().view(rows, C // 32, 32)
    exponent = torch.clamp(torch.frexp(blocks.abs().amax(2)).exponent - 3, min=-127)
    scaled = blocks.double() * torch.exp2(-exponent.double())[..., None]
    size = torch.clamp(scaled.abs(), max=6.0)
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(size, min=1.0))), max=2.0) - 1)
    size = torch.round(size / step) * step  # (halves to even: 2.5 is 2, 5 is 4)
    code = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8) + 8 * (scaled < 0).to(torch.uint8)
    code = code.view(rows, C)
    groups = -(-C // 256)
    scales = torch.zeros(rows, groups * 8, dtype=torch.uint8, device=x.device)
    scales[:, :C // 32] = (exponent + 127).to(torch.uint8)
    return code[:, 0::2] + 16 * code[:, 1::2], scales.view(rows, groups, 8).transpose(0, 1).contiguous()


def _decode(codes, scales):
    rows, C = codes.shape[0], 2 * codes.shape[1]
    code = torch.stack([codes & 15, codes >> 4], -1).view(rows, C // 32, 32)
    size = (code & 7).float()
    size = torch.where(size < 4, size / 2, torch.where(size < 6, size - 2, 2 * size - 8))
    scale = torch.exp2(scales.transpose(0, 1).reshape(rows, -1)[:, :C // 32].float() - 127)
    return (torch.where(code > 7, -size, size) * scale[..., None]).view(rows, C)


def _plain_quantize(s):
    return [_decode(*_encode(s.x)).to(TYPES[s.case["out"]])]


def _plain_linear(s):
    y = _decode(*_encode(s.x)) @ _decode(s.w_codes, s.w_scales).T
    if s.bias is not None:
        y = y + s.bias
    return [y.to(TYPES[s.case["out"]])]


# ---- this library ---------------------------------------------------------------------------------------------------------

def _own_residual(s):
    from paper_2412_16112_amd import clear_block as cb
    case = s.case
    how = dict(kind=case["kind"], post=case["post"] or None, weight_offset=1.0 if case["per_item"] else 0.0, residual_scale=case["scale"])
    if not case["train"]:
        return list(cb.residual_norm(s.x, s.y, s.gate, s.weight, s.bias, s.post_weight, eps=EPS, **how))
    r, h, stats = cb.residual_norm(s.x, s.y, s.gate, s.weight, s.bias, s.post_weight, eps=EPS, save_stats=True, **how)
    dx, dy, d_gate, d_weight, d_bias, d_post = cb.residual_norm_backward(s.dr, s.dh, s.x, s.y, s.gate, s.weight, s.bias, s.post_weight, stats, **how)
    return [r, h, dx, dy, d_weight] + [d for d in (d_bias, d_gate, d_post) if d is not None]


def _own_clip(s):
    from paper_2412_16112_amd import clear_block as cb
    kind = 2.0 if s.case["norm"] == 2 else math.inf
    if not s.case["in_place"]:
        return list(cb.grad_norm(s.grads, norm_type=kind, max_norm=_bound(s)))
    norm = cb.clip_grads(s.grads, _bound(s), norm_type=kind, grad_scale=s.unscale)
    return [norm, s.g, s.v]


def _own_quantize(s):
    from paper_2412_16112_amd import clear_block as cb
    return [cb.mx_dequantize(cb.mx_quantize(s.x), dtype=TYPES[s.case["out"]])]


def _own_linear(s):
    from paper_2412_16112_amd import clear_block as cb
    return [cb.mx_linear(s.x, cb.MX4(s.w_codes, s.w_scales), s.bias, dtype=TYPES[s.case["out"]])]


def run(state):
    op = state.case["op"]
    if own:
        return {"residual": _own_residual, "clip": _own_clip, "quantize": _own_quantize, "linear": _own_linear}[op](state)
    return {"residual": _plain_residual, "clip": _plain_clip, "quantize": _plain_quantize, "linear": _plain_linear}[op](state)


# ---- bytes and operations ---------------------------------------------------------------------------------------------------

FOUR_BITS = 0.5 + 1 / 32  # bytes of a number, with its share of the scale


def work(case):
    op = case["op"]
    if op == "residual":
        n, passes = case["B"] * case["N"] * case["C"], 2 if case["train"] else 1
        # x, y, r, h; the gradients of all four | the vectors; their gradients
        vectors = (case["B"] if case["per_item"] else 1) * (2 if case["kind"] == "layer" else 1) + {"item": case["B"], "shared": 1, "": 0}[case["gate"]] + (1 if case["post"] else 0)
        flops = (10 + (4 if case["post"] else 0)) + ((22 + (10 if case["post"] else 0)) if case["train"] else 0)
        return {"bytes": passes * (n * 2 * (SIZES[case["dtype"]] + SIZES[case["stream"]]) + vectors * case["C"] * SIZES[case["weight"]]), "flops": n * flops}
    if op == "clip":
        matrices, vectors = (sum(math.prod(s) for s in shapes) for shapes in _shapes(case))
        return {"bytes": (matrices * SIZES[case["matrices"]] + vectors * SIZES[case["vectors"]]) * (2 if case["in_place"] else 1),
                "flops": (matrices + vectors) * (3 if case["in_place"] else 2)}
    if op == "quantize":
        n = case["M"] * case["C"]
        return {"bytes": n * (SIZES[case["dtype"]] + 2 * FOUR_BITS + SIZES[case["out"]]), "flops": 4 * n}
    M, C, F = case["M"], case["C"], case["F"]
    return {"bytes": M * C * SIZES[case["dtype"]] + F * C * FOUR_BITS + M * F * SIZES[case["out"]] + (4 * F if case["bias"] else 0), "flops": 2 * M * C * F}


# ---- definitions in 64 bits -------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"residual": _exact_residual, "clip": _exact_clip, "quantize": _exact_quantize, "linear": _exact_linear}[case["op"]](case, s)


def _exact_norm(x, kind):
    if kind == "layer":
        var, mean = torch.var_mean(x, dim=2, correction=0, keepdim=True)
        return (x - mean) / (var + EPS).sqrt()
    return x / (x.square().mean(2, keepdim=True) + EPS).sqrt()


def _exact_residual(case, s):
    # the formula in 64 bits; its gradients by differentiating it
    leaf = {k: v.double().requires_grad_() for k, v in s.__dict__.items() if isinstance(v, torch.Tensor)}
    dr, dh = leaf.pop("dr", None), leaf.pop("dh", None)
    per_row = {k: v.unsqueeze(1) if v.dim() == 2 else v for k, v in leaf.items()}
    z = _exact_norm(leaf["y"], case["post"]) * leaf["post_weight"] if case["post"] else leaf["y"]
    r = leaf["x"] * case["scale"] + z * per_row.get("gate", 1.0)
    h = _exact_norm(r, case["kind"]) * (per_row["weight"] + (1.0 if case["per_item"] else 0.0)) + per_row.get("bias", 0.0)
    out = [r.detach(), h.detach()]
    if case["train"]:
        names = ["x", "y", "weight", "bias", "gate", "post_weight"]
        out += torch.autograd.grad([r, h], [leaf[k] for k in names if k in leaf], [dr.detach(), dh.detach()])
    return out


def _exact_clip(case, s):
    g, v = s.g.double(), s.v.double()
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t, 2 if case["norm"] == 2 else math.inf) for t in (g, v)]), 2 if case["norm"] == 2 else math.inf)
    unscale = 4.0 if case["in_place"] else 1.0
    norm = norm * unscale
    factor = 0.5 / norm if norm > 0.5 else torch.ones_like(norm)
    return [norm, g * (factor * unscale), v * (factor * unscale)] if case["in_place"] else [norm, factor]


def _exact_four_bits(x):
    """The nearest of the numbers of 4 bits times the block's scale; halfway the one whose last bit is 0."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    blocks = x.double().unflatten(1, (-1, 32))
    top = blocks.abs().amax(2, keepdim=True)
    power = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))  # (rounded up just below a power of two: put right)
    power = power - (torch.pow(2.0, power) > top).double()
    scale = torch.where(top > 0, torch.pow(2.0, torch.clamp(power - 2, min=-127.0)), torch.ones_like(top))
    size = (blocks.abs() / scale).clamp(max=6.0)
    below = torch.bucketize(size, grid, right=True) - 1
    above = (below + 1).clamp(max=7)
    to_below, to_above = size - grid[below], grid[above] - size
    upward = (to_above < to_below) | ((to_above == to_below) & (above % 2 == 0))
    return (torch.where(upward, grid[above], grid[below]) * scale * blocks.sign()).flatten(1)


def _exact_quantize(case, s):
    return [_exact_four_bits(s.x)]


def _exact_linear(case, s):
    nibbles = torch.stack([s.w_codes.to(torch.int64) % 16, s.w_codes.to(torch.int64) // 16], 2).flatten(1)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=nibbles.device)
    w = torch.cat([grid, -grid])[nibbles]
    power = s.w_scales.permute(1, 0, 2).flatten(1)[:, :case["C"] // 32].double() - 127
    w = w * torch.pow(2.0, power).repeat_interleave(32, 1)
    y = torch.matmul(_exact_four_bits(s.x), w.t().contiguous())
    return [y if s.bias is None else y + s.bias.double()]
