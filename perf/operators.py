"""Timings of the operators that stand around the local attention in a transformer block and its training step: rotary
positions, layer norm, the gated feed-forward projection and the AdamW step, each in its plain form (elementary torch
operations in 32 bits) and through this library.

`listed()` names twelve cases, `draw(rng)` gives another of the same ranges, `prepare` makes what a program holds before the
call, `run` is one pass as such a program calls it, `work` the bytes and operations that a pass cannot do without, `exact` the
outputs from the operators' definitions in 64 bits.

A case's "op" is one of
  rotary  turns the queries and keys of a block by their tokens' angles (or back, for the gradient);
  norm    layer norm with one weight for all rows or one for each batch item; with "train" its backward pass too;
  gated   act(x Wg^T) * (x Wu^T); with "train" its backward pass too;
  adamw   one optimizer step over the parameters of some blocks, states in 32 or in 8 bits."""
import itertools
import math

import torch

own = False

BLOCK = 256  # elements that share a scale where AdamW's states are held in 8 bits


# ---- cases ------------------------------------------------------------------------------------------------------------

def _rotary(B, Hq, Hk, N, d, rot, dtype, interleaved, axes, gridW=0, n_text=0, far=0, inverse=False, token_major=False):
    return dict(op="rotary", B=B, Hq=Hq, Hk=Hk, N=N, d=d, rot=rot, dtype=dtype, interleaved=interleaved, axes=axes, gridW=gridW,
                n_text=n_text, far=far, inverse=inverse, token_major=token_major)


def _norm(B, N, C, dtype, weight, per_item, train, plus_one=False):
    return dict(op="norm", B=B, N=N, C=C, dtype=dtype, weight=weight, per_item=per_item, train=train, plus_one=plus_one)


def _gated(M, C, F, act, train):
    return dict(op="gated", M=M, C=C, F=F, act=act, train=train)


def _adamw(blocks, width, hidden, dtype, bits, master, step):
    return dict(op="adamw", blocks=blocks, width=width, hidden=hidden, dtype=dtype, bits=bits, master=master, step=step)


def listed():
    return [
        # one token of each of 16 text sequences at positions far into a long context: grouped heads, half layout
        dict(_rotary(16, 32, 8, 1, 128, 128, "bf16", False, 1, far=100000), name="rotary-single-tokens"),
        # queries and keys of a 2048 x 2048 pixel image and its prompt, as a projection stores them; three position axes
        dict(_rotary(1, 24, 24, 512 + 128 * 128, 128, 128, "bf16", True, 3, gridW=128, n_text=512, token_major=True), name="rotary-image-2048"),
        # the gradient's way back at a ragged image and prompt, two in the batch, half of each head turned, fp32
        dict(_rotary(2, 38, 38, 77 + 48 * 85, 64, 32, "f32", False, 2, gridW=85, n_text=77, inverse=True), name="rotary-gradient-ragged"),
        # a short prompt's rows: a fraction of the chip, launch bound
        dict(_norm(1, 77, 2432, "bf16", "bf16", False, False), name="norm-prompt"),
        # a training step's norm at 1024 x 1024 pixels, scale and shift from the conditioning of each batch item
        dict(_norm(2, 512 + 64 * 64, 2432, "bf16", "bf16", True, True, plus_one=True), name="norm-adaptive-train"),
        # an odd width in fp32, one weight for all rows, at 2048 x 2048 pixels with a short prompt
        dict(_norm(1, 333 + 128 * 128, 1111, "f32", "f32", False, True), name="norm-odd-f32-train"),
        # a single token through a text model's layer: both weights are read once
        dict(_gated(1, 4096, 11264, "silu", False), name="gated-single-token"),
        # a training step at 1024 x 1024 pixels
        dict(_gated(512 + 64 * 64, 2432, 6528, "silu", True), name="gated-train-1024"),
        # inference at 2048 x 2048 pixels with a short prompt, no row count a multiple of a tile
        dict(_gated(333 + 128 * 128, 2432, 9728, "gelu_tanh", False), name="gated-image-2048"),
        # the norms and adapters of a small model: many tensors of a few hundred elements, launch bound
        dict(_adamw(2, 96, 250, "f32", 32, False, 7), name="adamw-small"),
        # the weights of four blocks in bf16 with fp32 masters and fp32 states
        dict(_adamw(4, 1536, 4096, "bf16", 32, True, 1000), name="adamw-bf16-master"),
        # the same in fp32 with states of 8 bits; the states are read out as well, as for a checkpoint
        dict(_adamw(4, 1536, 4096, "f32", 8, False, 1000), name="adamw-8bit"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw_once(rng):
    op = rng.choice(["rotary", "norm", "gated", "adamw"])
    if op == "rotary":
        d = rng.choice([64, 128, 2 * rng.randint(16, 128)])
        rot = d if rng.random() < 0.5 else 2 * rng.randint(4, d // 2)
        Hq = _log_int(rng, 1, 40)
        Hk = Hq if rng.random() < 0.5 else rng.choice([h for h in range(1, Hq + 1) if Hq % h == 0])
        axes = rng.choice([1, 2, 3])
        dtype, interleaved = rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5
        if axes == 1:
            B, N = _log_int(rng, 1, 64), _log_int(rng, 1, 8192)
            N = 1 if rng.random() < 0.3 else N
            return _rotary(B, Hq, Hk, N, d, rot, dtype, interleaved, 1, far=_log_int(rng, 1, 1000000), inverse=rng.random() < 0.3, token_major=rng.random() < 0.5)
        gridH, gridW, n_text = _log_int(rng, 12, 128), _log_int(rng, 12, 128), rng.choice([0, 77, 333, 512])
        return _rotary(rng.choice([1, 2, 4]), Hq, Hk, n_text + gridH * gridW, d, rot, dtype, interleaved, axes, gridW=gridW, n_text=n_text,
                       inverse=rng.random() < 0.3, token_major=rng.random() < 0.5)
    if op == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        C = rng.choice([1536, 2432, 4096]) if rng.random() < 0.4 else _log_int(rng, 64, 8192)
        return _norm(rng.choice([1, 1, 2, 4]), _log_int(rng, 1, 16896), C, dtype, "f32" if dtype == "f32" else rng.choice(["bf16", "f32"]),
                     rng.random() < 0.4, rng.random() < 0.6, rng.random() < 0.4)
    if op == "gated":
        M = rng.choice([1, rng.randint(2, 64)]) if rng.random() < 0.3 else _log_int(rng, 64, 16896)
        return _gated(M, 8 * _log_int(rng, 32, 512), 8 * _log_int(rng, 64, 1408), rng.choice(["silu", "gelu_tanh"]), M > 64 and rng.random() < 0.5)
    dtype = rng.choice(["f32", "bf16"])
    return _adamw(rng.randint(1, 8), _log_int(rng, 64, 2432), _log_int(rng, 100, 6528), dtype, rng.choice([32, 32, 8]), dtype == "bf16" and rng.random() < 0.5,
                  _log_int(rng, 1, 10000))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        for k in w:
            most[c["op"], k] = max(most.get((c["op"], k), 0), w[k])
    while True:
        c = _draw_once(rng)
        w = work(c)
        if all(w[k] <= most[c["op"], k] for k in w) and all(c.get(k) != 3072 for k in ("C", "F", "width", "hidden")):
            return c


def _shapes(case):
    """Parameters of the blocks of a model: attention projections with biases, norms, the feed-forward layer's matrices."""
    w, h = case["width"], case["hidden"]
    block = [(w, w), (w,), (w, w), (w,), (w, w), (w,), (w, w), (w,), (w,), (w,), (h, w), (h, w), (w, h)]
    return block * case["blocks"]


def _padded(shapes):
    return [-(-math.prod(s) // BLOCK) * BLOCK for s in shapes]


# ---- inputs -----------------------------------------------------------------------------------------------------------

class State:
    """What run() gets: the case's plain values and the tensors made for it."""

    def __init__(self, **have):
        self.__dict__.update(have)


TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(gen, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _frequencies(case):
    """Radians a position, [axes, rot / 2] in 64 bits: each axis acts on a share of the pairs; one axis of a long context has
    its slow pairs stretched by 8."""
    half, axes = case["rot"] // 2, case["axes"]
    f = torch.zeros(axes, half, dtype=torch.float64)
    if axes == 1:
        f[0] = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        f[0] = torch.where(f[0] * 8192 < 2 * math.pi, f[0] / 8, f[0])
        return f
    first = half // 8 if axes == 3 else 0
    ends = ([first] if axes == 3 else []) + [first + (half - first) // 2, half]
    start = 0
    for a, end in enumerate(ends):
        n = end - start
        f[a, start:end] = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))
        start = end
    return f


def _positions(case, gen):
    """[axes, B, N], int64."""
    B, N, axes = case["B"], case["N"], case["axes"]
    if axes == 1:
        start = torch.randint(0, case["far"], (B, 1), generator=gen, device="cuda")
        return (start + torch.arange(N, device="cuda"))[None]
    image = torch.arange(N - case["n_text"], device="cuda")
    row, col = image // case["gridW"], image % case["gridW"]
    text = torch.zeros(case["n_text"], dtype=torch.int64, device="cuda")
    per_axis = [torch.cat([text, row]), torch.cat([text, col])]
    if axes == 3:
        per_axis = [torch.zeros(N, dtype=torch.int64, device="cuda")] + per_axis
    return torch.stack(per_axis)[:, None, :].expand(axes, B, N).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    if op == "rotary":
        t = TYPES[case["dtype"]]

        def heads(H):
            if case["token_major"]:
                return _normal(gen, (case["B"], case["N"], H, case["d"]), t).transpose(1, 2)
            return _normal(gen, (case["B"], H, case["N"], case["d"]), t)
        return State(case=case, q=heads(case["Hq"]), k=heads(case["Hk"]), positions=_positions(case, gen), freqs=_frequencies(case).cuda())
    if op == "norm":
        B, N, C, t, tw = case["B"], case["N"], case["C"], TYPES[case["dtype"]], TYPES[case["weight"]]
        shape = (B, C) if case["per_item"] else (C,)
        x = _normal(gen, (B, N, C), scale=1.5)
        x = (x + 0.5 * torch.randn((C,), generator=gen, device="cuda")).to(t)
        w = _normal(gen, shape, scale=0.1)
        return State(case=case, x=x, w=(w if case["plus_one"] else 1 + w).to(tw), b=_normal(gen, shape, tw, 0.1), dy=_normal(gen, (B, N, C), t) if case["train"] else None)
    if op == "gated":
        M, C, F, t = case["M"], case["C"], case["F"], torch.bfloat16
        return State(case=case, x=_normal(gen, (M, C), t), wg=_normal(gen, (F, C), t, 1.5 / math.sqrt(C)), wu=_normal(gen, (F, C), t, 1 / math.sqrt(C)),
                     dh=_normal(gen, (M, F), t) if case["train"] else None)
    # adamw: the tensors of each kind lie in one buffer, each from a multiple of BLOCK elements on
    t, shapes = TYPES[case["dtype"]], _shapes(case)
    padded = _padded(shapes)
    ends = list(itertools.accumulate(padded))
    starts, total = [0] + ends[:-1], ends[-1]
    real = torch.zeros(total, dtype=torch.float32, device="cuda")
    for s, at in zip(shapes, starts):
        real[at:at + math.prod(s)] = 1
    spread = torch.exp(1.5 * torch.randn(total, generator=gen, device="cuda"))  # gradients of weights differ in size
    p = torch.randn(total, generator=gen, device="cuda") * 0.03 * real
    g = torch.randn(total, generator=gen, device="cuda") * 0.01 * spread * real
    m = torch.randn(total, generator=gen, device="cuda") * 0.003 * spread * real
    v = (0.01 * spread) ** 2 * (0.5 + torch.rand(total, generator=gen, device="cuda")) * real

    def views(flat, each=1):
        return [flat[a // each:a // each + -(-math.prod(s) // each)].view(s if each == 1 else -1) for s, a in zip(shapes, starts)]
    s = State(case=case, t=case["step"], p=p.to(t), g=g.to(t), master=p if case["master"] else None)
    if case["bits"] == 8:
        (s.m, s.m_scale), (s.v, s.v_scale) = _quantize_m(m), _quantize_v(v)
        s.scales = list(zip(views(s.m_scale, BLOCK), views(s.v_scale, BLOCK)))
    else:
        s.m, s.v = m, v
    s.params, s.grads, s.exp_avgs, s.exp_avg_sqs = views(s.p), views(s.g), views(s.m), views(s.v)
    s.masters = views(s.master) if case["master"] else None
    return s


HYPER = dict(lr=3e-4, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.01)


# ---- plain forms --------------------------------------------------------------------------------------------------------

def _turned(x, cos, sin, case):
    half, rot = case["rot"] // 2, case["rot"]
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _plain_rotary(s):
    # (frequencies come in 64 bits, and so are the angles: at position 10^5 an angle in 32 bits is off by 10^-2)
    angle = (s.positions.double()[..., None] * s.freqs[:, None, None, :]).sum(0)[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if s.case["inverse"]:
        sin = -sin
    return [_turned(s.q, cos, sin, s.case), _turned(s.k, cos, sin, s.case)]


EPS = 1e-6


def _plain_norm(s):
    case = s.case
    x, w, b = s.x.float(), s.w.float(), s.b.float()
    if case["plus_one"]:
        w = 1 + w
    if case["per_item"]:
        w, b = w[:, None], b[:, None]
    centred = x - x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    xhat = centred * r
    y = (xhat * w + b).to(s.x.dtype)
    if not case["train"]:
        return [y]
    dy = s.dy.float()
    dyw = dy * w
    dx = r * (dyw - dyw.mean(-1, keepdim=True) - xhat * (dyw * xhat).mean(-1, keepdim=True))
    rows = (1,) if case["per_item"] else (0, 1)
    return [y, dx.to(s.x.dtype), (dy * xhat).sum(rows).to(s.w.dtype), dy.sum(rows).to(s.b.dtype)]


def _act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_gated(s):
    x, wg, wu = s.x.float(), s.wg.float(), s.wu.float()
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(g, s.case["act"])
    h = (a * u).to(s.x.dtype)
    if not s.case["train"]:
        return [h]
    dh = s.dh.float()
    dg, du = dh * u * da, dh * a
    return [h, (dg @ wg + du @ wu).to(s.x.dtype), (dg.T @ x).to(s.wg.dtype), (du.T @ x).to(s.wu.dtype)]


# States of 8 bits: blocks of 256 elements share a scale, the largest magnitude in the block.  The first moment is stored as
# the root of its share of the scale (a sign and 127 steps), the second, which is never negative, as the fourth root (255
# steps, and never 0 for a value that is not): small values keep their relative precision.

def _quantize_m(m):
    blocks = m.view(-1, BLOCK)
    scale = blocks.abs().amax(1)
    share = torch.where(scale[:, None] > 0, blocks.abs() / scale[:, None], torch.zeros_like(blocks))
    code = torch.round(torch.sqrt(share) * 127) * torch.sign(blocks)
    return code.to(torch.int8).view(-1), scale


def _quantize_v(v):
    blocks = v.view(-1, BLOCK)
    scale = blocks.amax(1)
    share = torch.where(scale[:, None] > 0, blocks / scale[:, None], torch.zeros_like(blocks))
    code = torch.round(torch.sqrt(torch.sqrt(share)) * 255)
    code = torch.where(blocks > 0, torch.clamp(code, min=1), code)
    return code.to(torch.uint8).view(-1), scale


def _decode_m(code, scale):
    t = code.float().view(-1, BLOCK) * (1 / 127)
    return (t * t.abs() * scale[:, None]).view(-1)


def _decode_v(code, scale):
    t = code.float().view(-1, BLOCK) * (1 / 255)
    t = t * t
    return (t * t * scale[:, None]).view(-1)


def _plain_adamw(s):
    eight, h = s.case["bits"] == 8, HYPER
    p, g = (s.p if s.master is None else s.master).float(), s.g.float()
    m, v = (_decode_m(s.m, s.m_scale), _decode_v(s.v, s.v_scale)) if eight else (s.m, s.v)
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1 - h["beta2"])
    denominator = torch.sqrt(v) * (1 / math.sqrt(1 - h["beta2"] ** s.t)) + h["eps"]
    p = p * (1 - h["lr"] * h["weight_decay"]) - (m / denominator) * (h["lr"] / (1 - h["beta1"] ** s.t))
    s.p.copy_(p.to(s.p.dtype))
    if s.master is not None:
        s.master.copy_(p)
    if eight:
        for kept, new in zip((s.m, s.m_scale, s.v, s.v_scale), _quantize_m(m) + _quantize_v(v)):
            kept.copy_(new)
        return [s.p, _decode_m(s.m, s.m_scale), _decode_v(s.v, s.v_scale)]
    s.m.copy_(m)
    s.v.copy_(v)
    return [s.p, m, v] + ([s.master] if s.master is not None else [])


# ---- this library ---------------------------------------------------------------------------------------------------------

def _own_rotary(s):
    from paper_2412_16112_amd import clear_block as cb
    return list(cb.rotary(s.q, s.k, s.positions, s.freqs, interleaved=s.case["interleaved"], inverse=s.case["inverse"]))


def _own_norm(s):
    from paper_2412_16112_amd import clear_block as cb
    offset = 1.0 if s.case["plus_one"] else 0.0
    if not s.case["train"]:
        return [cb.layer_norm(s.x, s.w, s.b, eps=EPS, weight_offset=offset)]
    y, stats = cb.layer_norm(s.x, s.w, s.b, eps=EPS, weight_offset=offset, save_stats=True)
    return [y, *cb.layer_norm_backward(s.dy, s.x, s.w, s.b, stats, weight_offset=offset)]


def _own_gated(s):
    from paper_2412_16112_amd import clear_block as cb
    if not s.case["train"]:
        return [cb.gated_ff(s.x, s.wg, s.wu, activation=s.case["act"])]
    h, pre = cb.gated_ff(s.x, s.wg, s.wu, activation=s.case["act"], save_pre=True)
    return [h, *cb.gated_ff_backward(s.dh, s.x, s.wg, s.wu, pre, activation=s.case["act"])]


def _own_adamw(s):
    from paper_2412_16112_amd import clear_block as cb
    eight = s.case["bits"] == 8
    cb.adamw_step(s.params, s.grads, s.exp_avgs, s.exp_avg_sqs, step=s.t, masters=s.masters, scales=s.scales if eight else None, **HYPER)
    if eight:
        return [s.p, *cb.adamw_decode(s.m, s.m_scale, s.v, s.v_scale)]
    return [s.p, s.m, s.v] + ([s.master] if s.master is not None else [])


def run(state):
    op = state.case["op"]
    if op == "adamw":
        state.t += 1
    if own:
        return {"rotary": _own_rotary, "norm": _own_norm, "gated": _own_gated, "adamw": _own_adamw}[op](state)
    return {"rotary": _plain_rotary, "norm": _plain_norm, "gated": _plain_gated, "adamw": _plain_adamw}[op](state)


# ---- bytes and operations ---------------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    size = {"bf16": 2, "f32": 4}
    if op == "rotary":
        tokens = case["B"] * case["N"]
        heads = case["Hq"] + case["Hk"]
        return {"bytes": tokens * heads * case["d"] * size[case["dtype"]] * 2 + 8 * tokens * case["axes"] + 8 * case["axes"] * case["rot"] // 2,
                "flops": tokens * heads * case["rot"] * 3}
    if op == "norm":
        rows, sets, C = case["B"] * case["N"], case["B"] if case["per_item"] else 1, case["C"]
        passes, per = (4, 2) if case["train"] else (2, 1)  # x and y; dy and dx | weight and bias; their gradients
        return {"bytes": rows * C * size[case["dtype"]] * passes + sets * C * size[case["weight"]] * 2 * per, "flops": rows * C * (19 if case["train"] else 8)}
    if op == "gated":
        M, C, F = case["M"], case["C"], case["F"]
        once = 2 * (M * C + 2 * F * C + M * F)  # x, both weights, the result; as much again for the gradients
        return {"bytes": once * (2 if case["train"] else 1), "flops": 4 * M * C * F * (3 if case["train"] else 1)}
    n = sum(math.prod(s) for s in _shapes(case))
    each = 3 * size[case["dtype"]] + (8 if case["master"] else 0)  # parameter read and written, gradient read; master
    each += 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8       # both states read and written; in 8 bits also read out
    return {"bytes": n * each, "flops": n * (14 if case["bits"] == 32 else 30)}


# ---- definitions in 64 bits -------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "norm": _exact_norm, "gated": _exact_gated, "adamw": _exact_adamw}[case["op"]](case, s)


def _exact_rotary(case, s):
    angle = torch.zeros(case["B"], case["N"], case["rot"] // 2, dtype=torch.float64, device="cuda")
    for a in range(case["axes"]):
        angle += s.positions[a].double().unsqueeze(-1) * s.freqs[a]
    turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle).unsqueeze(1)  # e^(i angle)
    out = []
    for x in (s.q, s.k):
        y = x.double().clone(memory_format=torch.contiguous_format)
        head = y[..., :case["rot"]]
        pairs = head.unflatten(-1, (-1, 2)) if case["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y[..., :case["rot"]] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        out.append(y)
    return out


def _exact_norm(case, s):
    x, w, b = s.x.double(), s.w.double() + (1.0 if case["plus_one"] else 0.0), s.b.double()
    if case["per_item"]:
        w, b = w.unsqueeze(1), b.unsqueeze(1)
    var, mean = torch.var_mean(x, dim=2, correction=0, keepdim=True)
    z = (x - mean) / (var + EPS).sqrt()
    out = [z * w + b]
    if case["train"]:
        # Jacobian of z in x: (I - 1 1^T / C - z z^T / C) / sigma, applied to dz = dy w
        dy, C = s.dy.double(), case["C"]
        dz = dy * w
        dx = (dz - (dz.sum(2, keepdim=True) + z * (dz * z).sum(2, keepdim=True)) / C) / (var + EPS).sqrt()
        dw, db = (dy * z).sum(1), dy.sum(1)
        out += [dx, dw, db] if case["per_item"] else [dx, dw.sum(0), db.sum(0)]
    return out


def _exact_gated(case, s):
    x, wg, wu = s.x.double(), s.wg.double(), s.wu.double()
    g, u = torch.matmul(x, wg.t().contiguous()), torch.matmul(x, wu.t().contiguous())
    if case["act"] == "silu":
        q = torch.sigmoid(g)
        a, slope = g * q, q + g * q * (1 - q)
    else:
        k, cubic = math.sqrt(2 / math.pi), 0.044715
        q = torch.sigmoid(2 * k * (g + cubic * g ** 3))  # (1 + tanh z) / 2 = 1 / (1 + e^(-2 z))
        a, slope = g * q, q + g * q * (1 - q) * 2 * k * (1 + 3 * cubic * g ** 2)
    out = [a * u]
    if case["train"]:
        dh = s.dh.double()
        du, dg = dh * a, dh * u * slope
        out += [torch.matmul(dg, wg) + torch.matmul(du, wu), torch.matmul(dg.t().contiguous(), x), torch.matmul(du.t().contiguous(), x)]
    return out


def _exact_adamw(case, s):
    t, h = case["step"] + 1, HYPER
    p, g = (s.master if case["master"] else s.p).double(), s.g.double()
    if case["bits"] == 8:
        m = (s.m.double() / 127).abs().square() * s.m.double().sign() * s.m_scale.double().repeat_interleave(BLOCK)
        v = (s.v.double() / 255) ** 4 * s.v_scale.double().repeat_interleave(BLOCK)
    else:
        m, v = s.m.double(), s.v.double()
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
    step = (m / (1 - h["beta1"] ** t)) / ((v / (1 - h["beta2"] ** t)).sqrt() + h["eps"])
    p = p - h["lr"] * h["weight_decay"] * p - h["lr"] * step
    if case["bits"] == 8:
        # the stored values: the nearest of the steps of the block's scale
        top_m = m.view(-1, BLOCK).abs().amax(1).clamp_min(1e-300).repeat_interleave(BLOCK)
        top_v = v.view(-1, BLOCK).amax(1).clamp_min(1e-300).repeat_interleave(BLOCK)
        m = (((m.abs() / top_m) ** 0.5 * 127).round() / 127) ** 2 * m.sign() * top_m
        code = ((v / top_v) ** 0.25 * 255).round()
        v = (torch.where(v > 0, code.clamp_min(1), code) / 255) ** 4 * top_v
    return [p, m, v] + ([p] if case["master"] else [])
