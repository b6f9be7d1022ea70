"""The AdamW step against its definition: in 64 bits, and bit for bit against the same fp32 operations in numpy (each rounded for itself), which is what makes
the codes of 8-bit states comparable at all - near a tie a last bit decides.

Tolerances.  Against 64 bits the new states carry 4 roundings (u = 2^-24 each) of their terms and the new parameter those of its step: 16 u of the terms' magnitudes."""
import numpy as np
import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.optim import AdamW

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
F = np.float32


def decode_m(code, scale):
    t = code.astype(F) * F(1 / 127)
    return t * np.abs(t) * np.repeat(scale, 256)[:code.size]


def decode_v(code, scale):
    t = code.astype(F) * F(1 / 255)
    t = t * t
    return t * t * np.repeat(scale, 256)[:code.size]


def encode(x, signed):
    """(codes, scales) of fp32 x by blocks of 256."""
    n = x.size
    blocks = np.zeros(-(-n // 256) * 256, dtype=F)
    blocks[:n] = x
    blocks = blocks.reshape(-1, 256)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        scale = np.abs(blocks).max(1)  # (NaN if there is one)
        fine = scale < np.inf
        share = np.where(scale[:, None] > 0, np.abs(blocks) / scale[:, None], F(0)).astype(F)
        root = np.sqrt(share) if signed else np.sqrt(np.sqrt(share))
        code = np.rint(root * F(127 if signed else 255))
    code = np.copysign(code, blocks) if signed else np.where(blocks > 0, np.maximum(code, 1), code)
    code = np.where(fine[:, None], code, 0)
    return code.reshape(-1)[:n].astype(np.int8 if signed else np.uint8), np.where(fine, scale, F(np.nan)).astype(F)


def step32(p, g, m, v, t, scale=None):
    """The formulas in fp32, one rounding an operation."""
    h = HYPER
    if scale is not None:
        g = g * F(scale)
    m = m * F(h["beta1"]) + g * F(1 - h["beta1"])
    v = v * F(h["beta2"]) + (g * g) * F(1 - h["beta2"])
    denominator = np.sqrt(v) * F(1 / np.sqrt(1 - h["beta2"] ** t)) + F(h["eps"])
    p = p * F(1 - h["lr"] * h["weight_decay"]) - (m / denominator) * F(h["lr"] / (1 - h["beta1"] ** t))
    return p, m, v


SIZES = [1, 3, 4, 255, 256, 257, 1000, 4096, 4097, 20001]


def tensors(dtype, seed=0, sizes=SIZES):
    g = torch.Generator().manual_seed(seed)
    p = [torch.randn(n, generator=g).to(dtype).cuda() for n in sizes]
    grads = [(torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g))).to(dtype).cuda() for n in sizes]
    return p, grads


def f32(t):
    return t.detach().float().cpu().numpy().reshape(-1)


@pytest.mark.parametrize("masters", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_states_of_32_bits(dtype, masters):
    params, grads = tensors(dtype)
    states = [cb.adamw_state(p) for p in params]
    kept = [p.float() + 1e-3 for p in params] if masters else None
    plain = [[f32(kept[i] if masters else params[i]), np.zeros(n, F), np.zeros(n, F)] for i, n in enumerate(SIZES)]
    for t in (1, 2, 3):
        before = [[a.astype(np.float64) for a in s] for s in plain]
        cb.adamw_step(params, grads, [s[0] for s in states], [s[1] for s in states], step=t, masters=kept, **HYPER)
        for i in range(len(SIZES)):
            plain[i] = list(step32(plain[i][0], f32(grads[i]), plain[i][1], plain[i][2], t))
            g = f32(grads[i]).astype(np.float64)
            p, m, v = before[i]
            m2, v2 = 0.9 * m + (1 - 0.9) * g, 0.99 * v + (1 - 0.99) * g * g
            step = 1e-2 / (1 - 0.9 ** t) * m2 / (np.sqrt(v2) / np.sqrt(1 - 0.99 ** t) + 1e-8)
            p2 = p * (1 - 1e-3) - step
            got = [f32(kept[i] if masters else params[i]), f32(states[i][0]), f32(states[i][1])]
            assert np.array_equal(got[1], plain[i][1]) and np.array_equal(got[2], plain[i][2])
            assert np.all(np.abs(got[1] - m2) <= 16 * U * (np.abs(m) + np.abs(g))) and np.all(np.abs(got[2] - v2) <= 16 * U * v2)
            if dtype == torch.float32 or masters:
                assert np.array_equal(got[0], plain[i][0])
                m_terms = (np.abs(m) + np.abs(g)) / np.maximum(np.abs(m2), 1e-300)  # (a moment of cancelled terms is less exact)
                assert np.all(np.abs(got[0] - p2) <= 16 * U * (np.abs(p) + np.abs(step) * (1 + m_terms)))
            rounded = torch.from_numpy(plain[i][0]).to(dtype)
            assert torch.equal(params[i].cpu(), rounded)
            if not masters:
                plain[i][0] = rounded.float().numpy()  # (the next step starts from what was stored)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_states_of_8_bits_bit_for_bit(dtype):
    params, grads = tensors(dtype, seed=4)
    states = [cb.adamw_state(p, 8) for p in params]
    plain = [[f32(p), np.zeros(p.numel(), np.int8), np.zeros(p.numel(), np.uint8), np.zeros(-(-p.numel() // 256), F), np.zeros(-(-p.numel() // 256), F)] for p in params]
    for t in (1, 2, 3, 4):
        grads = [g.roll(t) for g in grads]
        cb.adamw_step(params, grads, [s[0] for s in states], [s[1] for s in states], step=t, scales=[s[2] for s in states], **HYPER)
        for i in range(len(SIZES)):
            p, mc, vc, ms, vs = plain[i]
            p, m, v = step32(p, f32(grads[i]), decode_m(mc, ms), decode_v(vc, vs), t)
            (mc, ms), (vc, vs) = encode(m, True), encode(v, False)
            p = torch.from_numpy(p).to(dtype)
            plain[i] = [p.float().numpy(), mc, vc, ms, vs]
            m8, v8, (sm, sv) = states[i]
            assert torch.equal(params[i].cpu(), p)
            assert np.array_equal(m8.cpu().numpy(), mc) and np.array_equal(v8.cpu().numpy(), vc)
            assert np.array_equal(f32(sm), ms) and np.array_equal(f32(sv), vs)
            dm, dv = cb.adamw_decode(m8, sm, v8, sv)
            assert np.array_equal(f32(dm), decode_m(mc, ms)) and np.array_equal(f32(dv), decode_v(vc, vs))
            # half a step of the root: 1/254 of the top, so |m| is off by at most (2 sqrt(|m| top) + top/254) / 254; likewise v by its fourth root
            top = np.repeat(ms, 256)[:m.size].astype(np.float64)
            assert np.all(np.abs(f32(dm) - m.astype(np.float64)) <= (2 * np.sqrt(np.abs(m) * top) + top / 254) / 254 * 1.0001)
            assert np.all((f32(dv) > 0) == (v > 0))


def test_codes_at_the_edges():
    # a gradient of one size, of two sizes that differ by 10^12, of zeros; blocks that are not full
    for values in ([1.0] * 300, [1e6] + [1e-6] * 299, [0.0] * 300, [-5.0, 0.0, 1e-30] * 100):
        p, g = torch.zeros(300).cuda(), torch.tensor(values).cuda()
        m, v, scales = cb.adamw_state(p, 8)
        cb.adamw_step([p], [g], [m], [v], step=1, scales=[scales], **HYPER)
        _, wm, wv = step32(np.zeros(300, F), f32(g), np.zeros(300, F), np.zeros(300, F), 1)
        for got, scale, want in ((m, scales[0], encode(wm, True)), (v, scales[1], encode(wv, False))):
            assert np.array_equal(got.cpu().numpy(), want[0]) and np.array_equal(f32(scale), want[1])


def test_not_finite_gradients():
    p, g = torch.ones(1000).cuda(), torch.ones(1000).cuda()
    g[300], g[700] = float("nan"), float("inf")
    q, m32, v32 = p.clone(), torch.zeros(1000).cuda(), torch.zeros(1000).cuda()
    cb.adamw_step([q], [g], [m32], [v32], step=1, **HYPER)
    bad = torch.isnan(q)
    assert bool(bad[300]) and bool(bad[700]) and int(bad.sum()) == 2  # (inf / inf)
    m, v, scales = cb.adamw_state(p, 8)
    cb.adamw_step([p], [g], [m], [v], step=1, scales=[scales], **HYPER)
    assert torch.equal(torch.isnan(p), bad) and torch.equal(p[~bad], q[~bad])
    dm, dv = cb.adamw_decode(m, scales[0], v, scales[1])
    blocks = torch.zeros(1000, dtype=torch.bool, device="cuda")
    blocks[256:768] = True  # the two blocks that hold them
    assert torch.equal(torch.isnan(dm), blocks) and torch.equal(torch.isnan(dv), blocks)
    assert not bool(m[256:768].any()) and not bool(v[256:768].any())


def test_many_tensors_skipped_ones_and_scaled_gradients():
    sizes = [(i * 37) % 700 for i in range(130)]  # three launches' worth, empty ones among them
    params, grads = tensors(torch.float32, seed=8, sizes=sizes)
    start = [p.clone() for p in params]
    states = [cb.adamw_state(p) for p in params]
    some = [None if i % 5 == 2 else g for i, g in enumerate(grads)]
    clip = torch.tensor(0.25, device="cuda")
    cb.adamw_step(params, some, [s[0] for s in states], [s[1] for s in states], step=1, grad_scale=clip, **HYPER)
    for i, n in enumerate(sizes):
        if i % 5 == 2:
            assert torch.equal(params[i], start[i]) and not bool(states[i][0].any())
        else:
            p, m, v = step32(f32(start[i]), f32(grads[i]), np.zeros(n, F), np.zeros(n, F), 1, scale=0.25)
            assert np.array_equal(f32(params[i]), p) and np.array_equal(f32(states[i][0]), m) and np.array_equal(f32(states[i][1]), v)
    cb.adamw_step([], [], [], [], step=1, **HYPER)


def test_unaligned_tensors_leave_their_neighbours_alone():
    for dtype in (torch.float32, torch.bfloat16):
        for bits in (32, 8):
            n = 777
            room = lambda t: torch.full((n + 2,), 3, dtype=t, device="cuda")
            p, g = room(dtype), room(dtype)
            m, v = (room(torch.float32), room(torch.float32)) if bits == 32 else (room(torch.int8), room(torch.uint8))
            inner = [t[1:-1] for t in (p, g, m, v)]
            a, b = torch.randn(n, device="cuda").to(dtype), torch.randn(n, device="cuda").to(dtype)
            inner[0].copy_(a), inner[1].copy_(b), inner[2].zero_(), inner[3].zero_()
            zero = lambda: tuple(torch.zeros(4, device="cuda") for _ in range(2))
            s1, s2 = zero(), zero()
            cb.adamw_step([inner[0]], [inner[1]], [inner[2]], [inner[3]], step=2, scales=[s1] if bits == 8 else None, **HYPER)
            fresh = cb.adamw_state(a, bits)
            cb.adamw_step([a], [b], [fresh[0]], [fresh[1]], step=2, scales=[s2] if bits == 8 else None, **HYPER)
            assert torch.equal(inner[0], a) and torch.equal(inner[2], fresh[0]) and torch.equal(inner[3], fresh[1]) and torch.equal(s1[0], s2[0])
            assert all(float(t[0]) == 3 and float(t[-1]) == 3 for t in (p, g, m, v))


def test_optimizer():
    for bits in (32, 8):
        params, grads = tensors(torch.bfloat16, seed=11)
        same = [p.clone() for p in params]
        opt = AdamW(params, state_bits=bits, masters=True, **HYPER)
        states, masters = [cb.adamw_state(p, bits) for p in same], [p.float() for p in same]
        for t in (1, 2):
            for p, g in zip(params, grads):
                p.grad = g.clone()
            opt.step()
            cb.adamw_step(same, grads, [s[0] for s in states], [s[1] for s in states], step=t, masters=masters,
                          scales=[s[2] for s in states] if bits == 8 else None, **HYPER)
        opt.zero_grad()
        assert all(p.grad is None for p in params)
        assert all(torch.equal(a, b) for a, b in zip(params, same)) and all(torch.equal(a, b) for a, b in zip(opt.masters, masters))
        mixed = AdamW([torch.ones(5, device="cuda"), torch.ones(5, device="cuda", dtype=torch.bfloat16)], lr=0.1, state_bits=bits)  # (a step that bf16 shows)
        mixed.step([torch.ones(5, device="cuda"), torch.ones(5, device="cuda", dtype=torch.bfloat16)])
        assert float(mixed.params[0][0]) < 1 and float(mixed.params[1][0]) < 1


def test_on_another_stream_and_in_a_graph():
    params, grads = tensors(torch.float32, seed=2)
    states = [cb.adamw_state(p, 8) for p in params]
    work = lambda ps, ss: cb.adamw_step(ps, grads, [s[0] for s in ss], [s[1] for s in ss], step=5, scales=[s[2] for s in ss], **HYPER)
    other = [p.clone() for p in params]
    others = [cb.adamw_state(p, 8) for p in other]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(params, states)
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(params, states)  # (recorded, not run)
    work(other, others)
    for turn in range(3):
        assert all(torch.equal(a, b) for a, b in zip(params, other)) and all(torch.equal(a[0], b[0]) for a, b in zip(states, others)), turn
        graph.replay()
        work(other, others)
        torch.cuda.synchronize()


def test_refusals():
    p, g = torch.ones(10).cuda(), torch.ones(10).cuda()
    m, v = cb.adamw_state(p)
    m8, v8, scales = cb.adamw_state(p, 8)
    bf = torch.bfloat16
    for bad in [lambda: cb.adamw_step([p], [g], [m], [v], step=0, **HYPER), lambda: cb.adamw_step([p], [g.to(bf)], [m], [v], step=1, **HYPER),
                lambda: cb.adamw_step([p], [g], [m8], [v8], step=1, **HYPER), lambda: cb.adamw_step([p], [g], [m], [v], step=1, scales=[scales], **HYPER),
                lambda: cb.adamw_step([p, p.to(bf)], [g, g.to(bf)], [m, m], [v, v], step=1, **HYPER), lambda: cb.adamw_step([p], [g], [m], [v[:9]], step=1, **HYPER),
                lambda: cb.adamw_step([p], [g, g], [m], [v], step=1, **HYPER), lambda: cb.adamw_step([p], [g], [m], [v], step=1, **dict(HYPER, beta1=1.0)),
                lambda: cb.adamw_step([p], [g], [m], [v], step=1, **dict(HYPER, lr=float("nan"))), lambda: cb.adamw_step([p], [g], [m], [v], step=1, masters=[p.to(bf)], **HYPER),
                lambda: cb.adamw_step([p.view(2, 5).t()], [g.view(2, 5).t()], [m], [v], step=1, **HYPER), lambda: cb.adamw_step([p.half()], [g.half()], [m], [v], step=1, **HYPER),
                lambda: cb.adamw_step([p], [g], [m], [v], step=1, grad_scale=torch.ones(1), **HYPER), lambda: cb.adamw_state(p, 16),
                lambda: cb.adamw_decode(m, scales[0], v8, scales[1]), lambda: AdamW([torch.ones(3)])]:
        with pytest.raises(ca.ClearAttnError):
            bad()
    assert bool((p == 1).all())
