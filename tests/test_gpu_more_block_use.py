"""The gated residual with its norms, the gradients' norm and the products of 4-bit operands as a program uses them: gradients by autograd against differences, other streams, captured graphs, tensors whose offsets
pass 32 bits, and runs of them together."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.optim import AdamW
from tests import more_block_util as ref
from tests.test_gpu_block_mx import operands, product
from tests.test_gpu_block_streams import on

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def drawer(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s, k=1.0: k * torch.randn(*s, generator=g, device="cuda")


# ---- gradients

@pytest.mark.parametrize("kind,post", [("layer", None), ("rms", "layer"), ("layer", "rms")])
def test_gradients_against_differences(kind, post):
    """A change of the inputs by e d changes <r, u> + <h, v> by 2 e <gradient, d> between -e and +e: the third-order term is taken off by a second e (Richardson); what is left of fp32's rounding in r and h, 2^-24 of
    their sizes at 3 x 200 x 2 places added as independent errors, over 2 e, is under 10^-4 of the change for e = 0.02."""
    draw = drawer(3)
    names = ["x", "y", "gate", "weight", "bias", "post_weight"]
    at = dict(zip(names, (draw(3, 2, 100), draw(3, 2, 100), draw(3, 100), draw(3, 100), draw(3, 100), draw(100))))
    if post is None:
        del at["post_weight"]
    u, v = draw(3, 2, 100), draw(3, 2, 100)
    value = lambda t: sum((a.double() * b.double()).sum() for a, b in zip(ag.residual_norm(**t, kind=kind, post=post, residual_scale=0.5, eps=1e-2), (u, v)))
    leaf = {k: t.clone().requires_grad_() for k, t in at.items()}
    value(leaf).backward()
    for name in at:
        d = draw(*at[name].shape)
        slope = lambda e: float(value({**at, name: at[name] + e * d}) - value({**at, name: at[name] - e * d})) / (2 * e)
        want = (4 * slope(0.02) - slope(0.04)) / 3
        size = float((leaf[name].grad.double() * d.double()).norm())
        assert abs(float((leaf[name].grad.double() * d.double()).sum()) - want) <= 2e-3 * size + 1e-3 * abs(want), name


def test_autograd_gives_what_the_backward_call_gives():
    draw = drawer(5)
    x, y, gate, weight, bias = draw(2, 50, 384).to(BF), draw(2, 50, 384).to(BF), draw(2, 384).to(BF), draw(384).to(BF), draw(384).to(BF)
    dr, dh = draw(2, 50, 384).to(BF), draw(2, 50, 384).to(BF)
    how = dict(kind="rms", post="rms")
    _, _, stats = cb.residual_norm(x, y, gate, weight, bias, save_stats=True, **how)

    def grads(use, wanted=(True,) * 5):
        leaf = [t.clone().requires_grad_(w) for t, w in zip((x, y, gate, weight, bias), wanted)]
        r, h = ag.residual_norm(*leaf, **how)
        use(r, h)
        return [t.grad for t in leaf]
    want = cb.residual_norm_backward(dr, dh, x, y, gate, weight, bias, None, stats, **how)
    for a, b in zip(grads(lambda r, h: torch.autograd.backward([r, h], [dr, dh])), want):
        assert torch.equal(a, b)
    for a, b in zip(grads(lambda r, h: torch.autograd.backward([r, h], [dr, dh]), (False, True, False, True, False)), want):
        assert a is None or torch.equal(a, b)
    # one of the two outputs alone; gradients that are expanded
    for a, b in zip(grads(lambda r, h: h.backward(dh)), cb.residual_norm_backward(None, dh, x, y, gate, weight, bias, None, stats, **how)):
        assert torch.equal(a, b)
    for a, b in zip(grads(lambda r, h: r.backward(dr)), cb.residual_norm_backward(dr, torch.zeros_like(dh), x, y, gate, weight, bias, None, stats, **how)):
        assert torch.equal(a, b)
    ones = torch.ones_like(x)
    for a, b in zip(grads(lambda r, h: (r.sum() + h.sum()).backward()), cb.residual_norm_backward(ones, ones, x, y, gate, weight, bias, None, stats, **how)):
        assert torch.equal(a, b)


def test_autograd_keeps_nothing_without_gradients_and_takes_any_layout():
    draw = drawer(6)
    x, y = draw(4, 300, 512).to(BF), draw(300, 4, 512).to(BF).transpose(0, 1)
    w = draw(512).to(BF).requires_grad_()
    with torch.no_grad():
        r, h = ag.residual_norm(x, y, weight=w)
    assert not r.requires_grad and not h.requires_grad
    r2, h2 = ag.residual_norm(x, y, weight=w)
    assert torch.equal(h, h2) and h2.requires_grad
    for t in (draw(512, 7).to(BF).t(), draw(2, 3, 4, 512).to(BF), draw(1, 9, 1024).to(BF)[..., ::2], draw(1, 1, 512).to(BF).expand(2, 6, 512)):
        a, b = ag.residual_norm(t, t, weight=w), cb.residual_norm(t.contiguous(), t.contiguous(), weight=w)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_gradient_of_a_gradient_is_refused():
    x = torch.randn(2, 3, 64, device="cuda", requires_grad=True)
    _, h = ag.residual_norm(x, x.detach())
    grad, = torch.autograd.grad(h.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()


def test_more_items_than_the_sums_have_sets():
    x = torch.zeros(65536, 1, 8, device="cuda")
    with pytest.raises(ca.ClearAttnError):
        ag.residual_norm(x, x, gate=torch.zeros(65536, 8, device="cuda", requires_grad=True))
    r, h = cb.residual_norm(x, x, gate=torch.zeros(65536, 8, device="cuda"))
    assert r.shape == x.shape


# ---- streams and graphs

def calls():
    draw = drawer(7)
    x, y, gate, w, pw = draw(2, 400, 640).to(BF), draw(2, 400, 640).to(BF), draw(2, 640), draw(640), draw(640)
    dr, dh = draw(2, 400, 640).to(BF), draw(2, 400, 640).to(BF)
    stats = cb.residual_norm(x, y, gate, w, w, pw, post="rms", save_stats=True)[2]
    grads = [draw(300, 77), draw(5001).to(BF)]
    scale = torch.tensor(0.5, device="cuda")

    def clipped(s):
        kept = [g.clone() for g in grads]
        if s is not None:
            torch.cuda.ExternalStream(s).wait_stream(torch.cuda.current_stream())
        return (cb.clip_grads(kept, 1.0, grad_scale=scale, stream=s), *kept)
    xs, q, bias = operands(300, 2432, 520, BF)
    bias = bias.cuda()
    long, ql, _ = operands(100, 8192, 130, BF)
    return [lambda s: cb.residual_norm(x, y, gate, w, w, pw, post="rms", save_stats=True, stream=s),
            lambda s: cb.residual_norm_backward(dr, dh, x, y, gate, w, w, pw, stats, post="rms", stream=s),
            lambda s: cb.grad_norm(grads, max_norm=1.0, stream=s), clipped, lambda s: tuple(cb.mx_quantize(xs, stream=s)), lambda s: (cb.mx_dequantize(q, stream=s),),
            lambda s: (cb.mx_linear(xs, q, bias, stream=s),), lambda s: (cb.mx_linear(xs[:2], q, stream=s),), lambda s: (cb.mx_linear(long, ql, stream=s),)]


def test_every_call_on_a_named_stream():
    side = torch.cuda.Stream()
    for i, call in enumerate(calls()):
        want = call(None)
        got = on(side, call)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.parametrize("number", range(9))
def test_captured_and_replayed(number):
    call = calls()[number]
    want = [t.clone() for t in call(None)]
    graph, others = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(None)
    with torch.cuda.graph(others):
        again = call(None)
    for _ in range(3):
        for t in (*got, *again):
            t.zero_()
        graph.replay()
        others.replay()
        eager = call(None)
        torch.cuda.synchronize()
        for a, b, c, d in zip(got, again, eager, want):
            assert torch.equal(a, d) and torch.equal(b, d) and torch.equal(c, d)


def test_a_training_step_captured():
    draw = drawer(9)
    w0 = [draw(64, 64, k=0.1).to(BF), draw(64).to(BF)]
    x, y, target = draw(2, 30, 64).to(BF), draw(2, 30, 64).to(BF), draw(2, 30, 64).to(BF)

    def step(params, opt):
        r, h = ag.residual_norm(x, y, gate=params[1], weight=params[1])
        loss = ((h.reshape(-1, 64) @ params[0]).view_as(r) + r - target).float().square().mean()
        grads = torch.autograd.grad(loss, params)
        opt.step(grads, max_norm=0.1)
        return grads

    eager = [w.clone().requires_grad_() for w in w0]
    one = AdamW(eager, lr=1e-2)
    for _ in range(3):
        step(eager, one)
        one.steps = 0
    captured = [w.clone().requires_grad_() for w in w0]
    other = AdamW(captured, lr=1e-2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (what the libraries under torch set up on their first call)
        warm = [w.clone().requires_grad_() for w in w0]
        step(warm, AdamW(warm))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured, other)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager, captured):
        assert torch.equal(a, b)
    assert torch.equal(one.grad_norm, other.grad_norm) and float(one.grad_norm) > 0.1


# ---- offsets past 32 bits

@pytest.fixture
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def test_residual_far_apart(room):
    far = (1 << 31) + 64  # elements from one item to the next
    flat = [torch.empty(far + 400, dtype=BF, device="cuda") for _ in range(4)]
    x, y, dr, dh = (t.as_strided((2, 3, 128), (far, 128, 1)).normal_() for t in flat)
    gate = torch.randn(2, 128, device="cuda")
    r, h, stats = cb.residual_norm(x, y, gate, save_stats=True)
    near = [t.contiguous() for t in (x, y, dr, dh)]
    want = cb.residual_norm(near[0], near[1], gate, save_stats=True)
    assert all(torch.equal(a, b) for a, b in zip((r, h, stats), want))
    got = cb.residual_norm_backward(dr, dh, x, y, gate, None, None, None, stats)
    for a, b in zip(got, cb.residual_norm_backward(near[2], near[3], near[0], near[1], gate, None, None, None, stats)):
        assert a is None and b is None or torch.equal(a, b)
    cb.residual_norm(x, y, gate, out=(x, y))
    assert torch.equal(x, want[0]) and torch.equal(y, want[1])


def test_long_gradients(room):
    n = (1 << 32) + 12345
    g = torch.zeros(n, dtype=BF, device="cuda")
    places = torch.tensor([0, 1, (1 << 31) + 5, (1 << 32) - 1, 1 << 32, n - 1], device="cuda")
    g[places] = torch.tensor([3.0, 4.0, 12.0, -84.0, 3612.0, -8.0], device="cuda").to(BF)
    norm, factor = cb.grad_norm([g, torch.ones(7, device="cuda")], max_norm=1.0)
    want = math.sqrt(float(g[places].double().square().sum()) + 7)
    assert abs(float(norm) - want) <= want * 2.0 ** -23
    kept = g[places].float()
    cb.scale_grads([g], torch.tensor(0.5, device="cuda"))
    assert torch.equal(g[places].float(), 0.5 * kept)


def test_4_bit_operands_far_apart(room):
    F, C = 4200, 512
    x, w, _ = operands(300, C, F, BF)
    ld = 1 << 20  # bytes from one row of codes to the next: 4.4 GB
    codes = torch.empty(F * ld, dtype=torch.uint8, device="cuda").as_strided((F, C // 2), (ld, 1))
    codes.copy_(w.codes)
    far = cb.MX4(codes, w.scales)
    for tokens in (3, 300):
        assert torch.equal(cb.mx_linear(x[:tokens], far), cb.mx_linear(x[:tokens], w))
    assert torch.equal(cb.mx_dequantize(far), cb.mx_dequantize(w))
    del codes, far
    step = (1 << 31) + 8  # elements from one token to the next, in and out
    spread = torch.empty(2 * step + C, dtype=BF, device="cuda").as_strided((3, C), (step, 1))
    spread.copy_(x[:3])
    out = torch.empty(2 * step + F, dtype=BF, device="cuda").as_strided((3, F), (step, 1))
    cb.mx_linear(spread, w, out=out)
    assert torch.equal(out, cb.mx_linear(x[:3], w))
    q, want = cb.mx_quantize(spread), cb.mx_quantize(x[:3])
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)


def test_many_tokens_of_4_bits(room):
    M, C, F = 2_200_000, 256, 1000  # 2.2 G outputs
    x = torch.empty(M, C, dtype=BF, device="cuda").normal_()
    w = cb.mx_quantize(torch.randn(F, C, device="cuda"))
    y = cb.mx_linear(x, w)
    for part in (slice(0, 70), slice(M - 70, M)):
        values, _ = ref.quantized(x[part].cpu())
        want, off = product(values, w, None, BF)
        ref.check(y[part], want, off, "product")


# ---- together

def test_a_block_in_4_bits():
    """Two sublayers of an inference step with weights in 4 bits, the norm's output taken to 4 bits once for three projections, against the same in 64 bits from the operators' definitions at every step's own inputs."""
    draw = drawer(11)
    B, N, C = 2, 173, 320
    x, y = draw(B, N, C).to(BF), draw(B, N, C).to(BF)
    gate, scale, shift = draw(B, C, k=0.3).to(BF), draw(B, C, k=0.1).to(BF), draw(B, C, k=0.1).to(BF)
    weights = [cb.mx_quantize(draw(n, C, k=C ** -0.5)) for n in (C, C, 77)]
    r, h = cb.residual_norm(x, y, gate, scale, shift, weight_offset=1.0)
    q = cb.mx_quantize(h)
    assert q.codes.shape == (B, N, C // 2) and q.scales.shape == (2, B * N, 8)
    values, _ = ref.quantized(h.reshape(-1, C).cpu())
    for w in weights:
        got = cb.mx_linear(q, w)
        want, off = product(values, w, None, BF)
        assert got.shape == (B, N, w.codes.shape[0])
        ref.check(got.reshape(B * N, -1), want, off, "projection")
        assert torch.equal(got, cb.mx_linear(h, w))
    z = cb.mx_linear(q, weights[0])
    exact_r, exact_h = ref.residual_norm(*(t.double().cpu() for t in (r, z, gate, scale, shift)), None, "layer", None, 1e-6, 1.0, 1.0, 0.0)
    r2, h2 = cb.residual_norm(r, z, gate, scale, shift, weight_offset=1.0)
    ref.check(r2, exact_r, ref.half_step(BF) * exact_r.abs() + 8 * ref.FP32 * (r.double().cpu().abs() + 8), "r")
    # (two matrix products lie between inputs and here; h itself is of the norm of r in fp32, off by 64 half steps of r's largest over its deviation)
    size = exact_r.abs().amax(-1, keepdim=True) / exact_r.std(-1, keepdim=True)
    ref.check(h2, exact_h, ref.half_step(BF) * exact_h.abs() + 64 * ref.FP32 * (size * 2 + exact_h.abs() + 1), "h")


def test_clipped_training_steps_against_plain_operations():
    """Gated residual, gated projection, loss, backward, clipping inside the optimizer's step: three steps against the same in fp32 torch operations on fp32 parameters.  The projection rounds its operands' gradients to bf16:
    2^-9 of each term, and every bf16 tensor between adds as much; 2 % of a gradient's norm is allowed as for the example's block, and 1 % of the norm of all, whose errors average."""
    draw = drawer(13)
    C, F = 128, 256
    x, y = draw(2, 60, C).to(BF), draw(2, 60, C).to(BF)
    params = [(1 + draw(C, k=0.1)).to(BF), draw(C, k=0.1).to(BF), draw(C, k=0.5).to(BF), draw(F, C, k=C ** -0.5).to(BF), draw(F, C, k=C ** -0.5).to(BF)]
    mine = [p.clone().requires_grad_() for p in params]
    opt = AdamW(mine, lr=1e-3, masters=True)
    for step in range(3):
        r, h = ag.residual_norm(x, y, gate=mine[2], weight=mine[0], bias=mine[1], post="rms")
        loss = ag.gated_ff(h.reshape(-1, C), mine[3], mine[4]).float().square().mean() + r.float().square().mean()
        loss.backward()
        plain = [p.detach().float().cpu().requires_grad_() for p in mine]
        er, eh = ref.residual_norm(x.float().cpu(), y.float().cpu(), plain[2], plain[0], plain[1], None, "layer", "rms", 1e-6, 1.0, 0.0, 0.0)
        eh = eh.reshape(-1, C)
        g = eh @ plain[3].t()
        ((g / (1 + torch.exp(-g)) * (eh @ plain[4].t())).square().mean() + er.square().mean()).backward()
        for a, b in zip(mine, plain):
            assert float((a.grad.float().cpu() - b.grad).norm() / b.grad.norm()) < 0.02
        norm = torch.cat([b.grad.flatten() for b in plain]).norm()
        factor = float(torch.clamp(0.05 / torch.cat([a.grad.float().flatten() for a in mine]).norm(), max=1.0))
        before = [m.clone() for m in opt.masters]
        first = [m.clone() for m in opt.exp_avgs]
        opt.step(max_norm=0.05)
        assert abs(float(opt.grad_norm) - float(norm)) < 0.01 * float(norm)
        for a, m, old in zip(mine, opt.exp_avgs, first):
            want = 0.9 * old.double() + 0.1 * factor * a.grad.double()
            assert bool(((m.double() - want).abs() <= 16 * ref.FP32 * (old.double().abs() + factor * a.grad.double().abs())).all())
        assert all(not torch.equal(a, b) for a, b in zip(opt.masters, before))
        opt.zero_grad()


def test_the_example_uses_them():
    spec = importlib.util.spec_from_file_location("finetune_block", os.path.join(ROOT, "examples", "finetune_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.finetune(n_text=9, grid=12, heads=2, radius=4, steps=3, say=None)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
