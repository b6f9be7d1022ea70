"""The gated feed-forward projection and its gradients against the definition in 64 bits.

Tolerances.  A product of depth K in fp32, added up 8 or 16 terms at a time, is off by at most (K / 8 + 16) u of the sum of its terms' magnitudes
(u = 2^-24).  h = act(g) u carries those of g (slope at most 1.13) and of u, and its rounding to bf16: 2^-8 of itself.  dG and dU are rounded to bf16 (2^-9
each, independent of one another) before they are summed with weights w: the error of the sum has a spread of at most 2^-9 / sqrt(3) * sqrt(sum (dG w)^2), of which
8 are allowed, on top of the accumulation's bound and the output's rounding."""
import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.autograd import gated_ff as gated_autograd
from tests import block_util as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def inputs(M, C, F, seed=0, dev="cuda"):
    g = torch.Generator().manual_seed(seed)
    bf = lambda *s, k=1.0: (torch.randn(*s, generator=g) * k).to(torch.bfloat16).to(dev)
    return bf(M, C), bf(F, C, k=1.5 / C ** 0.5), bf(F, C, k=1 / C ** 0.5), bf(M, F)


def products(x, w):
    """x w^T in 64 bits and its error bound."""
    x, w = x.double(), w.double()
    depth = x.shape[1] / 8 + 16
    return x @ w.T, depth * U * (x.abs() @ w.abs().T)


def check(got, want, slack, what):
    bad = (got.double() - want).abs() > slack + 2.0 ** -8 * want.abs()
    assert not bool(bad.any()), "%s: %d of %d off, largest error %g of %g" % (what, int(bad.sum()), bad.numel(), float((got.double() - want).abs().max()), float(want.abs().max()))


def check_forward(x, wg, wu, act, h, pre=None):
    g, eg = products(x, wg)
    u, eu = products(x, wu)
    a = ref.activation(g, act)
    # (the activation itself, in fp32 with the fast exponential: 16 u of its terms)
    check(h, a * u, 1.13 * eg * (u.abs() + eu) + (a.abs() + 1.13 * eg) * eu + 16 * U * (1 + g.abs()) * (g.abs() + 0.2) * u.abs(), "h")
    if pre is not None:
        assert bool(((pre[0].double() - g).abs() <= eg).all()) and bool(((pre[1].double() - u).abs() <= eu).all())


def check_backward(dh, x, wg, wu, act, dx, dwg, dwu):
    g, _ = products(x, wg)
    u, _ = products(x, wu)
    d = dh.double()
    dg, du = d * u * ref.activation_slope(g, act), d * ref.activation(g, act)
    rounding = 8 * 2.0 ** -9 / 3 ** 0.5

    def bound(pairs, depth):
        spread = sum(p.square() @ q.square() for p, q in pairs).sqrt()
        return rounding * spread + (depth / 8 + 64) * U * sum(p.abs() @ q.abs() for p, q in pairs)
    if dx is not None:
        check(dx, dg @ wg.double() + du @ wu.double(), bound([(dg, wg.double()), (du, wu.double())], 2 * wg.shape[0]), "dx")
    if dwg is not None:
        check(dwg, dg.T @ x.double(), bound([(dg.T, x.double())], x.shape[0]), "dwg")
        check(dwu, du.T @ x.double(), bound([(du.T, x.double())], x.shape[0]), "dwu")


SIZES = [  # tokens, channels, hidden: one token; each number of token blocks; around the switch to tiles; ragged in every direction; several tiles; both tile sizes
    (1, 8, 8), (1, 4096, 1000), (3, 264, 24), (16, 72, 40), (17, 1000, 88), (32, 64, 64), (33, 512, 136), (64, 2432, 72),
    (65, 8, 8), (65, 64, 64), (100, 72, 200), (128, 128, 128), (129, 136, 264), (257, 520, 328), (300, 2432, 1000), (1000, 328, 2056), (2049, 640, 3208), (5000, 264, 2600),
]


@pytest.mark.parametrize("size", SIZES)
def test_forward_and_gradients(size):
    M, C, F = size
    x, wg, wu, dh = inputs(M, C, F, seed=M + C)
    act = ["silu", "gelu_tanh", "gelu_erf"][(M + F // 8) % 3]
    h = cb.gated_ff(x, wg, wu, activation=act)
    h2, pre = cb.gated_ff(x, wg, wu, activation=act, save_pre=True)
    assert torch.equal(h, h2)
    check_forward(x, wg, wu, act, h, pre)
    got = cb.gated_ff_backward(dh, x, wg, wu, pre, activation=act)
    check_backward(dh, x, wg, wu, act, *got)
    again = cb.gated_ff_backward(dh, x, wg, wu, pre, activation=act)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    dx = cb.gated_ff_backward(dh, x, wg, wu, pre, activation=act, need=(True, False))
    assert torch.equal(dx[0], got[0]) and dx[1] is None
    dw = cb.gated_ff_backward(dh, x, wg, wu, pre, activation=act, need=(False, True))
    assert dw[0] is None and torch.equal(dw[1], got[1]) and torch.equal(dw[2], got[2])


@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "gelu_erf"])
def test_activations_over_their_range(act):
    # one channel of 8 carries the value: g and u are exact, from -60 to 60 and the infinities of large gates
    values = torch.cat([torch.linspace(-60, 60, 1985), torch.tensor([-3e38, 3e38, -1e30, 1e30, 0.0, -0.0, 1e-30])]).to(torch.bfloat16)
    x = torch.zeros(values.numel(), 8, dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = values, 1
    wg, wu = torch.zeros(8, 8, dtype=torch.bfloat16), torch.zeros(8, 8, dtype=torch.bfloat16)
    wg[:, 0], wu[:, 1] = 1, 1
    h, pre = cb.gated_ff(x.cuda(), wg.cuda(), wu.cuda(), activation=act, save_pre=True)
    g = values.double()
    want = torch.where(g < -1e3, torch.zeros_like(g), torch.where(g > 1e3, g, ref.activation(g, act)))  # (g^3 of the definition overflows out there)
    got = h[:, 3].double().cpu()
    assert not bool(torch.isnan(got).any())
    slack = 16 * U * (1 + g.abs()) * (g.abs() + 0.2)
    inner = g.abs() <= 1e3
    assert bool(((got - want).abs() <= slack + 2.0 ** -8 * want.abs())[inner].all()) and torch.equal(got[~inner], want[~inner])
    dh = torch.ones_like(h)
    dx = cb.gated_ff_backward(dh, x.cuda(), wg.cuda(), wu.cuda(), pre, activation=act, need=(True, False))[0].double().cpu()
    slope = torch.where(g < -1e3, torch.zeros_like(g), torch.where(g > 1e3, torch.ones_like(g), ref.activation_slope(g, act)))
    # dx of channel 0 is 8 act'(g), of channel 1 8 act(g), through one more rounding to bf16
    assert bool(((dx[:, 0] - 8 * slope).abs() <= 2.0 ** -7 * 8 * slope.abs() + 8 * 64 * U * (1 + g.clamp(-1e3, 1e3) ** 2)).all())
    fine = inner
    assert bool(((dx[:, 1] - 8 * want).abs() <= 2.0 ** -7 * 8 * want.abs() + 8 * slack)[fine].all())


@pytest.mark.parametrize("M", [5, 70, 300])
def test_strides_and_neighbours(M):
    C, F = 136, 200
    x, wg, wu, dh = inputs(M, C, F, seed=M)
    want, pre = cb.gated_ff(x, wg, wu, save_pre=True)
    grads = cb.gated_ff_backward(dh, x, wg, wu, pre)
    nan = float("nan")
    wide = lambda t, pad: torch.cat([t, torch.full((t.shape[0], pad), nan, dtype=t.dtype, device="cuda")], 1)[:, :t.shape[1]]
    packed = torch.cat([wg, wu], 0)  # one weight of 2 F rows
    xs, gs, us = wide(x, 8), wide(packed, 24)[:F], wide(packed, 24)[F:]
    room = torch.full((M, F + 16), 5.0, dtype=x.dtype, device="cuda")
    h, pre2 = cb.gated_ff(xs, gs, us, out=room[:, 8:F + 8], save_pre=True)
    assert torch.equal(h, want) and torch.equal(pre2, pre)
    assert bool((room[:, :8] == 5).all()) and bool((room[:, F + 8:] == 5).all())
    got = cb.gated_ff_backward(wide(dh, 16), xs, gs, us, pre)
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    three = x.view(1, M, C)
    assert torch.equal(cb.gated_ff(three, wg, wu), want.view(1, M, F))


@pytest.mark.parametrize("M", [3, 200])
def test_not_finite_stays_in_its_row_and_column(M):
    x, wg, wu, dh = inputs(M, 72, 96, seed=2)
    clean, pre = cb.gated_ff(x, wg, wu, save_pre=True)
    x2, wg2 = x.clone(), wg.clone()
    x2[1, 70] = float("nan")
    wg2[17, 71] = float("inf")
    bad = cb.gated_ff(x2, wg2, wu)
    rows = [i for i in range(M) if i != 1]
    cols = [i for i in range(96) if i != 17]
    assert torch.equal(bad[rows][:, cols], clean[rows][:, cols]) and bool(torch.isnan(bad[1]).all())
    assert not bool(torch.isfinite(bad[:, 17]).all())


def test_no_tokens():
    x, wg, wu, dh = inputs(4, 64, 72)
    h, pre = cb.gated_ff(x[:0], wg, wu, save_pre=True)
    dx, dwg, dwu = cb.gated_ff_backward(dh[:0], x[:0], wg, wu, pre)
    assert h.shape == (0, 72) and dx.shape == (0, 64) and not bool(dwg.any()) and not bool(dwu.any())


def test_gradient_by_differences():
    # the directional derivative of the 64-bit definition against the kernel's gradients, which carry bf16 roundings: 2^-9 a term, independent
    x, wg, wu, dh = inputs(90, 40, 48, seed=7)
    leaves = [t.clone().requires_grad_() for t in (x, wg, wu)]
    gated_autograd(*leaves, activation="gelu_tanh").backward(dh)
    base = [t.double() for t in (x, wg, wu)]
    loss = lambda x_, g_, u_: float((ref.activation(x_ @ g_.T, "gelu_tanh") * (x_ @ u_.T) * dh.double()).sum())
    for i in range(3):
        v = torch.randn(base[i].shape, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(i))
        step = 1e-5
        moved = [loss(*[t + s * step * v if j == i else t for j, t in enumerate(base)]) for s in (1, -1)]
        grad = leaves[i].grad.double()
        assert abs((moved[0] - moved[1]) / (2 * step) - float((grad * v).sum())) <= 8 * 2.0 ** -8 * float((grad * v).square().sum().sqrt()) + 1e-3


def test_refusals():
    x, wg, wu, dh = inputs(4, 64, 72)
    _, pre = cb.gated_ff(x, wg, wu, save_pre=True)
    for bad in [lambda: cb.gated_ff(x.float(), wg, wu), lambda: cb.gated_ff(x, wg, wu[:64]), lambda: cb.gated_ff(x[:, :56], wg, wu), lambda: cb.gated_ff(x, wg, wu, activation="tanh"),
                lambda: cb.gated_ff(x[:, :60].contiguous(), wg[:, :60].contiguous(), wu[:, :60].contiguous()), lambda: cb.gated_ff(x.t()[:4, :4].t(), wg, wu),
                lambda: cb.gated_ff(x, wg.cpu(), wu), lambda: cb.gated_ff(x, wg[:70], wu[:70]), lambda: cb.gated_ff(x, wg, wu, out=torch.empty(5, 72, dtype=x.dtype, device="cuda")),
                lambda: cb.gated_ff_backward(dh, x, wg, wu, pre[:, :3]), lambda: cb.gated_ff_backward(dh[:3], x, wg, wu, pre),
                lambda: cb.gated_ff(torch.empty(4 * 64 + 1, dtype=x.dtype, device="cuda")[1:].view(4, 64), wg, wu)]:
        with pytest.raises(ca.ClearAttnError):
            bad()


def test_stream_and_graph():
    x, wg, wu, dh = inputs(300, 128, 264)

    def work():
        h, pre = cb.gated_ff(x, wg, wu, save_pre=True)
        return [h, *cb.gated_ff_backward(dh, x, wg, wu, pre), cb.gated_ff(x[:3], wg, wu)]
    want = [t.clone() for t in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = work()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for turn in range(3):
        x.mul_(0.5)
        graph.replay()
        eager = work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), turn
