"""Tensors whose offsets pass 32 bits: what lies beyond is compared with a call on a copy of it, or with the definition in 64 bits."""
import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from tests import block_util as ref
from tests.test_gpu_block_gated import U, check, products

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def test_rotary():
    N, H, d = 420000, 41, 128  # 2.2 G elements, 4.4 GB
    q = torch.empty(1, N, H, d, dtype=torch.bfloat16, device="cuda").normal_().transpose(1, 2)
    positions, freqs = torch.arange(N, device="cuda"), cb.rotary_frequencies(d, device="cuda")
    for interleaved in (True, False):
        y = cb.rotary(q, None, positions, freqs, interleaved=interleaved)[0]
        for part in (slice(0, 50), slice(N - 50, N)):
            want = cb.rotary(q[:, :, part].contiguous(), None, positions[part].contiguous(), freqs, interleaved=interleaved)[0]
            assert torch.equal(y[:, :, part], want)
        del y


def test_layer_norm():
    B, N, C = 2, 140000, 8200  # 2.3 G elements
    x = torch.empty(B, N, C, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(B, C, device="cuda")
    y, stats = cb.layer_norm(x, w, w, save_stats=True)
    dx, dw, db = cb.layer_norm_backward(y, x, w, w, stats)
    tail = slice(N - 40, N)
    z, s = cb.layer_norm(x[:, tail].contiguous(), w, w, save_stats=True)
    assert torch.equal(y[:, tail], z) and torch.equal(stats[:, :, tail], s)
    assert torch.equal(dx[:, tail], cb.layer_norm_backward(z, x[:, tail].contiguous(), w, w, s, need=(True, False, False))[0])
    # sums over 140 000 rows, in fp32 by groups: 4e-6 of the terms' magnitudes
    for c in (0, C - 1):
        terms = y[1, :, c].double()
        assert abs(float(db[1, c]) - float(terms.sum())) <= 4e-6 * float(terms.abs().sum())


def test_gated():
    M, C, F = 270000, 64, 8200  # 2.2 G outputs, each product 8.9 GB
    g = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda *s, k=1.0: (torch.randn(*s, generator=g, device="cuda") * k).bfloat16()
    x, wg, wu = draw(M, C), draw(F, C, k=0.15), draw(F, C, k=0.12)
    dh = torch.empty(M, F, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    h, pre = cb.gated_ff(x, wg, wu, save_pre=True)
    dx, dwg, dwu = cb.gated_ff_backward(dh, x, wg, wu, pre)
    for rows in (slice(0, 40), slice(M - 40, M)):
        gate, eg = products(x[rows], wg)
        up, eu = products(x[rows], wu)
        a = ref.activation(gate, "silu")
        check(h[rows], a * up, 1.13 * eg * (up.abs() + eu) + (a.abs() + 1.13 * eg) * eu + 16 * U * (1 + gate.abs()) * (gate.abs() + 0.2) * up.abs(), "h")
        assert bool(((pre[0, rows].double() - gate).abs() <= eg).all()) and bool(((pre[1, rows].double() - up).abs() <= eu).all())
        d = dh[rows].double()
        dg, du = d * up * ref.activation_slope(gate, "silu"), d * a
        spread = (dg.square() @ wg.double().square() + du.square() @ wu.double().square()).sqrt()
        check(dx[rows], dg @ wg.double() + du @ wu.double(), 8 * 2.0 ** -9 / 3 ** 0.5 * spread + (2 * F / 8 + 64) * U * (dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs()), "dx")
    for col in (0, F - 1):  # one hidden channel's weights over all tokens
        gate, up, d = x.double() @ wg[col].double(), x.double() @ wu[col].double(), dh[:, col].double()
        for got, weight in ((dwg[col], d * up * ref.activation_slope(gate, "silu")), (dwu[col], d * ref.activation(gate, "silu"))):
            terms = weight[:, None] * x.double()
            bound = 8 * 2.0 ** -9 / 3 ** 0.5 * terms.square().sum(0).sqrt() + (M / 8 + 64) * U * terms.abs().sum(0)
            check(got, terms.sum(0), bound, "dw")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    n = 2 ** 31 + 70000
    p, grad = torch.empty(n, device="cuda").normal_(), torch.empty(n, device="cuda").normal_()
    states = cb.adamw_state(p, bits)
    tail = slice(n - 70000 // 256 * 256 - n % 256, n)  # from a block's beginning on
    assert tail.start % 256 == 0
    q, s = p[tail].clone(), cb.adamw_state(p[tail], bits)
    call = lambda a, b, st: cb.adamw_step([a], [b], [st[0]], [st[1]], step=1, lr=1e-2, scales=[st[2]] if bits == 8 else None)
    call(p, grad, states)
    call(q, grad[tail].clone(), s)
    assert torch.equal(p[tail], q) and torch.equal(states[0][tail], s[0]) and torch.equal(states[1][tail], s[1])
    if bits == 8:
        dm, dv = cb.adamw_decode(states[0], states[2][0], states[1], states[2][1])
        want = cb.adamw_decode(s[0], s[2][0], s[1], s[2][1])
        assert torch.equal(dm[tail], want[0]) and torch.equal(dv[tail], want[1])
