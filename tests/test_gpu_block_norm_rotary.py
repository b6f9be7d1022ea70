"""Layer norm and rotary positions against their definitions in 64 bits.

Tolerances.  A result rounded to bf16 is off by at most 2^-9 of itself; 2^-8 leaves as much for the fp32 value before the rounding.
In fp32 (unit roundoff u = 2^-24) a rotation adds a few roundings of each product and a sine and cosine good to 4 u: under 16 u (|x| + |y|).  A row's mean and
variance are sums of at most 64 values in a lane and 9 levels of lanes and waves, so off by less than 80 u of the mean magnitude; inputs of unit spread
and an offset under 2 leave xhat off by under 3 * 80 u = 1.5e-5, doubled for the weight.  A weight's gradient is a sum over rows of terms that carry the error of
their xhat: under 2e-5 of the sum of the terms' magnitudes, and 2^-8 of itself where it is rounded to bf16."""
import pytest
import torch

from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.autograd import layer_norm as norm_autograd
from paper_2412_16112_amd.autograd import rotary as rotary_autograd
from tests import block_util as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def close(got, want, slack, dtype):
    """|got - want| <= slack, and 2^-8 |want| on top for bf16; NaN and infinities where `want` has them."""
    got, want = got.double().cpu(), want.double()
    bound = slack + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(want), torch.isnan(got))
    bad = (got - want).abs() > bound
    assert not bool((bad & fine).any()), "%d off, largest %g" % (int((bad & fine).sum()), float((got - want).abs()[fine].max()))


# ---- rotary -------------------------------------------------------------------------------------------------------------

def turned_slack(x, half, interleaved, scale):
    """16 u (|x| + |y|) scale for the channels of a pair, 0 for the copied ones."""
    a = x.double().cpu().abs()
    out = torch.zeros_like(a)
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    pair = (a[..., first] + a[..., second]) * 16 * U * abs(scale)
    out[..., first], out[..., second] = pair, pair
    return out


ROTARY = [  # B, Hq, Hk, N, d, rot, axes
    (1, 1, 0, 1, 2, 2, 1), (2, 3, 1, 5, 64, 64, 1), (1, 24, 24, 70, 128, 128, 3), (3, 8, 2, 1, 128, 128, 1), (2, 5, 5, 33, 64, 32, 2),
    (1, 9, 3, 17, 78, 44, 2), (1, 2, 2, 300, 96, 10, 1), (1, 40, 8, 3, 256, 254, 4), (1, 2, 1, 9, 130, 130, 1),
]


def rotary_inputs(B, Hq, Hk, N, d, rot, axes, dtype, seed=0, far=1000):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(B, Hq, N, d, generator=g).to(dtype).cuda()
    k = torch.randn(B, Hk, N, d, generator=g).to(dtype).cuda() if Hk else None
    positions = torch.randint(-far, far, (axes, B, N), generator=g).cuda()
    freqs = torch.stack([cb.rotary_frequencies(rot, theta=100.0 * (a + 3)) for a in range(axes)]).cuda()
    return q, k, positions, freqs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("shape", ROTARY)
def test_rotary(shape, interleaved, dtype):
    q, k, positions, freqs = rotary_inputs(*shape, TYPES[dtype])
    half = freqs.shape[1]
    for inverse, scale, pos in [(False, 1.0, positions), (True, 1.25, positions.int())]:
        got = cb.rotary(q, k, pos, freqs, interleaved=interleaved, scale=scale, inverse=inverse)
        for x, y in zip((q, k), got):
            if x is not None:
                close(y, ref.rotary(x, positions, freqs, interleaved, scale, inverse), turned_slack(x, half, interleaved, scale), TYPES[dtype])
                assert torch.equal(y[..., 2 * half:], x[..., 2 * half:])  # copied, bit for bit


def test_rotary_far_positions_lose_no_precision():
    q, k, _, freqs = rotary_inputs(2, 4, 1, 6, 128, 128, 1, torch.float32)
    positions = torch.tensor([[[0, 1, 10 ** 6, 2 ** 31, 2 ** 40, -(2 ** 40)]] * 2]).cuda()
    # (an angle of 2^40 radians is off by 2^-13 in 64 bits, in the definition as in the kernel: twice that, times the pair)
    slack = turned_slack(q, 64, True, 1.0)
    slack[..., 4:, :] += 2 * 2.0 ** -13 * 2 * q.double().cpu().abs().max()
    close(cb.rotary(q, k, positions, freqs)[0], ref.rotary(q, positions, freqs, True), slack, torch.float32)


@pytest.mark.parametrize("interleaved", [True, False])
def test_rotary_strides_in_place_and_unaligned(interleaved):
    B, H, N, d = 2, 6, 37, 64
    q, k, positions, freqs = rotary_inputs(B, H, H, N, d, 48, 1, torch.bfloat16, seed=3)
    want = cb.rotary(q, k, positions, freqs, interleaved=interleaved)
    packed = torch.stack([q, k, torch.zeros_like(q)], 0).permute(1, 3, 0, 2, 4).contiguous()  # [B, N, 3, H, d], as a projection gives it
    pq, pk = packed[:, :, 0].transpose(1, 2), packed[:, :, 1].transpose(1, 2)
    got = cb.rotary(pq, pk, positions, freqs, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    cb.rotary(pq, pk, positions, freqs, interleaved=interleaved, out_q=pq, out_k=pk)
    assert torch.equal(pq, want[0]) and torch.equal(pk, want[1]) and not bool(packed[:, :, 2].any())
    room = torch.full((q.numel() + 2,), 7.0, dtype=q.dtype, device="cuda")  # 2-byte aligned, and nothing beside is touched
    odd = room[1:-1].view(q.shape)
    odd.copy_(q)
    cb.rotary(odd, None, positions, freqs, interleaved=interleaved, out_q=odd)
    assert torch.equal(odd, want[0]) and float(room[0]) == 7.0 and float(room[-1]) == 7.0
    shared = torch.arange(N, device="cuda")
    a = cb.rotary(q, k, shared, freqs[0], interleaved=interleaved)
    b = cb.rotary(q, k, shared.expand(1, B, N), freqs, interleaved=interleaved)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_rotary_not_finite_stays_in_its_pair():
    q, _, positions, freqs = rotary_inputs(1, 2, 0, 4, 64, 64, 1, torch.float32)
    clean = cb.rotary(q, None, positions, freqs)[0]
    q[0, 1, 2, 10] = float("nan")
    q[0, 0, 1, 3] = float("inf")
    bad = cb.rotary(q, None, positions, freqs)[0]
    touched = torch.zeros_like(q, dtype=torch.bool)
    touched[0, 1, 2, 10:12] = True
    touched[0, 0, 1, 2:4] = True
    assert torch.equal(bad[~touched], clean[~touched]) and bool(torch.isnan(bad[0, 1, 2, 10:12]).all())


def test_rotary_gradient_by_the_formula_and_by_differences():
    q, k, positions, freqs = rotary_inputs(1, 2, 1, 5, 16, 12, 2, torch.float32, far=20)
    q, k = q.requires_grad_(), k.requires_grad_()
    wq, wk = torch.randn_like(q), torch.randn_like(k)
    yq, yk = rotary_autograd(q, k, positions, freqs, interleaved=False, scale=0.75)
    ((yq * wq).sum() + (yk * wk).sum()).backward()
    for x, w in ((q, wq), (k, wk)):
        close(x.grad, ref.rotary(w, positions, freqs, False, 0.75, inverse=True), turned_slack(w, 6, False, 0.75), torch.float32)
        v = torch.randn(x.shape, dtype=torch.float64)
        # (the map is linear: a difference of any length gives the derivative)
        base = x.detach().double().cpu()
        loss = lambda t: (ref.rotary(t, positions, freqs, False, 0.75) * w.double().cpu()).sum()
        assert abs(float((loss(base + v) - loss(base - v)) / 2) - float((x.grad.double().cpu() * v).sum())) < 1e-4


def test_rotary_empty_and_refusals():
    q, k, positions, freqs = rotary_inputs(1, 2, 2, 4, 64, 64, 1, torch.bfloat16)
    assert cb.rotary(q[:, :, :0], k[:, :, :0], positions[:, :, :0], freqs)[0].shape == (1, 2, 0, 64)
    with pytest.raises(ca.ClearAttnError):
        cb.rotary(q, k[:, :, :3], positions, freqs)
    with pytest.raises(ca.ClearAttnError):
        cb.rotary(q, k, positions.float(), freqs)
    with pytest.raises(ca.ClearAttnError):
        cb.rotary(q, k, positions, freqs.float())
    with pytest.raises(ca.ClearAttnError):
        cb.rotary(q, k, positions[:, :, :3], freqs)
    with pytest.raises(ca.ClearAttnError):
        cb.rotary(q.half(), None, positions, freqs)
    with pytest.raises(ca.ClearAttnError):
        cb.rotary(q.cpu(), None, positions, freqs)
    with pytest.raises(ca.ClearAttnError) as e:  # rot_dim 66 of 64 channels
        cb.rotary(q, k, positions, cb.rotary_frequencies(66, device="cuda"))
    assert e.value.status == ca.CLEAR_ERR_INVALID_ARG
    wide = torch.zeros(1, 2, 8, 64, dtype=q.dtype, device="cuda")
    with pytest.raises(ca.ClearAttnError):  # neither in place nor apart
        cb.rotary(wide[:, :, :4], None, positions, freqs, out_q=wide[:, :, 1:5])


# ---- layer norm -----------------------------------------------------------------------------------------------------------

def norm_inputs(B, N, C, dtype, wdtype, per_item, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(B, N, C, generator=g) + torch.randn(C, generator=g)).to(dtype)
    shape = (B, C) if per_item else (C,)
    w, b = (1 + 0.2 * torch.randn(shape, generator=g)).to(wdtype), (0.2 * torch.randn(shape, generator=g)).to(wdtype)
    return x.cuda(), w.cuda(), b.cuda(), torch.randn(B, N, C, generator=g).to(dtype).cuda()


NORM = [  # B, N, C: one element, a lane's part, ragged ends, each number of waves a row takes
    (1, 1, 1), (1, 3, 2), (2, 5, 7), (1, 300, 64), (2, 33, 173), (1, 2049, 40), (2, 70, 1111), (1, 9, 1537), (3, 41, 2432), (1, 20, 3100), (2, 10, 4096),
    (1, 5, 4099), (1, 11, 6500), (1, 4, 8192), (1, 3, 9001), (1, 6, 12345), (1, 3, 16384),
]


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("shape", NORM)
def test_layer_norm_and_its_gradients(shape, types):
    B, N, C = shape
    for per_item, offset in [(False, 0.0), (True, 1.0)]:
        x, w, b, dy = norm_inputs(B, N, C, TYPES[types[0]], TYPES[types[1]], per_item, seed=C)
        eps = 1e-2 if C < 8 else 1e-6  # (a row of one or two channels may have hardly any variance)
        y, stats = cb.layer_norm(x, w, b, eps=eps, weight_offset=offset, save_stats=True)
        leaf = [t.double().cpu().requires_grad_() for t in (x, w, b)]
        want = ref.layer_norm(*leaf, eps, offset)
        weight = (offset + leaf[1].detach()).abs()
        weight = weight.unsqueeze(1) if per_item else weight
        r = 1 / torch.sqrt(((leaf[0] - leaf[0].mean(-1, keepdim=True)) ** 2).mean(-1, keepdim=True) + eps).detach()
        unit = 3e-5 * torch.clamp(r, min=1.0)  # (the spread of the inputs is about 1; rows of few channels may have less)
        close(y, want.detach(), unit * (weight + 1), x.dtype)
        assert torch.equal(y, cb.layer_norm(x, w, b, eps=eps, weight_offset=offset))
        close(stats[0], leaf[0].detach().mean(-1), 2e-5, torch.float32)
        want.backward(dy.double().cpu())
        got = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset)
        dyw = (dy.double().cpu().abs() * weight)
        close(got[0], leaf[0].grad, r * 4 * unit * (dyw + dyw.mean(-1, keepdim=True) * (1 + torch.clamp(r, min=1.0))) * 4, x.dtype)
        xhat = ref.layer_norm(leaf[0].detach(), None, None, eps, 0.0).abs()
        rows = 1 if per_item else (0, 1)
        terms = dy.double().cpu().abs()
        close(got[1], leaf[1].grad, (terms * (2e-5 * xhat + unit)).sum(rows), w.dtype)
        close(got[2], leaf[2].grad, 2e-5 * terms.sum(rows), w.dtype)
        again = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset)
        assert all(torch.equal(s, t) for s, t in zip(got, again))
        only = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset, need=(False, True, True))
        assert only[0] is None and torch.equal(only[1], got[1]) and torch.equal(only[2], got[2])
        only = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset, need=(True, False, False))
        assert torch.equal(only[0], got[0]) and only[1] is None


def test_layer_norm_without_weights():
    x, w, b, dy = norm_inputs(2, 19, 200, torch.float32, torch.float32, False)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    y, stats = cb.layer_norm(x, save_stats=True)
    assert torch.equal(y, cb.layer_norm(x, one, zero))
    assert torch.equal(cb.layer_norm(x, None, b), cb.layer_norm(x, one, b))
    full = cb.layer_norm_backward(dy, x, one, zero, stats)
    dx, dw, db = cb.layer_norm_backward(dy, x, None, b, stats)
    assert torch.equal(dx, full[0]) and dw is None and torch.equal(db, full[2])


@pytest.mark.parametrize("C", [40, 2432, 5000])
def test_layer_norm_strides_in_place_and_unaligned(C):
    x, w, b, dy = norm_inputs(2, 21, C, torch.bfloat16, torch.float32, True, seed=5)
    want, stats = cb.layer_norm(x, w, b, save_stats=True)
    grads = cb.layer_norm_backward(dy, x, w, b, stats)
    wide = torch.full((2, 21, C + 3), 9.0, dtype=x.dtype, device="cuda")
    view = wide[..., 1:C + 1]  # rows 2-byte aligned, with neighbours that must stay
    view.copy_(x)
    assert torch.equal(cb.layer_norm(view, w, b), want)
    dwide = torch.empty((2, 21, C + 5), dtype=x.dtype, device="cuda")[..., 2:C + 2]
    dwide.copy_(dy)
    got = cb.layer_norm_backward(dwide, view, w, b, stats)
    assert all(torch.equal(s, t) for s, t in zip(got, grads))
    token_major = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(cb.layer_norm(token_major, w, b), want)
    cb.layer_norm(view, w, b, out=view)
    assert torch.equal(view, want) and bool((wide[..., 0] == 9).all()) and bool((wide[..., C + 1:] == 9).all())


def test_layer_norm_large_mean_keeps_the_variance():
    # fp32 values 1000 + N(0, 1): the differences from the mean are exact to u * 1000, so xhat to 1000 * 80 u
    x = (1000 + torch.randn(3, 7, 900, generator=torch.Generator().manual_seed(1))).cuda()
    close(cb.layer_norm(x), ref.layer_norm(x.double().cpu(), None, None, 1e-6, 0.0), 1000 * 80 * U, torch.float32)


def test_layer_norm_not_finite_rows_stay_alone():
    x, w, b, dy = norm_inputs(1, 40, 300, torch.float32, torch.float32, False)
    clean, stats = cb.layer_norm(x, w, b, save_stats=True)
    dx = cb.layer_norm_backward(dy, x, w, b, stats)[0]
    x[0, 3, 5], x[0, 17, 299] = float("nan"), float("inf")
    y, stats = cb.layer_norm(x, w, b, save_stats=True)
    bad = cb.layer_norm_backward(dy, x, w, b, stats)[0]
    keep = [i for i in range(40) if i not in (3, 17)]
    assert torch.equal(y[:, keep], clean[:, keep]) and torch.equal(bad[:, keep], dx[:, keep])
    assert bool(torch.isnan(y[0, 3]).all()) and bool(torch.isnan(y[0, 17]).all())


def test_layer_norm_no_rows():
    x, w, b, dy = norm_inputs(1, 4, 64, torch.float32, torch.float32, False)
    y, stats = cb.layer_norm(x[:, :0], w, b, save_stats=True)
    dx, dw, db = cb.layer_norm_backward(dy[:, :0], x[:, :0], w, b, stats)
    assert y.shape == (1, 0, 64) and dx.shape == y.shape and not bool(dw.any()) and not bool(db.any())


def test_layer_norm_gradient_by_differences():
    x, w, b, dy = norm_inputs(2, 6, 50, torch.float32, torch.float32, True)
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    (norm_autograd(*leaves, eps=1e-6, weight_offset=1.0) * dy).sum().backward()
    base = [t.double().cpu() for t in (x, w, b)]
    loss = lambda *t: float((ref.layer_norm(*t, 1e-6, 1.0) * dy.double().cpu()).sum())
    g = torch.Generator().manual_seed(9)
    for i in range(3):
        v = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
        step = 1e-4  # central difference: error step^2 times a third derivative, under 1e-5
        moved = [loss(*[t + s * step * v if j == i else t for j, t in enumerate(base)]) for s in (1, -1)]
        assert abs((moved[0] - moved[1]) / (2 * step) - float((leaves[i].grad.double().cpu() * v).sum())) < 2e-3


def test_layer_norm_refusals():
    x, w, b, dy = norm_inputs(2, 3, 64, torch.float32, torch.float32, False)
    for bad in [lambda: cb.layer_norm(x, w[:63], b), lambda: cb.layer_norm(x, w, b.bfloat16()), lambda: cb.layer_norm(x.half()), lambda: cb.layer_norm(x, eps=-1.0),
                lambda: cb.layer_norm(x.transpose(1, 2)), lambda: cb.layer_norm(x, w.cpu(), b), lambda: cb.layer_norm(x[0], w.expand(2, 64).contiguous(), None),
                lambda: cb.layer_norm(torch.zeros(1, 1, 16385, device="cuda")), lambda: cb.layer_norm(x, eps=float("nan")),
                lambda: cb.layer_norm(x, out=x[:, :1].expand(2, 3, 64)), lambda: cb.layer_norm_backward(dy, x, w, b, torch.zeros(2, 2, 2, device="cuda"))]:
        with pytest.raises(ca.ClearAttnError):
            bad()


# ---- streams and graphs ---------------------------------------------------------------------------------------------------

def test_norm_and_rotary_on_another_stream_and_in_a_graph():
    x, w, b, dy = norm_inputs(2, 500, 256, torch.bfloat16, torch.bfloat16, True)
    q, k, positions, freqs = rotary_inputs(1, 4, 2, 100, 64, 64, 1, torch.bfloat16)

    def work():
        y, stats = cb.layer_norm(x, w, b, save_stats=True)
        return [y, *cb.layer_norm_backward(dy, x, w, b, stats), *cb.rotary(q, k, positions, freqs)]
    want = [t.clone() for t in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = work()
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(got, want))
    with torch.cuda.graph(graph):
        held = work()
    for turn in range(3):
        x.mul_(1.5)
        q.neg_()
        graph.replay()
        eager = work()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(held, eager)), turn
