"""The gated residual with its norms on the GPU against its definition in 64 bits, gradients against those of differentiating it.

How far results may be off: a result is rounded to its type once (half a step of it); before that it is formed in fp32 from terms whose sizes are worked out here from the exact
values, with at most 64 half steps of fp32 of these (a row's sums are trees over at most 8 x 64 x 16 elements, a column's over at most 20 rows in sequence and the workgroups' partial sums)."""
import itertools

import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from tests import more_block_util as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def tensors(B, N, C, dtype, stream, wdtype, gate, per_item, seed=0):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(*shape, generator=g)
    x, y = (1.5 * draw(B, N, C) + 0.5).to(stream), (2 * draw(B, N, C) - 0.3).to(dtype)
    vector = lambda many: draw(B, C) if many else draw(C)
    gate = vector(gate == "item").to(wdtype) if gate else None
    weight, bias = (1 + 0.2 * vector(per_item)).to(wdtype), (0.2 * vector(per_item)).to(wdtype)
    return x, y, gate, weight, bias, (1 + 0.2 * draw(C)).to(wdtype), draw(B, N, C).to(stream), draw(B, N, C).to(dtype)


def top(t):
    return t.abs().amax(-1, keepdim=True)


def expected(x, y, gate, weight, bias, pw, dr, dh, kind, post, scale, offset, post_offset):
    """Exact results and how far fp32 may be off them before the rounding to a type: {name: (value, off)}."""
    leaf = {k: None if v is None else v.double().requires_grad_() for k, v in dict(x=x, y=y, gate=gate, weight=weight, bias=bias, pw=pw).items()}
    r, h = ref.residual_norm(*leaf.values(), kind, post, EPS, scale, offset, post_offset)
    dh = dh.double()
    drd = torch.zeros_like(r) if dr is None else dr.double()
    names = [k for k, v in leaf.items() if v is not None]
    grads = dict(zip(names, torch.autograd.grad([r, h], [leaf[k] for k in names], [drd, dh])))
    with torch.no_grad():
        E = 64 * ref.FP32
        X, Y = leaf["x"], leaf["y"]
        one = torch.ones((), dtype=torch.float64)
        w = one if weight is None else ref.wide(leaf["weight"]) + offset
        p = one if pw is None or post is None else leaf["pw"] + post_offset
        g = one if gate is None else ref.wide(leaf["gate"])
        centred = lambda v, k: v - v.mean(-1, keepdim=True) if k == "layer" else v
        inv = lambda v, k: 1 / torch.sqrt((centred(v, k) ** 2).mean(-1, keepdim=True) + EPS)
        uy, iy = (ref.unit(Y, post, EPS), inv(Y, post)) if post else (Y, one)
        off_uy = top(Y) * iy if post else 0 * Y  # (of the unit form: the mean's and the differences' roundings are of y's size)
        off_z = (off_uy + uy.abs()) * p.abs() if post else 0 * Y
        off_r = (scale * X).abs() + (g * uy * p).abs() + g.abs() * off_z
        ir, ur = inv(r, kind), ref.unit(r, kind, EPS)
        off_ur = (top(r) + top(off_r)) * ir + ur.abs()
        out = {"r": (r, E * off_r), "h": (h, E * (off_ur * w.abs() + h.abs() + (0 if bias is None else ref.wide(leaf["bias"]).abs())))}
        dyw = (dh * w).abs()
        off_d = drd.abs() + ir * (top(dyw) * (1 + top(ur)) * (1 + top(off_ur)))
        dz_off = g.abs() * off_d
        d_size = (scale * off_d)
        out["x"] = (grads["x"], E * d_size)
        off_dz = dz_off * p.abs()
        out["y"] = (grads["y"], E * (iy * (top(off_dz) * (1 + top(uy)) * (1 + top(off_uy))) if post else off_dz))
        over = lambda t, like: t.sum(1) if like.dim() == 2 else t.sum((0, 1))
        if weight is not None:
            out["weight"] = (grads["weight"], E * over(dh.abs() * off_ur, weight))
        if bias is not None:
            out["bias"] = (grads["bias"], E * over(dh.abs(), bias))
        if gate is not None:
            out["gate"] = (grads["gate"], E * over(off_d * ((uy * p).abs() + off_z), gate))
        if post and pw is not None:
            out["pw"] = (grads["pw"], E * over(dz_off * (uy.abs() + off_uy), pw))
    return {k: (v.detach(), o) for k, (v, o) in out.items()}


def compare(got, want):
    for name, t in got.items():
        value, off = want[name]
        ref.check(t, value, off + ref.half_step(t.dtype) * value.abs(), name)


def run(ts, kind, post, scale, offset, post_offset, **more):
    x, y, gate, weight, bias, pw, dr, dh = (None if t is None else t.cuda() for t in ts)
    how = dict(kind=kind, post=post, residual_scale=scale, weight_offset=offset, post_offset=post_offset)
    r, h, stats = cb.residual_norm(x, y, gate, weight, bias, pw, eps=EPS, save_stats=True, **how)
    grads = cb.residual_norm_backward(dr, dh, x, y, gate, weight, bias, pw, stats, **how)
    out = dict(zip(("r", "h", "x", "y", "gate", "weight", "bias", "pw"), (r, h) + grads))
    return {k: v for k, v in out.items() if v is not None}


SIZES = [(1, 1, 1), (2, 3, 5), (1, 2, 8), (2, 7, 64), (1, 1, 512), (3, 33, 257), (1, 601, 136), (2, 50, 1111), (1, 31, 1536), (1, 77, 2432), (2, 40, 2560), (1, 20, 4096), (2, 9, 5003),
         (1, 7, 6149), (1, 5, 8192)]
TYPES = [(BF, BF, BF), (BF, BF, F32), (BF, F32, BF), (BF, F32, F32), (F32, F32, F32), (F32, F32, BF)]
KINDS = list(itertools.product(("layer", "rms"), (None, "layer", "rms")))


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(d).split(".")[1] for d in t))
def test_against_definition(size, types):
    n = SIZES.index(size) + TYPES.index(types)
    kind, post = KINDS[n % 6]
    gate, per_item = [("item", True), ("shared", False), (None, True), ("item", False), ("shared", True)][n % 5]
    ts = list(tensors(*size, *types, gate, per_item, seed=n))
    if post is None:
        ts[5] = None
    numbers = (kind, post, (1.0, 0.7)[n % 2], (0.0, 1.0)[n // 2 % 2], (0.0, 0.25)[n // 3 % 2])
    compare(run(ts, *numbers), expected(*ts, *numbers))


@pytest.mark.parametrize("kind,post", KINDS)
@pytest.mark.parametrize("gate,per_item", [("item", True), ("shared", False), (None, False), ("item", False), ("shared", True)])
def test_every_form(kind, post, gate, per_item):
    ts = list(tensors(3, 37, 328, BF, BF, BF, gate, per_item))
    if post is None:
        ts[5] = None
    numbers = (kind, post, 0.5, 1.0, 0.0)
    compare(run(ts, *numbers), expected(*ts, *numbers))


@pytest.mark.parametrize("left_out", [("gate",), ("weight",), ("bias",), ("pw",), ("dr",), ("gate", "weight", "bias", "pw", "dr")], ids="-".join)
def test_without(left_out):
    names = ["x", "y", "gate", "weight", "bias", "pw", "dr", "dh"]
    ts = [None if k in left_out else t for k, t in zip(names, tensors(2, 19, 200, F32, F32, F32, "item", True))]
    numbers = ("layer", "rms", 1.0, 1.0, 0.5)
    compare(run(ts, *numbers), expected(*ts, *numbers))


@pytest.mark.parametrize("need", [n for n in itertools.product((True, False), repeat=6) if sum(n) in (1, 2, 5)])
def test_only_what_is_wanted(need):
    x, y, gate, weight, bias, pw, dr, dh = (t.cuda() for t in tensors(2, 37, 1000, BF, BF, F32, "item", False))
    r, h, stats = cb.residual_norm(x, y, gate, weight, bias, pw, post="rms", save_stats=True)
    everything = cb.residual_norm_backward(dr, dh, x, y, gate, weight, bias, pw, stats, post="rms")
    some = cb.residual_norm_backward(dr, dh, x, y, gate, weight, bias, pw, stats, post="rms", need=need)
    for wanted, a, b in zip(need, everything, some):
        assert torch.equal(a, b) if wanted else b is None


@pytest.mark.parametrize("C", [5, 300, 2432, 8190])
@pytest.mark.parametrize("dtype,stream", [(BF, BF), (BF, F32), (F32, F32)])
def test_in_place_and_strided(C, dtype, stream):
    x, y, gate, weight, bias, pw, dr, dh = (t.cuda() for t in tensors(3, 21, C, dtype, stream, F32, "item", True))
    apart = lambda t, k: torch.empty(t.shape[1], t.shape[0], C + k, dtype=t.dtype, device="cuda")[..., k:].transpose(0, 1).copy_(t)  # [B, N, C] with rows of a batch interleaved, off alignment
    r, h, stats = cb.residual_norm(x, y, gate, weight, bias, pw, post="layer", save_stats=True)
    xs, ys, drs, dhs = apart(x, 3), apart(y, 1), apart(dr, 5), apart(dh, 2)
    grads = cb.residual_norm_backward(dr, dh, x, y, gate, weight, bias, pw, stats, post="layer")
    for a, b in zip(grads, cb.residual_norm_backward(drs, dhs, xs, ys, gate, weight, bias, pw, stats, post="layer")):
        assert torch.equal(a, b)
    versions = xs._version, ys._version
    r2, h2 = cb.residual_norm(xs, ys, gate, weight, bias, pw, post="layer", out=(xs, ys))
    assert r2 is xs and h2 is ys and torch.equal(xs, r) and torch.equal(ys, h)
    assert xs._version > versions[0] and ys._version > versions[1]


def test_a_bad_row_is_its_own():
    x, y, gate, weight, bias, pw, dr, dh = (t.cuda() for t in tensors(1, 40, 777, BF, BF, BF, "item", True))
    good = cb.residual_norm(x, y, gate, weight, bias, pw, post="rms", save_stats=True)
    for bad in (float("nan"), float("inf")):
        x2 = x.clone()
        x2[0, 17, 5] = bad
        r, h, stats = cb.residual_norm(x2, y, gate, weight, bias, pw, post="rms", save_stats=True)
        others = [i for i in range(40) if i != 17]
        assert torch.equal(r[:, others], good[0][:, others]) and torch.equal(h[:, others], good[1][:, others])
        assert h[0, 17].isnan().all()
        a = cb.residual_norm_backward(dr, dh, x2, y, gate, weight, bias, pw, stats, post="rms")
        b = cb.residual_norm_backward(dr, dh, x, y, gate, weight, bias, pw, good[2], post="rms")
        assert torch.equal(a[0][:, others], b[0][:, others]) and torch.equal(a[1][:, others], b[1][:, others])


def test_rows_of_zeros_and_constants():
    x, y = torch.zeros(1, 3, 100, device="cuda"), torch.zeros(1, 3, 100, device="cuda")
    x[0, 1] = 7.0
    r, h, stats = cb.residual_norm(x, y, kind="layer", post="rms", eps=1e-6, save_stats=True)
    assert torch.equal(r, x) and torch.equal(h, torch.zeros_like(h))
    dx, dy, *_ = cb.residual_norm_backward(torch.ones_like(x), torch.ones_like(y), x, y, None, None, None, None, stats, kind="layer", post="rms")
    assert dx.isfinite().all() and dy.isfinite().all()


def test_no_rows():
    x = torch.empty(2, 0, 64, device="cuda")
    w = torch.randn(2, 64, device="cuda")
    shared = torch.randn(64, device="cuda")
    r, h, stats = cb.residual_norm(x, x.clone(), w, shared, shared, save_stats=True)
    assert r.shape == x.shape and h.shape == x.shape
    grads = cb.residual_norm_backward(x, x, x, x, w, shared, shared, None, stats)
    assert all(torch.equal(g, torch.zeros_like(g)) for g in grads if g is not None) and grads[2].shape == w.shape
    none = torch.empty(0, 5, 64, device="cuda")
    r, h, stats = cb.residual_norm(none, none.clone(), w[:0], shared, shared, save_stats=True)
    grads = cb.residual_norm_backward(none, none, none, none, w[:0], shared, shared, None, stats)
    assert grads[2].shape == (0, 64) and torch.equal(grads[3], torch.zeros_like(shared))


def test_the_same_from_call_to_call():
    ts = tensors(2, 700, 2432, BF, BF, BF, "item", False)
    first = run(ts, "layer", "rms", 1.0, 0.0, 0.0)
    for _ in range(3):
        again = run(ts, "layer", "rms", 1.0, 0.0, 0.0)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_many_rows_of_a_batch():
    # (several turns of every workgroup, sets that do not share rows evenly)
    ts = list(tensors(5, 1203, 24, F32, F32, F32, "item", False))
    numbers = ("rms", None, 1.0, 0.0, 0.0)
    ts[5] = None
    want = expected(*ts, *numbers)
    # (a workgroup has up to 1203 / (51 x 8) = 3 rows in sequence, the join up to 5 x 51 partials in 16 sequences: within the 64)
    compare(run(ts, *numbers), want)
