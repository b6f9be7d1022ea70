"""The gated residual's backward pass through the C entry point with dX on dR's place and dY on dH's, bit for bit what it gives beside them.  At widths that are no whole chunks a lane's load reaches back over elements that
its neighbour stores; every workgroup has several rows, the next of which may be under way while one is stored."""
import itertools

import pytest
import torch

from paper_2412_16112_amd import clear_block as cb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# (width, rows of each of two items: over two turns of 256 workgroups, which have 16 teams of waves at most at the narrow widths and one at the wide ones)
SIZES = [(5, 4500), (300, 4500), (511, 4500), (2432, 900), (5003, 400), (8190, 400), (8192, 400)]


def backward(dr, dh, x, y, gate, weight, pw, stats, dx, dy, post, wanted):
    B, N, C = x.shape
    vectors = [torch.empty_like(v) if v is not None else None for v in (gate, weight, weight, pw)] if wanted else [None] * 4
    floats = cb.lib().clear_block_residual_norm_workspace(B, N, C, int(gate.dim() == 2), 0)
    ws = torch.empty(floats, dtype=F32, device="cuda")
    strides = cb._Strides12(*(s for t in (dr, dh, x, y, dx, dy) for s in t.stride()[:2]))
    cb._call("clear_block_residual_norm_backward", x.device, None, dr.data_ptr(), dh.data_ptr(), x.data_ptr(), y.data_ptr(), gate.data_ptr(), weight.data_ptr(), cb._ptr(pw), stats.data_ptr(),
             dx.data_ptr(), dy.data_ptr(), *map(cb._ptr, vectors), B, N, C, strides, int(gate.dim() == 2), 0, cb.CLEAR_NORM_LAYER, cb.NORMS[post], 0.75, 1.0, 0.5, cb._code(y), cb._code(x),
             cb._code(gate), ws.data_ptr())
    return vectors


@pytest.mark.parametrize("C,N", SIZES)
@pytest.mark.parametrize("dtype,stream", [(BF, BF), (BF, F32), (F32, F32)], ids=["bf16", "mixed", "fp32"])
@pytest.mark.parametrize("post,layout", [(None, "apart"), ("layer", "apart"), ("rms", "together")])
def test_gradients_on_the_places_of_what_came_back(C, N, dtype, stream, post, layout):
    g = torch.Generator(device="cuda").manual_seed(C)
    draw = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    x, y, dr, dh = draw(2, N, C).to(stream), draw(2, N, C).to(dtype), draw(2, N, C).to(stream), draw(2, N, C).to(dtype)
    gate, weight, pw = draw(2, C) if layout == "apart" else draw(C), draw(C), draw(C) if post else None
    stats = cb.residual_norm(x, y, gate, weight, weight, pw, post=post, residual_scale=0.75, weight_offset=1.0, post_offset=0.5, save_stats=True)[2]
    dx, dy = torch.empty_like(x), torch.empty_like(y)
    want = [dx, dy, *backward(dr, dh, x, y, gate, weight, pw, stats, dx, dy, post, True)]

    def room(t, k):
        """(t in rows of a buffer that leave k elements between them, the items' rows in turn, off alignment; the buffer)."""
        if layout == "together":
            return t.clone(), None
        flat = torch.full((N, 2, C + k), 7.0, dtype=t.dtype, device="cuda")
        return flat[..., k:].transpose(0, 1).copy_(t), flat
    for wanted in (True, False):
        (r, r_flat), (h, h_flat) = room(dr, 3), room(dh, 1)
        got = [r, h, *backward(r, h, x, y, gate, weight, pw, stats, r, h, post, wanted)]
        for name, a, b in zip(("dx", "dy", "gate", "weight", "bias", "post weight"), got, want):
            assert a is None and (b is None or not wanted) or torch.equal(a, b), name
        for flat, k in ((r_flat, 3), (h_flat, 1)):
            assert flat is None or bool((flat[..., :k] == 7).all())


@pytest.mark.parametrize("alone", ["dx", "dy"])
def test_one_of_them_alone(alone):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, y, dr, dh = (torch.randn(2, 900, 2430, generator=g, device="cuda").to(BF) for _ in range(4))
    gate = torch.randn(2430, generator=g, device="cuda")
    stats = cb.residual_norm(x, y, gate, gate, gate, save_stats=True, residual_scale=0.75, weight_offset=1.0)[2]
    dx, dy = torch.empty_like(x), torch.empty_like(y)
    want = backward(dr, dh, x, y, gate, gate, None, stats, dx, dy, None, True)
    r, h = dr.clone(), dh.clone()
    to = (r, torch.empty_like(y)) if alone == "dx" else (torch.empty_like(x), h)
    got = backward(r, h, x, y, gate, gate, None, stats, *to, None, True)
    assert torch.equal(to[0], dx) and torch.equal(to[1], dy)
    assert all(torch.equal(a, b) for a, b in itertools.zip_longest(got[:3], want[:3]))
