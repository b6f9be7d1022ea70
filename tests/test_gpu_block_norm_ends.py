"""Ends of layer norm's rows: every remainder of a row's last chunk (8 channels a lane, or two fours), behind one and behind many lanes, with neighbours that must neither
enter the result nor change."""
import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from tests import block_util as ref
from tests.test_gpu_block_norm_rotary import TYPES, close, norm_inputs

pytestmark = pytest.mark.gpu


def apart(x, before, after, value):
    """x as a view of rows with `before` and `after` elements of `value` around each, and all of that."""
    room = torch.full((*x.shape[:-1], before + x.shape[-1] + after), value, dtype=x.dtype, device=x.device)
    view = room[..., before:before + x.shape[-1]]
    view.copy_(x)
    return view, room


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("base", [8, 256, 504, 1024, 1536, 2048, 2432, 2560, 4096])
def test_every_remainder(base, types):
    dtype, wdtype = TYPES[types[0]], TYPES[types[1]]
    for C in range(base, base + 9):
        x, w, b, dy = norm_inputs(1, 9, C, dtype, wdtype, False, seed=C)
        # (bounds as for the other shapes: the spread of the inputs is about 1, sums in fp32)
        leaf = [t.double().cpu().requires_grad_() for t in (x, w, b)]
        want = ref.layer_norm(*leaf, 1e-6, 0.0)
        want.backward(dy.double().cpu())
        r = 1 / torch.sqrt(((leaf[0] - leaf[0].mean(-1, keepdim=True)) ** 2).mean(-1, keepdim=True) + 1e-6).detach()
        unit = 3e-5 * torch.clamp(r, min=1.0)
        weight = leaf[1].detach().abs()
        xv, _ = apart(x, 1, 3, float("nan"))
        dv, _ = apart(dy, 2, 1, float("nan"))
        out, room = apart(torch.zeros_like(x), 3, 2, 7.0)
        _, stats = cb.layer_norm(xv, w, b, out=out, save_stats=True)
        close(out, want.detach(), unit * (weight + 1), dtype)
        assert bool((room[..., :3] == 7).all()) and bool((room[..., 3 + C:] == 7).all())
        dx, dw, db = cb.layer_norm_backward(dv, xv, w, b, stats)
        dyw = dy.double().cpu().abs() * weight
        close(dx, leaf[0].grad, r * 4 * unit * (dyw + dyw.mean(-1, keepdim=True) * (1 + torch.clamp(r, min=1.0))) * 4, dtype)
        xhat = ref.layer_norm(leaf[0].detach(), None, None, 1e-6, 0.0).abs()
        terms = dy.double().cpu().abs()
        close(dw, leaf[1].grad, (terms * (2e-5 * xhat + unit)).sum((0, 1)), wdtype)
        close(db, leaf[2].grad, 2e-5 * terms.sum((0, 1)), wdtype)
