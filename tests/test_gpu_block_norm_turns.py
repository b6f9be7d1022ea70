"""Layer norm's backward pass where a workgroup goes through several turns of rows, the last of them ragged: what is fetched ahead, the sums over turns, the rows that are not there.

Tolerances are test_gpu_block_norm_rotary's: a weight's gradient is a sum of at most 40 turns in a register, 16 teams and 256 partials in fours of 64, under 100 roundings (6e-6) of
the terms' magnitudes on top of the error of their xhat."""
import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from tests import block_util as ref
from tests.test_gpu_block_norm_rotary import TYPES, norm_inputs

pytestmark = pytest.mark.gpu

TURNS = [  # B, N, C: rows for every number of waves and chunks that a row takes, filling its last chunk and not
    (2, 4501, 40), (1, 9001, 512), (1, 4700, 1000), (1, 4700, 1024), (2, 2350, 1111), (1, 4503, 1536), (2, 1500, 1700), (2, 1501, 2048), (2, 1500, 2432), (1, 2601, 3072),
    (1, 1100, 3100), (3, 701, 4096), (1, 1101, 5000), (1, 1500, 6144), (1, 700, 7000), (3, 301, 8192), (2, 400, 9001), (1, 601, 12288), (1, 600, 12345), (2, 303, 16384),
]


def close(got, want, slack, dtype):
    bound = slack + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
    off = (got.double() - want).abs()
    assert not bool((~(off <= bound)).any()), "%d off, largest %g of %g" % (int((~(off <= bound)).sum()), float(off.max()), float(want.abs().max()))


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("shape", TURNS)
def test_several_turns(shape, types):
    B, N, C = shape
    for per_item, offset in [(False, 0.0), (True, 1.0)]:
        x, w, b, dy = norm_inputs(B, N, C, TYPES[types[0]], TYPES[types[1]], per_item, seed=C + N)
        _, stats = cb.layer_norm(x, w, b, weight_offset=offset, save_stats=True)
        leaf = [t.double().requires_grad_() for t in (x, w, b)]
        ref.layer_norm(*leaf, 1e-6, offset).backward(dy.double())
        dx, dw, db = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset)
        centred = leaf[0].detach() - leaf[0].detach().mean(-1, keepdim=True)
        r = 1 / torch.sqrt(centred.square().mean(-1, keepdim=True) + 1e-6)
        unit = 3e-5 * torch.clamp(r, min=1.0)
        weight = (offset + leaf[1].detach()).abs()
        terms = dy.double().abs()
        dyw = terms * (weight.unsqueeze(1) if per_item else weight)
        close(dx, leaf[0].grad, r * 4 * unit * (dyw + dyw.mean(-1, keepdim=True) * (1 + torch.clamp(r, min=1.0))) * 4, x.dtype)
        rows = 1 if per_item else (0, 1)
        close(dw, leaf[1].grad, (terms * (2e-5 * (centred * r).abs() + unit)).sum(rows), w.dtype)
        close(db, leaf[2].grad, 2e-5 * terms.sum(rows), w.dtype)
        again = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset)
        assert all(torch.equal(s, t) for s, t in zip((dx, dw, db), again))
        parts = cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset, need=(False, True, True)), cb.layer_norm_backward(dy, x, w, b, stats, weight_offset=offset, need=(True, False, False))
        assert torch.equal(parts[0][1], dw) and torch.equal(parts[0][2], db) and torch.equal(parts[1][0], dx)
        # rows elsewhere, with neighbours that must not enter
        wide = torch.full((B, N, C + 3), float("nan"), dtype=x.dtype, device="cuda")[..., 1:C + 1]
        wide.copy_(x)
        assert all(torch.equal(s, t) for s, t in zip((dx, dw, db), cb.layer_norm_backward(dy, wide, w, b, stats, weight_offset=offset)))
