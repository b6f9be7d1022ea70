"""Backward calls on nothing: a tensor without elements has no address, so a gradient that is asked for and one that is not look the same."""
from paper_2412_16112_amd import clear_attn as ca
from tests.test_block_host import gated_backward, ll, norm_backward


def test_layer_norm_backward_of_no_rows():
    nothing = dict(dY=None, X=None, stats=None, dX=None, dw=None, db=None, ws=None)
    assert norm_backward(rows=0, **nothing) == ca.CLEAR_OK
    assert norm_backward(groups=0, per_group=1, **nothing) == ca.CLEAR_OK
    assert norm_backward(rows=0, **dict(nothing, w=None)) == ca.CLEAR_OK
    assert norm_backward(**dict(nothing, rows=5)) == ca.CLEAR_ERR_INVALID_ARG
    assert norm_backward(rows=0, channels=0, **nothing) == ca.CLEAR_ERR_INVALID_ARG  # (what is wrong stays wrong)


def test_gated_backward_of_no_tokens():
    nothing = dict(dH=None, X=None, pre=None, dX=None, dWg=None, dWu=None, ws=None)
    assert gated_backward(tokens=0, **nothing) == ca.CLEAR_OK
    assert gated_backward(**nothing) == ca.CLEAR_ERR_INVALID_ARG
    assert gated_backward(tokens=0, act=9, **nothing) == ca.CLEAR_ERR_INVALID_ARG
    assert gated_backward(tokens=0, **dict(nothing, dWg=1 << 32)) == ca.CLEAR_ERR_INVALID_ARG
    assert gated_backward(tokens=0, ld=ll(120, 64, 64, 64, 64, 64, 64), **nothing) == ca.CLEAR_ERR_INVALID_ARG
