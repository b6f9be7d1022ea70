"""Host-side checks of the gated residual with its norms, the gradients' norm and the operands in 4 bits that need no GPU: refusals of the C entry points before any device work (the
pointers here are numbers that nothing may follow), workspaces, refusals of the binding."""
import ctypes
import math

import pytest
import torch

from paper_2412_16112_amd import autograd as ag
from paper_2412_16112_amd import clear_attn as ca
from paper_2412_16112_amd import clear_block as cb

OK, INVALID, UNSUPPORTED = ca.CLEAR_OK, ca.CLEAR_ERR_INVALID_ARG, ca.CLEAR_ERR_UNSUPPORTED
BF, F32 = ca.CLEAR_BF16, ca.CLEAR_F32
P = [0x100000000 * i for i in range(1, 30)]  # places that are far apart


def ll(*v):
    return (ctypes.c_longlong * len(v))(*v)


def forward(**change):
    a = dict(X=P[0], Y=P[1], gate=P[2], weight=P[3], bias=P[4], post_weight=P[5], R=P[6], H=P[7], stats=P[8], groups=2, rows=10, channels=64, strides=ll(*[640, 64] * 4), gate_per_group=1,
             per_group=1, kind=1, post=2, eps=1e-6, scale=1.0, offset=0.0, post_offset=0.0, dtype=BF, stream_dtype=BF, weight_dtype=BF, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return cb.lib().clear_block_residual_norm(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(X=None), INVALID), (dict(Y=None), INVALID), (dict(R=None), INVALID), (dict(H=None), INVALID), (dict(strides=None), INVALID), (dict(groups=-1), INVALID), (dict(rows=-1), INVALID),
    (dict(channels=0), INVALID), (dict(channels=8193, strides=ll(*[81930, 8193] * 4)), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(groups=1 << 16, rows=1 << 15), UNSUPPORTED),
    (dict(kind=0), INVALID), (dict(kind=3), INVALID), (dict(post=-1), INVALID), (dict(post=3), INVALID), (dict(post=0), INVALID), (dict(dtype=2), INVALID), (dict(stream_dtype=2), INVALID),
    (dict(weight_dtype=-1), INVALID), (dict(dtype=F32), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(offset=math.nan), INVALID),
    (dict(post_offset=math.inf), INVALID), (dict(X=P[0] + 1), INVALID), (dict(H=P[7] + 1), INVALID), (dict(gate=P[2] + 1), INVALID), (dict(stats=P[8] + 2), INVALID),
    (dict(stream_dtype=F32, R=P[6] + 2), INVALID), (dict(strides=ll(640, 64, 640, 64, 640, 63, 640, 64)), INVALID), (dict(strides=ll(640, 64, 640, 64, 600, 64, 640, 64)), INVALID),
    (dict(strides=ll(640, 64, 640, 64, 640, 64, 640, -64)), INVALID), (dict(strides=ll(1 << 49, 64, 640, 64, 640, 64, 640, 64)), UNSUPPORTED), (dict(R=P[1]), INVALID), (dict(H=P[0]), INVALID),
    (dict(R=P[0] + 128), INVALID), (dict(H=P[6]), INVALID), (dict(R=P[0], strides=ll(640, 64, 640, 64, 1280, 128, 640, 64)), INVALID), (dict(stream_dtype=F32, H=P[0] + 64), INVALID),
    (dict(groups=0, X=None), OK), (dict(rows=0, R=None), OK),
])
def test_forward_refusals(change, status):
    assert forward(**change) == status
    assert status == OK or cb.lib().clear_block_last_error()


def backward(**change):
    a = dict(dR=P[0], dH=P[1], X=P[2], Y=P[3], gate=P[4], weight=P[5], post_weight=P[6], stats=P[7], dX=P[8], dY=P[9], d_gate=P[10], d_weight=P[11], d_bias=P[12], d_post_weight=P[13],
             groups=2, rows=10, channels=64, strides=ll(*[640, 64] * 6), gate_per_group=1, per_group=1, kind=1, post=2, scale=1.0, offset=0.0, post_offset=0.0, dtype=BF, stream_dtype=BF,
             weight_dtype=BF, workspace=P[14], stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return cb.lib().clear_block_residual_norm_backward(*a.values())


NONE_WANTED = dict(dX=None, dY=None, d_gate=None, d_weight=None, d_bias=None, d_post_weight=None)


@pytest.mark.parametrize("change,status", [
    (dict(dH=None), INVALID), (dict(X=None), INVALID), (dict(Y=None), INVALID), (dict(stats=None), INVALID), (dict(workspace=None), INVALID), (dict(strides=None), INVALID), (NONE_WANTED, INVALID),
    (dict(gate=None), INVALID), (dict(weight=None), INVALID), (dict(post_weight=None), INVALID), (dict(post=0), INVALID), (dict(kind=7), INVALID), (dict(groups=65536, rows=1), UNSUPPORTED),
    (dict(dtype=F32), UNSUPPORTED), (dict(channels=9000), UNSUPPORTED), (dict(dX=P[8] + 1), INVALID), (dict(workspace=P[14] + 2), INVALID), (dict(dX=P[2]), INVALID), (dict(dX=P[1]), INVALID), (dict(dY=P[0]), INVALID),
    (dict(dY=P[3]), INVALID), (dict(dX=P[9]), INVALID), (dict(dX=P[0] + 128), INVALID), (dict(strides=ll(*[640, 64] * 4, 640, 60, 640, 64)), INVALID), (dict(scale=math.nan), INVALID),
    (dict(rows=0, **NONE_WANTED), OK), (dict(groups=0, gate=P[4], d_bias=None, d_post_weight=None), OK),
])
def test_backward_refusals(change, status):
    assert backward(**change) == status


def test_residual_workspaces():
    size = cb.lib().clear_block_residual_norm_workspace
    assert size(1, 1000, 64, 0, 0) > 0 and size(4, 1000, 64, 1, 0) > 0 and size(0, 5, 64, 1, 1) == 0 and size(3, 0, 64, 0, 0) == 0
    assert size(1, 1000, 8193, 0, 0) == -1 and size(-1, 1, 8, 0, 0) == -1 and size(1, 1 << 31, 8, 0, 0) == -1


def grads(*tensors):
    return (cb.Grad * len(tensors))(*tensors)


SOME = [(P[0], 1000, BF), (P[1], 33, F32)]


def norm(name="clear_block_grad_norm", **change):
    a = dict(n=2, tensors=grads(*SOME), kind=0, max_norm=1.0, unscale=P[2], norm=P[3], factor=P[4], workspace=P[5], stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return getattr(cb.lib(), name)(*a.values())


NORM_REFUSALS = [
    (dict(n=-1), INVALID), (dict(tensors=None), INVALID), (dict(kind=2), INVALID), (dict(max_norm=-1.0), INVALID), (dict(max_norm=math.nan), INVALID), (dict(workspace=None), INVALID),
    (dict(unscale=P[2] + 1), INVALID), (dict(norm=P[3] + 2), INVALID), (dict(factor=P[4] + 1), INVALID), (dict(workspace=P[5] + 4), INVALID), (dict(tensors=grads((P[0], -1, BF), SOME[1])), INVALID),
    (dict(tensors=grads((P[0], (1 << 35) + 1, BF), SOME[1])), UNSUPPORTED), (dict(tensors=grads((P[0], 5, 2), SOME[1])), INVALID), (dict(tensors=grads((P[0] + 1, 5, BF), SOME[1])), INVALID),
    (dict(tensors=grads((P[0] + 2, 5, F32), SOME[1])), INVALID),
]


@pytest.mark.parametrize("change,status", NORM_REFUSALS + [(dict(norm=None, factor=None), INVALID)])
def test_norm_refusals(change, status):
    assert norm(**change) == status


@pytest.mark.parametrize("change,status", NORM_REFUSALS + [
    (dict(tensors=grads((P[0], 100, BF), (P[0], 5, F32))), INVALID), (dict(tensors=grads((P[0], 100, BF), (P[0] + 196, 5, F32))), INVALID), (dict(tensors=grads((P[0] + 40, 100, BF), (P[0], 11, F32))), INVALID),
])
def test_clip_refusals(change, status):
    assert norm("clear_block_grad_clip", **change) == status


@pytest.mark.parametrize("change", [
    dict(unscale=P[0] + 100), dict(unscale=P[1] + 4 * 32), dict(norm=P[0] + 1996), dict(factor=P[1]), dict(norm=P[2]), dict(factor=P[2]), dict(norm=P[4]), dict(workspace=P[0]), dict(workspace=P[1] + 128),
    dict(tensors=grads(SOME[0], (P[5] + 8, 3, F32))),
])
def test_clip_refuses_scalars_and_partials_among_the_gradients(change):
    assert norm("clear_block_grad_clip", **change) == INVALID


@pytest.mark.parametrize("factor", [P[0], P[0] + 1996, P[1] + 128])
def test_scale_refuses_a_factor_among_the_gradients(factor):
    assert cb.lib().clear_block_grad_scale(2, grads(*SOME), factor, None) == INVALID


@pytest.mark.parametrize("n,tensors,factor,status", [
    (2, grads(*SOME), None, INVALID), (2, grads(*SOME), P[3] + 2, INVALID), (-1, grads(*SOME), P[3], INVALID), (2, None, P[3], INVALID), (2, grads((P[0], 100, BF), (P[0] + 198, 5, BF)), P[3], INVALID),
    (0, None, P[3], OK), (2, grads((P[0], 0, BF), (None, 7, F32)), P[3], OK),
])
def test_scale_refusals(n, tensors, factor, status):
    assert cb.lib().clear_block_grad_scale(n, tensors, factor, None) == status


def test_norm_workspaces():
    size = cb.lib().clear_block_grad_norm_workspace
    assert size(2, grads(*SOME)) > 0 and size(0, None) == 0 and size(1, grads((P[0], 0, BF))) == 0 and size(1, grads((P[0], -1, BF))) == -1
    many = grads(*[(P[0] + 64 * i, 7, F32) for i in range(500)])
    assert size(500, many) == 500 * 8


def quantize(**change):
    a = dict(X=P[0], codes=P[1], scales=P[2], rows=10, channels=512, ld_x=512, ld_codes=256, ld_scales=80, dtype=BF, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return cb.lib().clear_block_mx_quantize(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(X=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(rows=-1), INVALID), (dict(channels=0), INVALID), (dict(channels=48), UNSUPPORTED),
    (dict(channels=(1 << 20) + 32), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(X=P[0] + 1), INVALID), (dict(codes=P[1] + 8), INVALID), (dict(scales=P[2] + 4), INVALID),
    (dict(ld_codes=240), INVALID), (dict(ld_codes=264), UNSUPPORTED), (dict(ld_codes=(1 << 20) + 16), UNSUPPORTED), (dict(ld_scales=72), INVALID), (dict(ld_scales=84), UNSUPPORTED),
    (dict(ld_scales=1 << 36), UNSUPPORTED), (dict(ld_x=-1), INVALID), (dict(ld_x=(1 << 32) + 1), UNSUPPORTED), (dict(codes=P[0] + 512), INVALID), (dict(scales=P[1] + 1024), INVALID), (dict(rows=0, X=None), OK),
])
def test_quantize_refusals(change, status):
    assert quantize(**change) == status


def dequantize(**change):
    a = dict(codes=P[1], scales=P[2], Y=P[0], rows=10, channels=512, ld_codes=256, ld_scales=80, ld_y=512, dtype=F32, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return cb.lib().clear_block_mx_dequantize(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(Y=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(channels=16), UNSUPPORTED), (dict(ld_y=500), INVALID), (dict(Y=P[0] + 2), INVALID), (dict(Y=P[1]), INVALID),
    (dict(Y=P[2] - 4), INVALID), (dict(dtype=-1), INVALID), (dict(ld_codes=128), INVALID), (dict(rows=0), OK),
])
def test_dequantize_refusals(change, status):
    assert dequantize(**change) == status


def linear(**change):
    a = dict(X=P[0], X_scales=P[1], W=P[2], W_scales=P[3], bias=P[4], Y=P[5], tokens=10, channels=512, outputs=33, strides=ll(256, 80, 256, 264, 33), x_dtype=BF, bias_dtype=BF, out_dtype=BF, workspace=P[6],
             stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return cb.lib().clear_block_mx_linear(*a.values())


PLAIN_X = dict(X_scales=None, strides=ll(512, 0, 256, 264, 33))


@pytest.mark.parametrize("change,status", [
    (dict(X=None), INVALID), (dict(W=None), INVALID), (dict(W_scales=None), INVALID), (dict(Y=None), INVALID), (dict(strides=None), INVALID), (dict(tokens=-1), INVALID), (dict(outputs=0), INVALID),
    (dict(outputs=(1 << 20) + 1), UNSUPPORTED), (dict(channels=500), UNSUPPORTED), (dict(bias_dtype=3), INVALID), (dict(out_dtype=3), INVALID), (dict(PLAIN_X, x_dtype=3), INVALID), (dict(Y=P[5] + 1), INVALID),
    (dict(bias=P[4] + 1), INVALID), (dict(W=P[2] + 8), INVALID), (dict(X=P[0] + 8), INVALID), (dict(PLAIN_X, X=P[0] + 1), INVALID), (dict(strides=ll(256, 80, 256, 264, 32)), INVALID),
    (dict(strides=ll(256, 80, 250, 264, 33)), INVALID), (dict(strides=ll(256, 80, 264, 264, 33)), UNSUPPORTED), (dict(strides=ll(256, 80, 256, 256, 33)), INVALID), (dict(strides=ll(256, 72, 256, 264, 33)), INVALID),
    (dict(strides=ll(256, 80, 256, 264, (1 << 32) + 1)), UNSUPPORTED), (dict(PLAIN_X, workspace=None), INVALID), (dict(workspace=P[6] + 8), INVALID), (dict(Y=P[0]), INVALID), (dict(Y=P[1]), INVALID),
    (dict(Y=P[2]), INVALID), (dict(Y=P[3] + 16), INVALID), (dict(Y=P[4] - 2), INVALID), (dict(tokens=0, X=None), OK),
])
def test_linear_refusals(change, status):
    assert linear(**change) == status


def test_linear_workspaces():
    size = cb.lib().clear_block_mx_linear_workspace
    assert size(0, 512, 64, 0) == 0 and size(4, 512, 64, 0) == 0 and size(5, 512, 64, 0) > 0 and size(5, 512, 64, 1) == 0
    assert size(10, 500, 64, 0) == -1 and size(10, 512, 0, 0) == -1 and size(1 << 31, 512, 64, 0) == -1
    assert size(100, 8192, 130, 1) > 0  # (a long contraction and few outputs: in parts)


X, V = torch.zeros(2, 3, 64), torch.zeros(64)
MX = cb.MX4(torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(1, 5, 8, dtype=torch.uint8))


@pytest.mark.parametrize("bad", [
    lambda: cb.residual_norm(X, X[:1]), lambda: cb.residual_norm(X, X, kind="batch"), lambda: cb.residual_norm(X, X, kind=None), lambda: cb.residual_norm(X, X, post="group"), lambda: cb.residual_norm(X, X, gate=V[:63]),
    lambda: cb.residual_norm(X, X, weight=torch.zeros(3, 64)), lambda: cb.residual_norm(X, X, weight=torch.zeros(2, 64), bias=V), lambda: cb.residual_norm(X, X, V, V.bfloat16()),
    lambda: cb.residual_norm(X, X, post_weight=V), lambda: cb.residual_norm(X, X, post_weight=torch.zeros(2, 64), post="rms"), lambda: cb.residual_norm(X, X, gate=torch.zeros(64, 2)[:, 0]),
    lambda: cb.residual_norm(X.half(), X.half()), lambda: cb.residual_norm(X, X), lambda: cb.residual_norm(torch.tensor(1.0), torch.tensor(1.0)), lambda: ag.residual_norm(X, X),
    lambda: cb.residual_norm_backward(X, X, X, X, None, None, None, None, X), lambda: cb.grad_norm([]), lambda: cb.grad_norm([None]), lambda: cb.grad_norm([V]), lambda: cb.grad_norm([V], norm_type=1),
    lambda: cb.clip_grads([V], 1.0), lambda: cb.scale_grads([V], V[0]), lambda: cb.mx_quantize(X), lambda: cb.mx_dequantize(MX), lambda: cb.mx_dequantize(X), lambda: cb.mx_dequantize((X, X)),
    lambda: cb.mx_dequantize(cb.MX4(MX.codes, MX.scales[:, :4])), lambda: cb.mx_dequantize(cb.MX4(MX.codes[:, :20], MX.scales)), lambda: cb.mx_dequantize(cb.MX4(MX.codes.t(), MX.scales)),
    lambda: cb.MX4(MX.codes[None], MX.scales).rows(0, 1), lambda: cb.MX4(MX.codes[0], MX.scales[:, :1]).rows(0, 16),
    lambda: cb.mx_linear(X, MX), lambda: cb.mx_linear(X, X), lambda: cb.mx_linear(X[..., :32], MX), lambda: cb.mx_linear(MX, MX), lambda: cb.mx_linear(X, MX, bias=V),
])
def test_binding_refusals(bad):
    with pytest.raises(ca.ClearAttnError):
        bad()


def test_rows_of_tensors_of_many_axes():
    t = torch.zeros(3, 4, 5, 96)
    assert cb._any_rows(t, "t") == (60, 96) and cb._any_rows(t[..., 32:64], "t") == (60, 96) and cb._any_rows(t[:, :, 2, :32], "t") == (12, 480) and cb._any_rows(t[:, 1:2, 3:4, :64], "t") == (3, 1920)
    assert cb._any_rows(t[1, 2, 3:4, :32], "t") == (1, 32) and cb._any_rows(t[0, 0, 0], "t") == (1, 96) and cb._any_rows(t[:0, :, :, :32], "t")[0] == 0
    assert cb._any_rows(t[:1, :1, :1, :32].expand(3, 4, 5, 32), "t") == (60, 0)
    for bad in (t[:, 1:3, :, :32], t.transpose(0, 1), t[:, :, :2], t.expand(2, 3, 4, 5, 96)[..., :32], t[..., ::2]):
        with pytest.raises(ca.ClearAttnError):
            cb._any_rows(bad, "t")
