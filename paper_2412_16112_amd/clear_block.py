"""Thin ctypes binding of the operators around the attention (include/clear_block.h, same library as clear_attn): rotary
positions, layer norm, gated residual with its norms, gated feed-forward projection, products of operands in 4 bits, AdamW
step, norm and clipping of gradients.  Argument marshalling only: PyTorch tensors are used for
device memory, workspaces and streams; every step runs in the HIP kernels, and there is no fallback.

Refusals raise ClearAttnError, as in clear_attn.  Each call enqueues on `stream` (default: torch's current stream of the tensors' device); with another
one the caller orders it with torch's, before the call (results are allocated for torch's stream) and after it.  These calls are not differentiable (autograd.py has
the forms that are); the tensors that a caller gives them to write into - outputs, parameters, masters - count as changed for autograd afterwards."""
import collections
import ctypes
import math
import operator

import numpy as np
import torch

from . import clear_attn as ca
from .clear_attn import CLEAR_BF16, CLEAR_ERR_INVALID_ARG, CLEAR_ERR_MISMATCH, CLEAR_ERR_UNSUPPORTED, CLEAR_F32, CLEAR_OK, ClearAttnError  # noqa: F401

CLEAR_ROPE_PLAIN, CLEAR_ROPE_LINEAR, CLEAR_ROPE_BASE, CLEAR_ROPE_PARTS = range(4)
CLEAR_ACT_SILU, CLEAR_ACT_GELU_TANH, CLEAR_ACT_GELU_ERF = range(3)
ACTIVATIONS = {"silu": CLEAR_ACT_SILU, "gelu_tanh": CLEAR_ACT_GELU_TANH, "gelu_erf": CLEAR_ACT_GELU_ERF}
SCALINGS = {"plain": CLEAR_ROPE_PLAIN, "linear": CLEAR_ROPE_LINEAR, "base": CLEAR_ROPE_BASE, "parts": CLEAR_ROPE_PARTS}
CLEAR_NORM_NONE, CLEAR_NORM_LAYER, CLEAR_NORM_RMS = range(3)
NORMS = {None: CLEAR_NORM_NONE, "layer": CLEAR_NORM_LAYER, "rms": CLEAR_NORM_RMS}
CLEAR_GRAD_NORM_2, CLEAR_GRAD_NORM_MAX = range(2)
MX_BLOCK, MX_GROUP = 32, 256  # channels that share a scale where a matrix is in 4 bits, and channels of a group of scales
STATE_BLOCK = 256  # elements that share a scale where AdamW's states have 8 bits

EXPORTS = [
    "clear_block_last_error", "clear_block_rotary", "clear_block_rotary_frequencies", "clear_block_layer_norm",
    "clear_block_layer_norm_backward", "clear_block_layer_norm_workspace", "clear_block_gated_ff", "clear_block_gated_ff_backward",
    "clear_block_gated_ff_workspace", "clear_block_adamw", "clear_block_adamw_decode", "clear_block_residual_norm",
    "clear_block_residual_norm_backward", "clear_block_residual_norm_workspace", "clear_block_grad_norm", "clear_block_grad_norm_workspace",
    "clear_block_grad_clip", "clear_block_grad_scale", "clear_block_mx_quantize", "clear_block_mx_dequantize", "clear_block_mx_linear", "clear_block_mx_linear_workspace",
]


class AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("n", ctypes.c_longlong)]


class Grad(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_longlong), ("dtype", ctypes.c_int)]


_Strides3, _Strides4, _Strides5, _Strides6, _Strides7, _Strides8, _Strides12 = (ctypes.c_longlong * n for n in (3, 4, 5, 6, 7, 8, 12))
_lib = None


def lib():
    """The loaded C library with the signatures of clear_block.h (raises if it has not been built)."""
    global _lib
    if _lib is None:
        L = ca.lib()
        i, vp, ll, f, d = ctypes.c_int, ctypes.c_void_p, ctypes.c_longlong, ctypes.c_float, ctypes.c_double
        L.clear_block_last_error.argtypes = []
        L.clear_block_rotary.argtypes = [vp, vp, i, vp, vp, i, vp, ll, ll, i, i, i, vp, i, vp, i, vp, f, i, i, vp]
        L.clear_block_rotary_frequencies.argtypes = [vp, i, d, i, d, d, d, d]
        L.clear_block_layer_norm.argtypes = [vp, vp, vp, vp, vp, ll, ll, i, vp, i, f, f, i, i, vp]
        L.clear_block_layer_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, ll, ll, i, vp, i, f, i, i, vp, vp]
        L.clear_block_layer_norm_workspace.argtypes = [ll, ll, i, i]
        L.clear_block_gated_ff.argtypes = [vp, vp, vp, vp, vp, ll, i, i, ll, ll, ll, ll, i, vp]
        L.clear_block_gated_ff_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ll, i, i, vp, i, vp, vp]
        L.clear_block_gated_ff_workspace.argtypes = [ll, i, i]
        L.clear_block_adamw.argtypes = [i, vp, i, i, d, d, d, d, d, ll, vp, vp]
        L.clear_block_adamw_decode.argtypes = [vp, vp, vp, vp, vp, vp, ll, vp]
        L.clear_block_residual_norm.argtypes = [vp] * 9 + [ll, ll, i, vp, i, i, i, i, f, f, f, f, i, i, i, vp]
        L.clear_block_residual_norm_backward.argtypes = [vp] * 14 + [ll, ll, i, vp, i, i, i, i, f, f, f, i, i, i, vp, vp]
        L.clear_block_residual_norm_workspace.argtypes = [ll, ll, i, i, i]
        L.clear_block_grad_norm.argtypes = [i, vp, i, d, vp, vp, vp, vp, vp]
        L.clear_block_grad_clip.argtypes = L.clear_block_grad_norm.argtypes
        L.clear_block_grad_norm_workspace.argtypes = [i, vp]
        L.clear_block_grad_scale.argtypes = [i, vp, vp, vp]
        L.clear_block_mx_quantize.argtypes = [vp, vp, vp, ll, i, ll, ll, ll, i, vp]
        L.clear_block_mx_dequantize.argtypes = [vp, vp, vp, ll, i, ll, ll, ll, i, vp]
        L.clear_block_mx_linear.argtypes = [vp, vp, vp, vp, vp, vp, ll, i, i, vp, i, i, i, vp, vp]
        L.clear_block_mx_linear_workspace.argtypes = [ll, i, i, i]
        for name in EXPORTS:
            getattr(L, name).restype = i
        L.clear_block_last_error.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name.endswith("_workspace"):
                getattr(L, name).restype = ll
        _lib = L
    return _lib


def _check(status):
    if status != CLEAR_OK:
        raise ClearAttnError(status, lib().clear_block_last_error().decode())


def _refuse(message, status=CLEAR_ERR_INVALID_ARG):
    raise ClearAttnError(status, message)


def _ptr(t):
    return None if t is None else t.data_ptr()


_codes = {torch.bfloat16: CLEAR_BF16, torch.float32: CLEAR_F32}


def _code(t):
    """ca._dtype_code, by a table."""
    code = _codes.get(t.dtype)
    return ca._dtype_code(t) if code is None else code


# Handle of torch's current stream of a device, without the Stream object around it (2 us a call) where torch offers that.
_current = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)  # (where there is a device tensor, the runtime has been started)


def _call(name, device, stream, *args):
    """The C function on the tensors' device and on `stream` (a handle; None: torch's current stream of that device).  Returns the stream's handle."""
    s = _current(device.index) if stream is None else stream
    f = getattr(_lib or lib(), name)
    if _current_device() == device.index:
        status = f(*args, s)
    else:
        with torch.cuda.device(device):
            status = f(*args, s)
    if status != CLEAR_OK:
        _check(status)
    return s


# A tensor that was written into counts as changed for autograd, as after one of torch's own in-place operations.
_changed = torch.autograd.graph.increment_version


def _new_like(t):
    """A new contiguous tensor of t's shape, dtype and device (half the time of torch.empty, which is given all three)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _on_device(ref, *others):
    """Refuses tensors (None skipped) that are not on ref's device, and a ref that is not on a GPU."""
    if not ref.is_cuda:
        _refuse("tensors must be device tensors")
    device = ref.get_device()
    for t in others:
        if t is not None and t.get_device() != device:
            _refuse("tensors must be on one device")


# ---- rotary positions ---------------------------------------------------------------------------------------------------

def rotary_frequencies(rot_dim, theta=10000.0, scaling="plain", factor=1.0, original_length=0.0, slow=1.0, fast=32.0, device="cpu"):
    """clear_block_rotary_frequencies: fp64 [rot_dim / 2], radians a position, of one axis.  scaling: "plain", "linear", "base", "parts"."""
    if scaling not in SCALINGS:
        _refuse("unknown scaling %r" % (scaling,))
    out = torch.empty(max(0, rot_dim // 2), dtype=torch.float64)
    _check(lib().clear_block_rotary_frequencies(out.data_ptr(), rot_dim, theta, SCALINGS[scaling], factor, original_length, slow, fast))
    return out.to(device)


def rotary(q, k, positions, freqs, interleaved=True, scale=1.0, inverse=False, out_q=None, out_k=None, stream=None):
    """clear_block_rotary: q [B, Hq, N, d] and k [B, Hk, N, d] (or None) turned by their tokens' angles; returns (q, k) turned.

    q and k may have any batch / head / token strides with contiguous channels.  positions: int32 or int64, [N], [B, N] or
    [axes, B, N] (any of the leading axes expanded); freqs: fp64 [axes, rot_dim / 2] or [rot_dim / 2].  out_q=q, out_k=k turns in place;
    by default new tensors laid out like q and k.  inverse=True is the way back, and the gradient's."""
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        _refuse("q and k must be [B, H, N, head_dim]")
    B, Hq, N, d = q.shape
    if k is not None and (k.shape[0], k.shape[2], k.shape[3], k.dtype) != (B, N, d, q.dtype):
        _refuse("q and k must agree in batch, tokens, head_dim and dtype", CLEAR_ERR_MISMATCH)
    dtype = ca._dtype_code(q)
    # (a new tensor keeps the order of a dense one's strides)
    given = [t for t in (out_q, out_k if k is not None else None) if t is not None]
    out_q = torch.empty_like(q) if out_q is None else out_q
    out_k = None if k is None else torch.empty_like(k) if out_k is None else out_k
    _on_device(q, k, out_q, out_k, positions, freqs)
    for x, y in ((q, out_q), (k, out_k)):
        if x is not None and not (y.shape == x.shape and y.dtype == x.dtype and (x.stride(3) == 1 and y.stride(3) == 1 or x.numel() == 0)):
            _refuse("an output must have its input's shape and dtype, and channels must be contiguous")
    if freqs.dim() == 1:
        freqs = freqs[None]
    if freqs.dim() != 2 or freqs.dtype != torch.float64 or not freqs.is_contiguous():
        _refuse("freqs must be a contiguous fp64 tensor [axes, rot_dim / 2]")
    axes, half = freqs.shape
    if positions.dtype not in (torch.int32, torch.int64):
        _refuse("positions must be int32 or int64")
    if positions.dim() < 1 or positions.dim() > 3 or positions.shape[-1] != N or (positions.dim() > 1 and positions.shape[-2] != B) or \
            (positions.shape[0] if positions.dim() == 3 else 1) != axes:
        _refuse("positions must be [N], [B, N] or [axes, B, N]")
    ps = [0] * (3 - positions.dim()) + list(positions.stride())
    sk = (0, 0, 0, 0, 0, 0) if k is None else (*k.stride()[:3], *out_k.stride()[:3])
    strides = _Strides12(*q.stride()[:3], *out_q.stride()[:3], *sk)
    _call("clear_block_rotary", q.device, stream, q.data_ptr(), out_q.data_ptr(), Hq, _ptr(k), _ptr(out_k), 0 if k is None else k.shape[1], strides, B, N, d,
          2 * half, int(bool(interleaved)), positions.data_ptr(), 64 if positions.dtype == torch.int64 else 32, _Strides3(*ps), axes, freqs.data_ptr(), scale,
          int(bool(inverse)), dtype)
    if given:
        _changed(given)
    return out_q, out_k


# ---- layer norm -----------------------------------------------------------------------------------------------------------

def _rows(x):
    """(groups, rows, channels) of a tensor [..., C] and a function that gives another such tensor's (group, row) strides."""
    if x.dim() < 1:
        _refuse("a tensor of at least one axis is needed")
    if x.dim() == 3:
        return x.shape[0], x.shape[1], x.shape[2]
    n = 1
    for s in x.shape[:-1]:
        n *= s
    return 1, n, x.shape[-1]


def _row_strides(t, name):
    if t.numel() == 0:  # (whatever its strides, it counts as contiguous)
        return [0, t.shape[-1]]
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s: channels must be contiguous" % name)
    if t.dim() == 3:
        return [t.stride(0), t.stride(1)]
    if t.dim() == 1:
        return [0, max(1, t.shape[0])]
    if t.dim() == 2:
        return [0, t.stride(0)]
    if not t.is_contiguous():
        _refuse("%s: a tensor of %d axes must be contiguous" % (name, t.dim()))
    return [0, t.shape[-1]]


def _norm_weights(x, weight, bias):
    """(per_group, weight dtype code): weight and bias are [C], or [B, C] for x [B, N, C]."""
    some = weight if weight is not None else bias
    for name, w in (("weight", weight), ("bias", bias)):
        if w is None:
            continue
        if w.dim() not in (1, 2) or w.shape[-1] != x.shape[-1] or (w.dim() == 2 and (x.dim() != 3 or w.shape[0] != x.shape[0])) or not w.is_contiguous():
            _refuse("%s must be contiguous, [C], or [B, C] for a tensor [B, N, C]" % name)
        if w.shape != some.shape or w.dtype != some.dtype:
            _refuse("weight and bias must agree in shape and dtype", CLEAR_ERR_MISMATCH)
    if some is None:
        return 0, CLEAR_F32
    return int(some.dim() == 2), ca._dtype_code(some)


def layer_norm(x, weight=None, bias=None, eps=1e-6, weight_offset=0.0, out=None, save_stats=False, stream=None):
    """clear_block_layer_norm over the last axis: xhat * (weight_offset + weight) + bias.

    weight and bias: [C], or [B, C] for x [B, N, C] (scale and shift per batch item; weight_offset=1 for 1 + scale).  x: bf16 or fp32, rows at
    any stride; out=x works in place.  Returns y, or (y, stats) with save_stats (fp32 [2, ...]: mean and 1/sqrt(var + eps) of every row)."""
    dtype = ca._dtype_code(x)
    groups, rows, C = _rows(x)
    per_group, wcode = _norm_weights(x, weight, bias)
    y = _new_like(x) if out is None else out
    _on_device(x, weight, bias, y)
    if y.shape != x.shape or y.dtype != x.dtype:
        _refuse("out must have the shape and dtype of x", CLEAR_ERR_MISMATCH)
    stats = torch.empty((2,) + tuple(x.shape[:-1]), dtype=torch.float32, device=x.device) if save_stats else None
    _call("clear_block_layer_norm", x.device, stream, x.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), _ptr(stats), groups, rows, C,
          _Strides4(*_row_strides(x, "x"), *_row_strides(y, "out")), per_group, eps, weight_offset, dtype, wcode)
    if out is not None:
        _changed(out)
    return (y, stats) if save_stats else y


def layer_norm_backward(dy, x, weight, bias, stats, weight_offset=0.0, need=(True, True, True), stream=None):
    """clear_block_layer_norm_backward: (dx, d_weight, d_bias) for what layer_norm(..., save_stats=True) was called with; None for a weight or bias
    that is None and where `need` says so."""
    dtype = ca._dtype_code(x)
    groups, rows, C = _rows(x)
    per_group, wcode = _norm_weights(x, weight, bias)
    _on_device(x, dy, weight, bias, stats)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        _refuse("dy must have the shape and dtype of x", CLEAR_ERR_MISMATCH)
    if stats.dtype != torch.float32 or not stats.is_contiguous() or tuple(stats.shape) != (2,) + tuple(x.shape[:-1]):
        _refuse("stats must be what layer_norm(..., save_stats=True) gave for x")
    dx = _new_like(x) if need[0] else None
    dw = _new_like(weight) if weight is not None and need[1] else None
    db = _new_like(bias) if bias is not None and need[2] else None
    if dx is None and dw is None and db is None:
        return None, None, None
    ws = None
    if dw is not None or db is not None:
        floats = lib().clear_block_layer_norm_workspace(groups, rows, C, per_group)
        if floats < 0:
            _check(CLEAR_ERR_UNSUPPORTED)
        ws = torch.empty(max(1, floats), dtype=torch.float32, device=x.device)
    strides = _Strides6(*_row_strides(dy, "dy"), *_row_strides(x, "x"), *(_row_strides(dx, "dx") if dx is not None else (0, 0)))
    s = _call("clear_block_layer_norm_backward", x.device, stream, dy.data_ptr(), x.data_ptr(), _ptr(weight), stats.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db),
              groups, rows, C, strides, per_group, weight_offset, dtype, wcode, _ptr(ws))
    if ws is not None and stream is not None:
        _record(ws, s)
    return dx, dw, db


def _record(t, stream):
    """A workspace that was used on another stream than torch's current one may not be handed out before that stream is done with it."""
    if stream != torch.cuda.current_stream(t.device).cuda_stream:
        t.record_stream(torch.cuda.ExternalStream(stream, device=t.device))


# ---- gated residual with its norms -----------------------------------------------------------------------------------------

_kinds = {"layer": CLEAR_NORM_LAYER, "rms": CLEAR_NORM_RMS}


def _residual_numbers(x, y, kind, post):
    """(kind, post, dtype, stream dtype, groups, rows, C) of a call."""
    if kind not in _kinds:
        _refuse("kind must be 'layer' or 'rms'")
    if post not in NORMS:
        _refuse("post must be None, 'layer' or 'rms'")
    if y.shape != x.shape:
        _refuse("x and y must have one shape", CLEAR_ERR_MISMATCH)
    return (_kinds[kind], NORMS[post], _code(y), _code(x)) + _rows(x)


def _residual_vectors(x, gate, weight, bias, post_weight, post):
    """(gate_per_group, per_group, weight dtype code): gate, weight and bias are [C], or [B, C] for x [B, N, C]; post_weight is [C]."""
    shape = x.shape
    one, many = shape[-1:], (shape[0], shape[2]) if len(shape) == 3 else None
    per_group, dtype = [0, 0, 0, 0], None
    for i, v in enumerate((gate, weight, bias, post_weight)):
        if v is None:
            continue
        if v.shape != one:
            if i == 3 or v.shape != many:
                _refuse("post_weight must be [C]" if i == 3 else "gate, weight and bias must be [C], or [B, C] for a tensor [B, N, C]")
            per_group[i] = 1
        if not v.is_contiguous():
            _refuse("gate, weight, bias and post_weight must be contiguous")
        if dtype is None:
            dtype = v.dtype
        elif v.dtype != dtype:
            _refuse("gate, weight, bias and post_weight must have one dtype", CLEAR_ERR_MISMATCH)
    if post_weight is not None and post is None:
        _refuse("post_weight without a post norm")
    if weight is not None and bias is not None and per_group[1] != per_group[2]:
        _refuse("weight and bias must agree in shape", CLEAR_ERR_MISMATCH)
    some = gate if gate is not None else weight if weight is not None else bias if bias is not None else post_weight
    return per_group[0], per_group[1] | per_group[2], CLEAR_F32 if some is None else _code(some)


def _strides_of(named):
    """(group, row) strides of the tensors (0, 0 for None)."""
    out = []
    for name, t in named:
        out += (0, 0) if t is None else _row_strides(t, name)
    return out


def residual_norm(x, y, gate=None, weight=None, bias=None, post_weight=None, kind="layer", post=None, eps=1e-6, residual_scale=1.0, weight_offset=0.0, post_offset=0.0,
                  out=None, save_stats=False, stream=None):
    """clear_block_residual_norm: what lies between two sublayers, x the residual stream and y a sublayer's output:
        r = residual_scale * x + gate * post(y) * (post_offset + post_weight),   h = norm(r) * (weight_offset + weight) + bias

    kind: the norm of r, post: the norm of y, "layer" or "rms" (post None: none).  gate, weight, bias: [C], or [B, C] for x [B, N, C], post_weight [C], of one dtype; each may be
    None.  x (and r) and y (and h): bf16 or fp32, rows at any stride, not x in bf16 beside y in fp32.  out: (r, h) to write to; r may be x and h may be y, else they must not share
    memory with each other, an input or a vector.  Returns (r, h), or (r, h, stats) with save_stats (for residual_norm_backward)."""
    kind_code, post_code, dtype, stream_dtype, groups, rows, C = _residual_numbers(x, y, kind, post)
    gate_per_group, per_group, wcode = _residual_vectors(x, gate, weight, bias, post_weight, post)
    r, h = (_new_like(x), _new_like(y)) if out is None else out
    _on_device(x, y, gate, weight, bias, post_weight, r, h)
    if out is None and x.is_contiguous() and y.is_contiguous():
        strides = _Strides8(*(rows * C if x.dim() == 3 else 0, C) * 4)
    else:
        if r.shape != x.shape or r.dtype != x.dtype or h.shape != y.shape or h.dtype != y.dtype:
            _refuse("out must have the shapes and dtypes of x and y", CLEAR_ERR_MISMATCH)
        strides = _Strides8(*_strides_of((("x", x), ("y", y), ("r", r), ("h", h))))
    stats = torch.empty((4 if post_code else 2,) + x.shape[:-1], dtype=torch.float32, device=x.device) if save_stats else None
    _call("clear_block_residual_norm", x.device, stream, x.data_ptr(), y.data_ptr(), _ptr(gate), _ptr(weight), _ptr(bias), _ptr(post_weight), r.data_ptr(), h.data_ptr(), _ptr(stats),
          groups, rows, C, strides, gate_per_group, per_group, kind_code, post_code, eps, residual_scale, weight_offset, post_offset, dtype, stream_dtype, wcode)
    if out is not None:
        _changed(list(out))
    return (r, h, stats) if save_stats else (r, h)


def residual_norm_backward(dr, dh, x, y, gate, weight, bias, post_weight, stats, kind="layer", post=None, residual_scale=1.0, weight_offset=0.0, post_offset=0.0,
                           need=(True,) * 6, stream=None):
    """clear_block_residual_norm_backward: (dx, dy, d_gate, d_weight, d_bias, d_post_weight) for what residual_norm(..., save_stats=True) was called with; None for a vector that is
    None and where `need` says so.  dr: the gradient of r, or None where nothing came back through it."""
    kind_code, post_code, dtype, stream_dtype, groups, rows, C = _residual_numbers(x, y, kind, post)
    gate_per_group, per_group, wcode = _residual_vectors(x, gate, weight, bias, post_weight, post)
    _on_device(x, y, dr, dh, gate, weight, bias, post_weight, stats)
    if dh.shape != y.shape or dh.dtype != y.dtype or (dr is not None and (dr.shape != x.shape or dr.dtype != x.dtype)):
        _refuse("dr and dh must have the shapes and dtypes of x and y", CLEAR_ERR_MISMATCH)
    if stats.dtype != torch.float32 or not stats.is_contiguous() or stats.shape != (4 if post_code else 2,) + x.shape[:-1]:
        _refuse("stats must be what residual_norm(..., save_stats=True) gave for x and y")
    grads = [_new_like(v) if v is not None and n else None for v, n in zip((x, y, gate, weight, bias, post_weight), need)]
    if all(g is None for g in grads):
        return tuple(grads)
    ws = None
    if any(g is not None for g in grads[2:]):
        floats = lib().clear_block_residual_norm_workspace(groups, rows, C, gate_per_group, per_group)
        if floats < 0:
            _check(CLEAR_ERR_UNSUPPORTED)
        ws = torch.empty(max(1, floats), dtype=torch.float32, device=x.device)
    if x.is_contiguous() and y.is_contiguous() and dh.is_contiguous() and (dr is None or dr.is_contiguous()):
        strides = (rows * C if x.dim() == 3 else 0, C) * 6
    else:
        strides = _strides_of((("dr", dr), ("dh", dh), ("x", x), ("y", y), ("dx", grads[0]), ("dy", grads[1])))
    s = _call("clear_block_residual_norm_backward", x.device, stream, _ptr(dr), dh.data_ptr(), x.data_ptr(), y.data_ptr(), _ptr(gate), _ptr(weight), _ptr(post_weight),
              stats.data_ptr(), *map(_ptr, grads), groups, rows, C, _Strides12(*strides), gate_per_group, per_group, kind_code, post_code, residual_scale, weight_offset,
              post_offset, dtype, stream_dtype, wcode, _ptr(ws))
    if ws is not None and stream is not None:
        _record(ws, s)
    return tuple(grads)


# ---- gated feed-forward projection ----------------------------------------------------------------------------------------

def _matrix(t, name, width):
    """(rows, row stride) of a bf16 tensor [..., width] whose leading axes are one axis of evenly spaced rows."""
    if t.dtype != torch.bfloat16:
        _refuse("%s must be bfloat16: the gated projection is built for bf16 only" % name, CLEAR_ERR_UNSUPPORTED)
    if t.dim() < 1 or t.shape[-1] != width:
        _refuse("%s must be [..., %d]" % (name, width), CLEAR_ERR_MISMATCH)
    if t.dim() != 2:
        if not t.is_contiguous():
            _refuse("%s: a tensor of %d axes must be contiguous" % (name, t.dim()))
        t = t.reshape(-1, width)
    if t.shape[0] == 0:  # (whatever its strides)
        return 0, width
    if t.stride(1) != 1:
        _refuse("%s: the last axis must be contiguous" % name)
    return t.shape[0], width if t.shape[0] <= 1 else t.stride(0)


def _activation(name):
    if name not in ACTIVATIONS:
        _refuse("unknown activation %r" % (name,))
    return ACTIVATIONS[name]


def _gated_weights(w_gate, w_up):
    if w_gate.dim() != 2 or w_up.shape != w_gate.shape:
        _refuse("w_gate and w_up must be [F, C], of one shape", CLEAR_ERR_MISMATCH)
    return w_gate.shape


def gated_ff(x, w_gate, w_up, activation="silu", out=None, save_pre=False, stream=None):
    """clear_block_gated_ff: act(x w_gate^T) * (x w_up^T) for bf16 x [..., C] and weights [F, C] (rows at any stride: halves of one packed
    [2 F, C] weight will do).  activation: "silu", "gelu_tanh", "gelu_erf".  Returns h [..., F], or (h, pre) with save_pre (fp32 [2, rows, F]: both products)."""
    act = _activation(activation)
    F, C = _gated_weights(w_gate, w_up)
    M, ld_x = _matrix(x, "x", C)
    _, ld_g = _matrix(w_gate, "w_gate", C)
    _, ld_u = _matrix(w_up, "w_up", C)
    h = x.new_empty(x.shape[:-1] + (F,)) if out is None else out
    rows, ld_h = _matrix(h, "out", F)
    if rows != M:
        _refuse("out must have a row for each of x", CLEAR_ERR_MISMATCH)
    _on_device(x, w_gate, w_up, h)
    pre = torch.empty((2, M, F), dtype=torch.float32, device=x.device) if save_pre else None
    _call("clear_block_gated_ff", x.device, stream, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), h.data_ptr(), _ptr(pre), M, C, F, ld_x, ld_g, ld_u, ld_h, act)
    if out is not None:
        _changed(out)
    return (h, pre) if save_pre else h


def gated_ff_backward(dh, x, w_gate, w_up, pre, activation="silu", need=(True, True), stream=None):
    """clear_block_gated_ff_backward: (dx, d_w_gate, d_w_up) for what gated_ff(..., save_pre=True) was called with.  need: whether dx, and whether
    the weights' gradients are wanted (None otherwise)."""
    act = _activation(activation)
    F, C = _gated_weights(w_gate, w_up)
    M, ld_x = _matrix(x, "x", C)
    rows, ld_dh = _matrix(dh, "dh", F)
    _, ld_g = _matrix(w_gate, "w_gate", C)
    _, ld_u = _matrix(w_up, "w_up", C)
    if rows != M:
        _refuse("dh must have a row for each of x", CLEAR_ERR_MISMATCH)
    if pre.dtype != torch.float32 or not pre.is_contiguous() or tuple(pre.shape) != (2, M, F):
        _refuse("pre must be what gated_ff(..., save_pre=True) gave for x")
    _on_device(x, dh, w_gate, w_up, pre)
    dx = _new_like(x) if need[0] else None
    dw = x.new_empty((2, F, C)) if need[1] else (None, None)
    if not need[0] and not need[1]:
        return None, None, None
    size = lib().clear_block_gated_ff_workspace(M, C, F)
    if size < 0:
        _check(CLEAR_ERR_UNSUPPORTED)
    ws = torch.empty(max(16, size), dtype=torch.uint8, device=x.device)
    s = _call("clear_block_gated_ff_backward", x.device, stream, dh.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), pre.data_ptr(), _ptr(dx), _ptr(dw[0]),
              _ptr(dw[1]), M, C, F, _Strides7(ld_dh, ld_x, ld_g, ld_u, C, C, C), act, ws.data_ptr())
    if stream is not None:
        _record(ws, s)
    return dx, dw[0], dw[1]


# ---- AdamW ------------------------------------------------------------------------------------------------------------------

def adamw_state(param, state_bits=32):
    """Zero states of a parameter: (m, v) fp32 of its shape, or for 8 bits (m int8, v uint8, (m_scale, v_scale) fp32 [ceil(n / 256)])."""
    if state_bits == 32:
        return torch.zeros_like(param, dtype=torch.float32), torch.zeros_like(param, dtype=torch.float32)
    if state_bits != 8:
        _refuse("state_bits must be 32 or 8")
    n = -(-param.numel() // STATE_BLOCK)
    scales = tuple(torch.zeros(n, dtype=torch.float32, device=param.device) for _ in range(2))
    return torch.zeros_like(param, dtype=torch.int8), torch.zeros_like(param, dtype=torch.uint8), scales


_dtype_of = operator.attrgetter("dtype")
_device_of, _ptr_of, _numel, _contiguous, _same_size = torch.Tensor.get_device, torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.is_same_size


def _alike(tensors, dtype, device):
    """Whether all are contiguous, of one dtype and on one device."""
    return set(map(_dtype_of, tensors)) == {dtype} and set(map(_device_of, tensors)) == {device} and all(map(_contiguous, tensors))


def _table(params, exp_avgs, exp_avg_sqs, masters, scales):
    """The descriptors of a call (rows of clear_block_adamw_tensor's eight words), gradients left out."""
    first = params[0]
    if not first.is_cuda:
        _refuse("parameters must be device tensors")
    device, n = first.get_device(), list(map(_numel, params))
    if not _alike(params, first.dtype, device):
        _refuse("the parameters of a call must be contiguous, of one dtype and on one device", CLEAR_ERR_MISMATCH)
    m_type, v_type = (torch.float32, torch.float32) if scales is None else (torch.int8, torch.uint8)
    if not (_alike(exp_avgs, m_type, device) and _alike(exp_avg_sqs, v_type, device) and list(map(_numel, exp_avgs)) == n and list(map(_numel, exp_avg_sqs)) == n):
        _refuse("states must be contiguous, on the parameters' device, of their sizes, and fp32, or int8 and uint8 with scales")
    table = np.zeros((len(n), 8), dtype=np.int64)
    places = list(map(_ptr_of, params))
    if len(set(places)) != len(places) and len(set(full := [p for p, k in zip(places, n) if k])) != len(full):
        _refuse("a parameter is there twice: it would be updated by two descriptors at once")
    table[:, 0] = places
    if masters is not None:
        if not (_alike(masters, torch.float32, device) and list(map(_numel, masters)) == n):
            _refuse("masters must be contiguous fp32, of their parameters' sizes and on their device")
        table[:, 2] = list(map(_ptr_of, masters))
    table[:, 3] = list(map(_ptr_of, exp_avgs))
    table[:, 4] = list(map(_ptr_of, exp_avg_sqs))
    if scales is not None:
        blocks = [-(-k // STATE_BLOCK) for k in n]
        for column, side in ((5, [s[0] for s in scales]), (6, [s[1] for s in scales])):
            if not (_alike(side, torch.float32, device) and list(map(_numel, side)) == blocks):
                _refuse("scales must be contiguous fp32, one for every 256 elements, on the parameters' device")
            table[:, column] = list(map(_ptr_of, side))
    table[:, 7] = n
    return table


def _set_grads(table, params, grads):
    """Writes the gradients into a table; the numbers of the parameters that have one, or None for all of them."""
    have = [g for g in grads if g is not None]
    if not have:
        table[:, 1] = 0
        return []
    of = params if len(have) == len(grads) else [p for p, g in zip(params, grads) if g is not None]
    if not (_alike(have, of[0].dtype, of[0].get_device()) and all(map(_same_size, have, of))):
        _refuse("a gradient must be contiguous and have its parameter's shape, dtype and device")
    if len(have) == len(grads):
        table[:, 1] = list(map(_ptr_of, have))
        return None
    table[:, 1] = [0 if g is None else g.data_ptr() for g in grads]
    return [i for i, g in enumerate(grads) if g is not None]


def _updated(some, *lists):
    """The parameters and masters of a call (None skipped), all or `some` of each, have been written.  (The states are in no graph.)"""
    for tensors in lists:
        if tensors is not None:
            _changed(tensors if some is None else [tensors[i] for i in some])


def _check_scale(grad_scale, device):
    if grad_scale is not None and not (grad_scale.dtype == torch.float32 and grad_scale.numel() == 1 and grad_scale.device == device):
        _refuse("grad_scale must be one fp32 value on the parameters' device")


def _launch(table, first, eight, step, lr, beta1, beta2, eps, weight_decay, grad_scale, stream):
    _call("clear_block_adamw", first.device, stream, len(table), table.ctypes.data, ca._dtype_code(first), 8 if eight else 32, lr, beta1, beta2, eps, weight_decay, step, _ptr(grad_scale))


def adamw_step(params, grads, exp_avgs, exp_avg_sqs, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, masters=None, scales=None,
               grad_scale=None, stream=None):
    """clear_block_adamw on lists of contiguous tensors, in place: params and grads of one dtype (bf16 or fp32), fp32 states, or int8 / uint8 states with
    scales [(m_scale, v_scale), ...] (adamw_state).  masters: fp32 parameters to update in the place of params, which receive them rounded.  step counts from 1.  A
    gradient that is None leaves its parameter and states as they are.  grad_scale: an fp32 device scalar that the gradients are multiplied by."""
    count = len(params)
    if not (len(grads) == len(exp_avgs) == len(exp_avg_sqs) == count) or (masters is not None and len(masters) != count) or (scales is not None and len(scales) != count):
        _refuse("the lists must have one entry for each parameter", CLEAR_ERR_MISMATCH)
    if count == 0:
        return
    table = _table(params, exp_avgs, exp_avg_sqs, masters, scales)
    some = _set_grads(table, params, grads)
    _check_scale(grad_scale, params[0].device)
    _launch(table, params[0], scales is not None, step, lr, beta1, beta2, eps, weight_decay, grad_scale, stream)
    _updated(some, params, masters)


def adamw_decode(m, m_scale, v, v_scale, stream=None):
    """clear_block_adamw_decode: the fp32 values of 8-bit states m (int8, with its scales) and v (uint8, with its scales)."""
    n = m.numel()
    blocks = -(-n // STATE_BLOCK)
    if not (m.dtype == torch.int8 and v.dtype == torch.uint8 and v.numel() == n and all(s.dtype == torch.float32 and s.numel() == blocks for s in (m_scale, v_scale))):
        _refuse("m must be int8, v uint8 of its size, scales fp32, one for every 256 elements")
    _on_device(m, v, m_scale, v_scale)
    if not all(t.is_contiguous() for t in (m, v, m_scale, v_scale)):
        _refuse("states and scales must be contiguous")
    out = [torch.empty(m.shape, dtype=torch.float32, device=m.device) for _ in range(2)]
    _call("clear_block_adamw_decode", m.device, stream, m.data_ptr(), m_scale.data_ptr(), v.data_ptr(), v_scale.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), n)
    return out[0], out[1]


# ---- norm and clipping of gradients ---------------------------------------------------------------------------------------------

def _grad_table(grads):
    """Descriptors (rows of clear_block_grad's three words) of the gradients that are there, these, and the first of them."""
    have = [g for g in grads if g is not None]
    if not have:
        _refuse("there must be a gradient")
    first = have[0]
    if not first.is_cuda:
        _refuse("tensors must be device tensors")
    if set(map(_device_of, have)) != {first.get_device()}:
        _refuse("gradients must be on one device")
    if not all(map(_contiguous, have)):
        _refuse("gradients must be contiguous")
    table = np.empty((len(have), 3), dtype=np.int64)
    table[:, 0] = list(map(_ptr_of, have))
    table[:, 1] = list(map(_numel, have))
    dtypes = list(map(_dtype_of, have))
    if dtypes.count(first.dtype) == len(dtypes):
        table[:, 2] = _code(first)
    else:
        table[:, 2] = list(map(_code, have))
    return table, have, first


def _grad_kind(norm_type):
    if norm_type not in (2, math.inf):
        _refuse("norm_type must be 2 or infinity", CLEAR_ERR_UNSUPPORTED)
    return CLEAR_GRAD_NORM_2 if norm_type == 2 else CLEAR_GRAD_NORM_MAX


def _launch_norm(name, grads, norm_type, max_norm, grad_scale, stream, factor):
    """The C function `name` on the gradients; (norm, the factor if asked for, the gradients that are there)."""
    kind = _grad_kind(norm_type)
    table, have, first = _grad_table(grads)
    device = first.device
    _check_scale(grad_scale, device)
    at = table.ctypes.data
    size = (_lib or lib()).clear_block_grad_norm_workspace(len(have), at)
    if size < 0:
        _check(CLEAR_ERR_UNSUPPORTED)
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=device)
    norm, factor, ws = new((), torch.float32), new((), torch.float32) if factor else None, new(size // 8, torch.float64)
    s = _call(name, device, stream, len(have), at, kind, 0.0 if max_norm is None else max_norm, _ptr(grad_scale), norm.data_ptr(), _ptr(factor), ws.data_ptr())
    if stream is not None:
        for t in (ws, norm, factor):  # (the factor may go to a step on that stream, and is nobody's then)
            if t is not None:
                _record(t, s)
    return norm, factor, have


def grad_norm(grads, norm_type=2.0, max_norm=None, grad_scale=None, stream=None):
    """clear_block_grad_norm: the norm of all gradients together (a list of contiguous bf16 and fp32 tensors; None is skipped), as an fp32 scalar on their device: nothing waits for
    it.  norm_type: 2 or math.inf.  grad_scale: an fp32 device scalar that the gradients are multiplied by (the inverse of a loss's scale).  With max_norm: (norm, factor), the factor
    grad_scale * min(1, max_norm / norm) (grad_scale where norm <= max_norm, be it 0 or infinite) being what adamw_step takes as its grad_scale."""
    norm, factor, _ = _launch_norm("clear_block_grad_norm", grads, norm_type, max_norm, grad_scale, stream, max_norm is not None)
    return norm if max_norm is None else (norm, factor)


def clip_grads(grads, max_norm, norm_type=2.0, grad_scale=None, stream=None):
    """clear_block_grad_clip: scales all gradients in place by grad_scale * min(1, max_norm / norm) and returns their norm, that of grad_scale times them (an fp32 scalar on their device).
    max_norm: a number >= 0; with math.inf the gradients are scaled by grad_scale alone."""
    if max_norm is None:
        _refuse("max_norm must be a number: gradients are not clipped without a bound")
    norm, _, have = _launch_norm("clear_block_grad_clip", grads, norm_type, max_norm, grad_scale, stream, False)
    _changed(have)
    return norm


def scale_grads(grads, factor, stream=None):
    """clear_block_grad_scale: every gradient times an fp32 device scalar, in place."""
    table, have, first = _grad_table(grads)
    if factor is None:
        _refuse("a factor is needed")
    _check_scale(factor, first.device)
    _call("clear_block_grad_scale", first.device, stream, len(have), table.ctypes.data, factor.data_ptr())
    _changed(have)


# ---- operands in 4 bits -----------------------------------------------------------------------------------------------------------

class MX4(collections.namedtuple("MX4", "codes scales")):
    """A matrix [..., C] in 4 bits: codes uint8 [..., C / 2], channel 2i in the low half of byte i, and scales uint8 [ceil(C / 256), rows, 8], byte [k, row, j] of channels 256 k + 32 j to + 31, standing for
    2^(byte - 127).  rows() is a range of rows, without copying."""
    __slots__ = ()

    def rows(self, first, last):
        if self.codes.dim() != 2:
            _refuse("a range of rows is one of a matrix of two axes")
        return MX4(self.codes[first:last], self.scales[:, first:last])


def _mx_groups(C):
    if C % MX_BLOCK or C == 0:
        _refuse("channels must be a multiple of %d" % MX_BLOCK, CLEAR_ERR_UNSUPPORTED)
    return -(-C // MX_GROUP)


def _mx_operand(t, name):
    """(rows, channels, bytes from row to row of codes, bytes from group to group of scales)."""
    if not isinstance(t, tuple) or len(t) != 2:
        _refuse("%s must be an MX4" % name)
    codes, scales = t
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() < 1:
        _refuse("%s: codes and scales must be uint8" % name)
    rows, ld = _any_rows(codes, name)
    C = 2 * codes.shape[-1]
    groups = _mx_groups(C)
    if scales.shape != (groups, rows, 8):
        _refuse("%s: scales must be [%d, %d, 8]" % (name, groups, rows), CLEAR_ERR_MISMATCH)
    if rows > 0 and not scales.is_contiguous() and (scales.stride(2) != 1 or (rows > 1 and scales.stride(1) != 8)):
        _refuse("%s: scales must be contiguous within a group" % name)
    return rows, C, ld, scales.stride(0)


def _any_rows(t, name):
    """(rows, row stride) of a tensor [..., C] whose leading axes are one axis of evenly spaced rows."""
    dims = t.dim()
    if dims < 1:
        _refuse("%s: a tensor of at least one axis is needed" % name)
    C = t.shape[-1]
    if t.is_contiguous():
        return (t.shape[0] if dims == 2 else t.numel() // C if C else 0), C
    if C > 1 and t.stride(-1) != 1:
        _refuse("%s: the last axis must be contiguous" % name)
    rows, ld = 1, C
    for n, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n > 1:
            if rows > 1 and stride != rows * ld:
                _refuse("%s: the rows must be evenly spaced" % name)
            rows, ld = rows * n, ld if rows > 1 else stride
    return rows, ld


def mx_quantize(x, stream=None):
    """clear_block_mx_quantize: x [..., C] (bf16 or fp32, C a multiple of 32, rows evenly spaced) to 4 bits with a scale for every 32 channels of a row: an MX4 (whole numbers: no gradient goes back
    through them)."""
    dtype = _code(x)
    _on_device(x)
    rows, ld = _any_rows(x, "x")
    C = x.shape[-1]
    groups = _mx_groups(C)
    codes = torch.empty(x.shape[:-1] + (C // 2,), dtype=torch.uint8, device=x.device)
    scales = torch.empty((groups, rows, 8), dtype=torch.uint8, device=x.device)
    _call("clear_block_mx_quantize", x.device, stream, x.data_ptr(), codes.data_ptr(), scales.data_ptr(), rows, C, ld, C // 2, 8 * rows, dtype)
    return MX4(codes, scales)


def mx_dequantize(t, dtype=torch.bfloat16, stream=None):
    """clear_block_mx_dequantize: the numbers that an MX4 stands for, in bf16 or fp32."""
    rows, C, ld, ld_scales = _mx_operand(t, "t")
    _on_device(*t)
    y = torch.empty(t[0].shape[:-1] + (C,), dtype=dtype, device=t[0].device)
    _call("clear_block_mx_dequantize", y.device, stream, t[0].data_ptr(), t[1].data_ptr(), y.data_ptr(), rows, C, ld, ld_scales, C, _code(y))
    return y


def mx_linear(x, w, bias=None, dtype=None, out=None, stream=None):
    """clear_block_mx_linear: x w^T + bias for w [F, C] in 4 bits (an MX4) and x [..., C]: an MX4, or bf16 or fp32, which the call takes to 4 bits first.  bias: [F], bf16 or fp32, or None.
    Returns [..., F] of `dtype` (bf16 by default), or out.  It has no backward pass: an x or a bias that requires a gradient is refused where gradients are on (torch.no_grad(), or detach())."""
    F, C, ld_w, ld_ws = _mx_operand(w, "w")
    if w[0].dim() != 2 or F < 1:
        _refuse("w must be [F, C], F >= 1")
    quantized = isinstance(x, tuple)
    if torch.is_grad_enabled() and ((not quantized and x.requires_grad) or (bias is not None and bias.requires_grad)):
        _refuse("no gradient goes through a 4-bit product: x and bias must not require one (torch.no_grad(), or detach())", CLEAR_ERR_UNSUPPORTED)
    if quantized:
        M, Cx, ld_x, ld_xs = _mx_operand(x, "x")
        lead, x_code, xp, xsp = x[0].shape[:-1], 0, x[0].data_ptr(), x[1].data_ptr()
    else:
        M, ld_x = _any_rows(x, "x")
        Cx, ld_xs, lead, x_code, xp, xsp = x.shape[-1], 0, x.shape[:-1], _code(x), x.data_ptr(), None
    if Cx != C:
        _refuse("x must be [..., %d]" % C, CLEAR_ERR_MISMATCH)
    if bias is not None and (bias.shape != (F,) or not bias.is_contiguous()):
        _refuse("bias must be contiguous, [%d]" % F, CLEAR_ERR_MISMATCH)
    device = w[0].device
    if out is None:
        y = torch.empty(tuple(lead) + (F,), dtype=torch.bfloat16 if dtype is None else dtype, device=device)
    else:
        y = out
        if y.shape != tuple(lead) + (F,) or (dtype is not None and y.dtype != dtype):
            _refuse("out must be %s, of the dtype asked for" % (list(lead) + [F],), CLEAR_ERR_MISMATCH)
    _on_device(w[0], w[1], bias, y, *(x if quantized else (x,)))
    _, ld_y = _any_rows(y, "out")
    out_code = _code(y)
    size = (_lib or lib()).clear_block_mx_linear_workspace(M, C, F, int(quantized))
    if size < 0:
        _check(CLEAR_ERR_UNSUPPORTED)
    ws = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    s = _call("clear_block_mx_linear", device, stream, xp, xsp, w[0].data_ptr(), w[1].data_ptr(), _ptr(bias), y.data_ptr(), M, C, F, _Strides5(ld_x, ld_xs, ld_w, ld_ws, ld_y),
              x_code, 0 if bias is None else _code(bias), out_code, _ptr(ws))
    if ws is not None and stream is not None:
        _record(ws, s)
    if out is not None:
        _changed(out)
    return y
