"""Thin ctypes binding of the operators around the attention (include/clear_block.h, same library as clear_attn): rotary
positions, layer norm, gated feed-forward projection, AdamW step.  Argument marshalling only: PyTorch tensors are used for
device memory, workspaces and streams; every step runs in the HIP kernels, and there is no fallback.

Refusals raise ClearAttnError, as in clear_attn.  Each call enqueues on `stream` (default: torch's current stream of the tensors' device); with another
one the caller orders it with torch's, before the call (results are allocated for torch's stream) and after it.  These calls are not differentiable (autograd.py has
the forms that are); the tensors that a caller gives them to write into - outputs, parameters, masters - count as changed for autograd afterwards."""
import ctypes
import operator

import numpy as np
import torch

from . import clear_attn as ca
from .clear_attn import CLEAR_BF16, CLEAR_ERR_INVALID_ARG, CLEAR_ERR_MISMATCH, CLEAR_ERR_UNSUPPORTED, CLEAR_F32, CLEAR_OK, ClearAttnError  # noqa: F401

CLEAR_ROPE_PLAIN, CLEAR_ROPE_LINEAR, CLEAR_ROPE_BASE, CLEAR_ROPE_PARTS = range(4)
CLEAR_ACT_SILU, CLEAR_ACT_GELU_TANH, CLEAR_ACT_GELU_ERF = range(3)
ACTIVATIONS = {"silu": CLEAR_ACT_SILU, "gelu_tanh": CLEAR_ACT_GELU_TANH, "gelu_erf": CLEAR_ACT_GELU_ERF}
SCALINGS = {"plain": CLEAR_ROPE_PLAIN, "linear": CLEAR_ROPE_LINEAR, "base": CLEAR_ROPE_BASE, "parts": CLEAR_ROPE_PARTS}
STATE_BLOCK = 256  # elements that share a scale where AdamW's states have 8 bits

EXPORTS = [
    "clear_block_last_error", "clear_block_rotary", "clear_block_rotary_frequencies", "clear_block_layer_norm",
    "clear_block_layer_norm_backward", "clear_block_layer_norm_workspace", "clear_block_gated_ff", "clear_block_gated_ff_backward",
    "clear_block_gated_ff_workspace", "clear_block_adamw", "clear_block_adamw_decode",
]


class AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("n", ctypes.c_longlong)]


_Strides3, _Strides4, _Strides6, _Strides7, _Strides12 = (ctypes.c_longlong * n for n in (3, 4, 6, 7, 12))
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
        for name in EXPORTS:
            getattr(L, name).restype = i
        L.clear_block_last_error.restype = ctypes.c_char_p
        L.clear_block_layer_norm_workspace.restype = ll
        L.clear_block_gated_ff_workspace.restype = ll
        _lib = L
    return _lib


def _check(status):
    if status != CLEAR_OK:
        raise ClearAttnError(status, lib().clear_block_last_error().decode())


def _refuse(message, status=CLEAR_ERR_INVALID_ARG):
    raise ClearAttnError(status, message)


def _ptr(t):
    return None if t is None else t.data_ptr()


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
