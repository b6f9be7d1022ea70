"""torch.autograd entry points for the CLEAR local attention and for the operators around it - rotary, layer_norm, residual_norm, gated_ff -
(argument marshalling only: forward and backward both run in the HIP library).

    from paper_2412_16112_amd.autograd import clear_attention
    O = clear_attention(Q, K, V, n_text=512, gridH=64, gridW=64, r=16)   # [B, H, N, 128] bf16, differentiable

Contexts (tile schedule, mask table, workspaces) are cached per (device, shape, mask); the cache keeps the
`MAX_CACHED_CONTEXTS` most recently used ones (an evicted context is destroyed once no pending backward holds it) and
`clear_context_cache()` empties it.  Gradients need bf16 tensors: the backward kernels are built for bf16 only, and
a call that asks for gradients of fp32 tensors is refused in the forward pass, not later inside `loss.backward()`.
Gradients are first-order: a gradient of a gradient (create_graph=True and a loss on it) raises.
"""
import torch
from torch.autograd.function import once_differentiable

from . import clear_attn as ca
from . import clear_block as cb

MAX_CACHED_CONTEXTS = 16
_contexts = {}  # insertion order = least recently used first


def _context(device, n_text, gridH, gridW, head_dim, r, dtype_code, mask_kind=ca.CLEAR_MASK_DISC, shift=0):
    key = (device.index, n_text, gridH, gridW, head_dim, r, dtype_code, mask_kind, shift)
    ctx = _contexts.pop(key, None)
    if ctx is None:
        with torch.cuda.device(device):
            ctx = ca.ClearAttn(n_text, gridH, gridW, head_dim, r, dtype_code, mask_kind, shift)
    _contexts[key] = ctx  # most recently used last
    while len(_contexts) > MAX_CACHED_CONTEXTS:
        # dropped, not destroyed: a saved-for-backward reference may still use it; ClearAttn.__del__ frees it with
        # the last reference (its kernels have been enqueued by then, and the free waits for the device)
        _contexts.pop(next(iter(_contexts)))
    return ctx


def clear_context_cache():
    _contexts.clear()


def _no_gradients(*tensors):
    """Whether a call on these tensors (None skipped) needs no backward pass.  To be asked outside the Function: inside its forward gradients are off, and needs_input_grad
    says what the tensors want, whatever the caller's mode."""
    return not (torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors))


class ClearAttentionFunction(torch.autograd.Function):
    @staticmethod
    def forward(fctx, Q, K, V, n_text, gridH, gridW, r, mask_kind=ca.CLEAR_MASK_DISC, shift=0):
        # bf16 tensors go in with whatever batch / head / token strides they have (transposed views of a projection's
        # [B, N, H, d] output included); only the channels must be contiguous
        strided = Q.dtype == torch.bfloat16
        if any(fctx.needs_input_grad[:3]) and not strided:
            raise ca.ClearAttnError(ca.CLEAR_ERR_UNSUPPORTED, "gradients need bf16 tensors: the backward pass is built for bf16 only "
                                    "(detach the fp32 inputs or cast them to bfloat16)")
        fix = (lambda t: t if t.stride(-1) == 1 else t.contiguous()) if strided else (lambda t: t.contiguous())
        Q, K, V = fix(Q), fix(K), fix(V)
        ctx = _context(Q.device, n_text, gridH, gridW, Q.shape[-1], r, ca._dtype_code(Q), mask_kind, shift)
        needs_grad = any(fctx.needs_input_grad[:3])
        with torch.cuda.device(Q.device):
            if strided:
                lse = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device) if needs_grad else None
                O = ctx.forward_strided(Q, K, V, lse=lse)
            elif needs_grad:
                O, lse = ctx.forward_lse(Q, K, V)
            else:
                O = ctx.forward(Q, K, V)
            if needs_grad:
                fctx.save_for_backward(Q, K, V, O, lse)
                fctx.clear_ctx = ctx
        return O

    @staticmethod
    @once_differentiable
    def backward(fctx, dO):
        Q, K, V, O, lse = fctx.saved_tensors
        dO = dO.to(Q.dtype)
        with torch.cuda.device(Q.device):
            if Q.dtype == torch.bfloat16:
                dQ, dK, dV = fctx.clear_ctx.backward_strided(Q, K, V, O, dO if dO.stride(-1) == 1 else dO.contiguous(), lse)
            else:
                dQ, dK, dV = fctx.clear_ctx.backward(Q, K, V, O, dO.contiguous(), lse)
        return dQ, dK, dV, None, None, None, None, None, None


def clear_attention(Q, K, V, n_text, gridH, gridW, r, mask_kind=ca.CLEAR_MASK_DISC, shift=0):
    """softmax(Q K^T / sqrt(d) under the CLEAR mask) V for [B, H, n_text + gridH*gridW, d] device tensors.
    mask_kind / shift select one of the compared local masks instead of the disc (clear_attn_create_masked)."""
    if _no_gradients(Q, K, V):
        Q, K, V = Q.detach(), K.detach(), V.detach()
    return ClearAttentionFunction.apply(Q, K, V, n_text, gridH, gridW, r, mask_kind, shift)


# ---- the operators around the attention (clear_block) -------------------------------------------------------------------------

def _channels_ok(t):
    """t (or None), or a contiguous copy where its channels are not."""
    return t if t is None or (t.dim() > 0 and t.stride(-1) == 1) else t.contiguous()


class RotaryFunction(torch.autograd.Function):
    @staticmethod
    def forward(fctx, q, k, positions, freqs, interleaved, scale):
        fctx.save_for_backward(positions, freqs)
        fctx.how = (interleaved, scale)
        fctx.has_k = k is not None
        return cb.rotary(q, k, positions, freqs, interleaved=interleaved, scale=scale)

    @staticmethod
    @once_differentiable
    def backward(fctx, dq, dk):
        positions, freqs = fctx.saved_tensors
        interleaved, scale = fctx.how
        # (the transposed map: the negative angle, the same scale)
        dq, dk = cb.rotary(_channels_ok(dq), _channels_ok(dk) if fctx.has_k else None, positions, freqs, interleaved=interleaved, scale=scale, inverse=True)
        return dq, dk, None, None, None, None


def rotary(q, k, positions, freqs, interleaved=True, scale=1.0):
    """clear_block.rotary, differentiable in q and k (k may be None)."""
    return RotaryFunction.apply(_channels_ok(q), _channels_ok(k), positions, freqs, interleaved, scale)


class LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(fctx, x, weight, bias, eps, weight_offset):
        y, stats = cb.layer_norm(x, weight, bias, eps=eps, weight_offset=weight_offset, save_stats=True)
        fctx.save_for_backward(x, weight, bias, stats)
        fctx.weight_offset = weight_offset
        return y

    @staticmethod
    @once_differentiable
    def backward(fctx, dy):
        x, weight, bias, stats = fctx.saved_tensors
        dx, dw, db = cb.layer_norm_backward(_rows_ok(dy), x, weight, bias, stats, weight_offset=fctx.weight_offset, need=fctx.needs_input_grad[:3])
        return dx, dw, db, None, None


def _rows_ok(t):
    """t, or a contiguous copy where its rows are not evenly spaced or its channels not contiguous (an expanded gradient, say)."""
    return t if t.dim() in (2, 3) and t.stride(-1) == 1 else t.contiguous()


def layer_norm(x, weight=None, bias=None, eps=1e-6, weight_offset=0.0):
    """clear_block.layer_norm, differentiable in x, weight and bias."""
    own = lambda t: t if t is None else t.contiguous()
    x, weight, bias = _rows_ok(x), own(weight), own(bias)
    if _no_gradients(x, weight, bias):
        return cb.layer_norm(x, weight, bias, eps=eps, weight_offset=weight_offset)
    if any(w is not None and w.dim() == 2 and w.shape[0] > 65535 for w in (weight, bias)):
        raise ca.ClearAttnError(ca.CLEAR_ERR_UNSUPPORTED, "gradients: at most 65535 items with a weight each")
    return LayerNormFunction.apply(x, weight, bias, eps, weight_offset)


class ResidualNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(fctx, x, y, gate, weight, bias, post_weight, eps, how):
        r, h, stats = cb.residual_norm(x, y, gate, weight, bias, post_weight, eps=eps, save_stats=True, **how)
        fctx.save_for_backward(x, y, gate, weight, bias, post_weight, stats)
        fctx.set_materialize_grads(False)
        fctx.how = how
        return r, h

    @staticmethod
    @once_differentiable
    def backward(fctx, dr, dh):
        x, y, gate, weight, bias, post_weight, stats = fctx.saved_tensors
        need = fctx.needs_input_grad[:6]
        if dr is None and dh is None:
            return (None,) * 8
        dh = y.new_zeros(y.shape) if dh is None else _rows_ok(dh)
        return cb.residual_norm_backward(None if dr is None else _rows_ok(dr), dh, x, y, gate, weight, bias, post_weight, stats, need=need, **fctx.how) + (None, None)


def residual_norm(x, y, gate=None, weight=None, bias=None, post_weight=None, kind="layer", post=None, eps=1e-6, residual_scale=1.0, weight_offset=0.0, post_offset=0.0):
    """clear_block.residual_norm, differentiable in x, y, gate, weight, bias and post_weight: (r, h)."""
    own = lambda t: t if t is None else t.contiguous()
    x, y, gate, weight, bias, post_weight = _rows_ok(x), _rows_ok(y), own(gate), own(weight), own(bias), own(post_weight)
    how = dict(kind=kind, post=post, residual_scale=residual_scale, weight_offset=weight_offset, post_offset=post_offset)
    if _no_gradients(x, y, gate, weight, bias, post_weight):
        return cb.residual_norm(x, y, gate, weight, bias, post_weight, eps=eps, **how)
    if any(v is not None and v.dim() == 2 and v.shape[0] > 65535 for v in (gate, weight, bias)):
        raise ca.ClearAttnError(ca.CLEAR_ERR_UNSUPPORTED, "gradients: at most 65535 items with a vector each")
    return ResidualNormFunction.apply(x, y, gate, weight, bias, post_weight, eps, how)


class GatedFFFunction(torch.autograd.Function):
    @staticmethod
    def forward(fctx, x, w_gate, w_up, activation):
        h, pre = cb.gated_ff(x, w_gate, w_up, activation=activation, save_pre=True)
        fctx.save_for_backward(x, w_gate, w_up, pre)
        fctx.activation = activation
        return h

    @staticmethod
    @once_differentiable
    def backward(fctx, dh):
        x, w_gate, w_up, pre = fctx.saved_tensors
        need = fctx.needs_input_grad
        dx, dg, du = cb.gated_ff_backward(_tokens_ok(dh), x, w_gate, w_up, pre, activation=fctx.activation, need=(need[0], need[1] or need[2]))
        return dx, dg if need[1] else None, du if need[2] else None, None


def _tokens_ok(t):
    """t, or a copy where the projection would not take its layout: rows 16-byte aligned, a multiple of 8 elements and under 2^20 apart (a single row anywhere)."""
    if t.dim() != 2 or t.stride(1) != 1 or (t.shape[0] > 1 and not (t.shape[1] <= t.stride(0) < 1 << 20 and t.stride(0) % 8 == 0)):
        t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone(memory_format=torch.contiguous_format)


def gated_ff(x, w_gate, w_up, activation="silu"):
    """clear_block.gated_ff, differentiable in x, w_gate and w_up.  x may lie in any way (it is copied where the projection needs it)."""
    x = _tokens_ok(x)
    if _no_gradients(x, w_gate, w_up):
        return cb.gated_ff(x, w_gate, w_up, activation=activation)
    return GatedFFFunction.apply(x, w_gate, w_up, activation)
