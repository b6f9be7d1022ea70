/*
 * clear_block.h -- C ABI of the operators that stand around the CLEAR local attention (clear_attn.h) in a transformer
 * block and its training step: rotary positions, layer norm, the gated feed-forward projection, the AdamW step.  Same
 * library (libclear_attn.so), status codes and data types as clear_attn.h.
 *
 * All tensors are DEVICE pointers owned by the caller and need the alignment of their element type only, unless stated
 * otherwise; strides count elements and the last axis is contiguous.  Every call enqueues all of its work on the stream
 * passed in, on the current device, and returns without synchronising; it allocates nothing (what it needs besides its
 * operands is a workspace that the caller passes), keeps nothing, and may be captured into a HIP graph.  A workspace's
 * content need not be kept between calls; calls that may overlap in time need one each.
 *
 * Errors: every function returns a clear_status; nothing throws or aborts; invalid arguments are rejected before any device
 * work.  clear_block_last_error gives the reason of the calling thread's last failure.
 *
 * Sums, statistics and states are held in fp32 (angles in fp64); results are rounded to the output's type once.  Every
 * result is the same from call to call, bit for bit: no atomics.
 */
#ifndef CLEAR_BLOCK_H
#define CLEAR_BLOCK_H

#include "clear_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Reason of the calling thread's last failed clear_block_* call; valid until its next one. */
const char* clear_block_last_error(void);

/* ---- Rotary positions -----------------------------------------------------------------------------------------------
 *
 * Turns the first rot_dim channels of every head of Q [B, Hq, N, head_dim] and K [B, Hk, N, head_dim] by the angles of
 * their tokens and writes all channels to Q_out and K_out (the rest copied):
 *     angle(b, n, i) = sum_a positions[a][b][n] * freqs[a][i],         i = 0 .. rot_dim/2 - 1
 *     (x, y) -> scale * (x cos - y sin, x sin + y cos)
 * where (x, y) are channels (2i, 2i + 1) if `interleaved`, else (i, i + rot_dim/2).  inverse != 0 turns by the negative
 * angle: with the same scale this is the transposed map, which takes the gradient of the outputs to that of the inputs.
 * The n_axes (1..4) position axes are added: one for a text, a row and a column for an image (the frequencies of pairs that an axis
 * does not act on are 0).  Positions are device integers of 32 or 64 bits (position_bits), any sign, at
 * positions + a*ps[0] + b*ps[1] + n*ps[2] with position_strides ps (0 repeats).  freqs: device fp64 [n_axes][rot_dim/2], radians
 * a position (clear_block_rotary_frequencies).  Angles are formed and reduced to a turn in fp64, so a far position costs no precision.
 *
 * strides: 12 values, (batch, head, token) of Q, Q_out, K, K_out.  An output is either its input itself (same pointer and strides:
 * in place) or its address range must not overlap either input's; its rows must not overlap: a stride of an axis with more than one
 * entry steps over all that the smaller ones reach.  Where Q or K is turned in place they must share no element: their address ranges
 * are apart, or they have strides in common and lie apart within each of their steps (slices of one projection's output).
 * K = K_out = NULL with Hk = 0: Q alone.  2 <= rot_dim <= head_dim <= 1024, rot_dim even.  dtype CLEAR_BF16 or CLEAR_F32.
 * B = 0 or N = 0 does nothing. */
int clear_block_rotary(const void* Q, void* Q_out, int Hq, const void* K, void* K_out, int Hk, const long long* strides, long long B,
                       long long N, int head_dim, int rot_dim, int interleaved, const void* positions, int position_bits,
                       const long long* position_strides, int n_axes, const double* freqs, float scale, int inverse, int dtype,
                       void* stream);

typedef enum {
    CLEAR_ROPE_PLAIN = 0,   /* f_i = theta^(-2i / rot_dim) */
    CLEAR_ROPE_LINEAR = 1,  /* f_i / factor: positions interpolated */
    CLEAR_ROPE_BASE = 2,    /* theta * factor^(rot_dim / (rot_dim - 2)) in the place of theta: the fastest pair is kept, the slowest stretched by factor */
    CLEAR_ROPE_PARTS = 3    /* f_i (w + (1 - w) / factor), w = (n - slow) / (fast - slow) cut to [0, 1], n = original_length f_i / 2 pi the
                               turns that the pair makes over the original context: fast pairs are kept, slow ones stretched */
} clear_rope_scaling;
/* Host only: the rot_dim/2 frequencies of one axis, to a HOST array.  theta > 1 and factor > 0 (unused by CLEAR_ROPE_PLAIN);
 * original_length > 0 and fast > slow >= 0 for CLEAR_ROPE_PARTS, which alone uses them. */
int clear_block_rotary_frequencies(double* freqs, int rot_dim, double theta, int scaling, double factor, double original_length,
                                   double slow, double fast);

/* ---- Layer norm -----------------------------------------------------------------------------------------------------
 *
 * X, Y [groups, rows, channels]; over the channels of each row, with mean mu and (biased) variance var,
 *     xhat = (x - mu) / sqrt(var + eps),   y = xhat * (weight_offset + weight) + bias.
 * weight and bias are contiguous, [channels] or, with per_group != 0, [groups, channels] (the adaptive norm of a diffusion block: scale and shift per
 * batch item, weight_offset 1); either may be NULL (no weight: y = xhat + bias).  stats: NULL, or fp32 [2, groups, rows],
 * which receives mu and 1 / sqrt(var + eps) for the backward pass.  The variance is that of the differences from the mean.
 * strides: (group, row) of X and Y, 4 values, in elements; Y may be X itself (same strides).  dtype of X and Y, weight_dtype of
 * weight and bias: CLEAR_BF16 or CLEAR_F32 each.  1 <= channels <= 16384; groups * rows < 2^31; eps >= 0. */
int clear_block_layer_norm(const void* X, const void* weight, const void* bias, void* Y, float* stats, long long groups, long long rows,
                           int channels, const long long* strides, int per_group, float eps, float weight_offset, int dtype,
                           int weight_dtype, void* stream);

/* Backward pass.  dY the gradient of Y, X and stats as the forward pass had and gave them; writes (each may be NULL, but not all where there are rows)
 *     dX = (dyw - mean(dyw) - xhat * mean(dyw * xhat)) / sqrt(var + eps),  dyw = dy * (weight_offset + weight),
 *     d_weight = sum dy * xhat,  d_bias = sum dy   over the rows (of a group with per_group, else of all groups; 0 for no rows),
 * the latter two laid out and typed like weight.  strides: (group, row) of dY, X, dX, 6 values; dX may be dY itself (same strides).
 * workspace: fp32, clear_block_layer_norm_workspace floats, needed for d_weight or d_bias.  With per_group at most 65535 groups. */
int clear_block_layer_norm_backward(const void* dY, const void* X, const void* weight, const float* stats, void* dX, void* d_weight,
                                    void* d_bias, long long groups, long long rows, int channels, const long long* strides,
                                    int per_group, float weight_offset, int dtype, int weight_dtype, float* workspace, void* stream);
/* Floats of that workspace (host only); -1 for sizes that the calls refuse. */
long long clear_block_layer_norm_workspace(long long groups, long long rows, int channels, int per_group);

/* ---- Gated feed-forward projection ------------------------------------------------------------------------------------
 *
 * H = act(X Wg^T) * (X Wu^T) for X [tokens, channels] and the weights Wg, Wu [hidden, channels]: both products, the activation
 * and the product in one pass.  bf16, fp32 accumulation, one rounding on output.  pre: NULL, or fp32 [2, tokens, hidden], which receives
 * the two products (gate first) for the backward pass.  ld_x, ld_gate, ld_up, ld_h: elements from one row to the next.  Pointers 16-byte
 * aligned; channels, hidden and the row strides multiples of 8; row strides < 2^20 (those of a single token are not looked at) and tokens < 2^31.  A few tokens take a form that
 * streams the weights once. */
typedef enum {
    CLEAR_ACT_SILU = 0,      /* g / (1 + e^-g) */
    CLEAR_ACT_GELU_TANH = 1, /* g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2 */
    CLEAR_ACT_GELU_ERF = 2   /* g (1 + erf(g / sqrt 2)) / 2 */
} clear_activation;
int clear_block_gated_ff(const void* X, const void* Wg, const void* Wu, void* H, float* pre, long long tokens, int channels, int hidden,
                         long long ld_x, long long ld_gate, long long ld_up, long long ld_h, int activation, void* stream);

/* Backward pass.  dH [tokens, hidden] the gradient of H, pre as the forward pass wrote it; writes (dX may be NULL; dWg and dWu both or neither; one of them where there are tokens)
 *     dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X   with  dG = dH * u * act'(g),  dU = dH * act(g)
 * in bf16 (dG and dU are rounded to bf16 as operands of the products; 0 for no tokens).  ld: the row strides of dH, X, Wg, Wu, dX, dWg, dWu, 7 values
 * under the rules above.  workspace: clear_block_gated_ff_workspace bytes, 16-byte aligned. */
int clear_block_gated_ff_backward(const void* dH, const void* X, const void* Wg, const void* Wu, const float* pre, void* dX, void* dWg,
                                  void* dWu, long long tokens, int channels, int hidden, const long long* ld, int activation,
                                  void* workspace, void* stream);
/* Bytes of that workspace (host only); -1 for sizes that the call refuses. */
long long clear_block_gated_ff_workspace(long long tokens, int channels, int hidden);

/* ---- AdamW --------------------------------------------------------------------------------------------------------------
 *
 * One optimizer step over n_tensors tensors in one launch per 56 of them.  For every element, in fp32,
 *     m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *     p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * with g multiplied by *grad_scale first where grad_scale (a device fp32 scalar: a clipping factor) is not NULL.  param and grad are of
 * dtype (CLEAR_BF16 or CLEAR_F32).  master: NULL, or the parameter in fp32, which is then the one that is read and updated, and
 * param receives it rounded.  A tensor whose grad is NULL, or that has no elements, is left as it is.
 *
 * state_bits 32: m and v are fp32.  state_bits 8: blocks of 256 elements of a tensor share a scale, the block's largest |m| (or v);
 *     m is int8 c:   m = scale * t |t|, t = c / 127     (stored c: the nearest, of the magnitude's root)
 *     v is uint8 c:  v = scale * t^4,   t = c / 255     (the nearest of the fourth root; a v > 0 is not stored as 0)
 * with ceil(n / 256) fp32 scales each in m_scale and v_scale.  The step itself uses the new m and v before they are stored.  A state that is not
 * finite makes its block's stored states NaN (both codes 0, scales NaN).
 * `tensors` is a HOST array, read before the call returns, as are the numbers of the step: a captured graph repeats them.  No two tensors may share memory.  n <= 2^35. */
typedef struct {
    void* param;
    const void* grad;
    float* master;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    long long n;
} clear_block_adamw_tensor;
int clear_block_adamw(int n_tensors, const clear_block_adamw_tensor* tensors, int dtype, int state_bits, double lr, double beta1, double beta2,
                      double eps, double weight_decay, long long step, const float* grad_scale, void* stream);
/* The values that 8-bit states of n elements stand for, in fp32 (for checkpoints and tests). */
int clear_block_adamw_decode(const void* m, const float* m_scale, const void* v, const float* v_scale, float* m_out, float* v_out,
                             long long n, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CLEAR_BLOCK_H */
