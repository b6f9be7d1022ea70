// C ABI of the operators around the attention (include/clear_block.h): argument checks and launches.
#include "../../include/clear_block.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "block_internal.h"

using namespace clear::block;

namespace {

thread_local std::string g_error;

// Nothing leaves a C entry point as an exception: a message that cannot be stored is dropped.
int fail(int code, const char* what, const char* why = "") noexcept
{
    try {
        g_error.assign(what);
        g_error.append(why);
    } catch (...) {
        g_error.clear();
    }
    return code;
}
int invalid(const char* what) noexcept { return fail(CLEAR_ERR_INVALID_ARG, what); }
int unsupported(const char* what) noexcept { return fail(CLEAR_ERR_UNSUPPORTED, what); }
int launched(hipError_t e, const char* what) noexcept { return e == hipSuccess ? CLEAR_OK : fail(CLEAR_ERR_HIP, what, hipGetErrorString(e)); }

bool known_dtype(int dtype) { return dtype == CLEAR_BF16 || dtype == CLEAR_F32; }
int size_of(int dtype) { return dtype == CLEAR_BF16 ? 2 : 4; }
bool aligned(const void* p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }

// Byte range [first, last) that a strided tensor spans.
struct Span {
    __int128 first, last;
};
Span span_of(const void* p, const long long* extent, const long long* stride, int axes, long long row, int size)
{
    __int128 last = row;
    for (int i = 0; i < axes; ++i) last += (__int128)(extent[i] - 1) * stride[i];
    return {(__int128)(uintptr_t)p, (__int128)(uintptr_t)p + last * size};
}
bool overlap(const Span& a, const Span& b) { return a.first < b.last && b.first < a.last; }
bool too_long(const Span& a) { return a.last > ((__int128)1 << 62); }

// Axes of one or two tensors by falling stride, without those on which nobody has a second entry.
struct Axes {
    int n = 0;
    long long stride[3], ep[3], eq[3];
    // (two tensors need to agree on a stride only where both step along it); false if they do not
    bool gather(const long long* p_extent, const long long* p_stride, const long long* q_extent, const long long* q_stride)
    {
        for (int i = 0; i < 3; ++i) {
            if (p_extent[i] <= 1 && q_extent[i] <= 1) continue;
            if (p_extent[i] > 1 && q_extent[i] > 1 && p_stride[i] != q_stride[i]) return false;
            const long long s = p_extent[i] > 1 ? p_stride[i] : q_stride[i];
            int at = n++;
            for (; at > 0 && stride[at - 1] < s; --at) stride[at] = stride[at - 1], ep[at] = ep[at - 1], eq[at] = eq[at - 1];
            stride[at] = s, ep[at] = p_extent[i], eq[at] = q_extent[i];
        }
        return true;
    }
    // Elements from the first to behind the last over the axes from `from` on.
    __int128 span(const long long* extent, int from, long long row) const
    {
        __int128 s = row;
        for (int i = from; i < n; ++i) s += (__int128)(extent[i] - 1) * stride[i];
        return s;
    }
};
// Whether no two rows of a tensor share an element, by strides that step over all that the smaller ones reach.
bool rows_are_own(const long long* extent, const long long* stride, long long row)
{
    Axes a;
    a.gather(extent, stride, extent, stride);
    for (int i = 0; i < a.n; ++i)
        if (a.stride[i] < a.span(a.ep, i + 1, row)) return false;
    return true;
}
// Whether two tensors share no element: their ranges are apart, or they are slices of one tensor, which lie apart within every step of the strides that they have in
// common.  (What cannot be told in this way counts as shared.)
bool elements_apart(const void* P, const long long* p_extent, const long long* p_stride, const void* Q, const long long* q_extent, const long long* q_stride, long long row, int size)
{
    if (!overlap(span_of(P, p_extent, p_stride, 3, row, size), span_of(Q, q_extent, q_stride, 3, row, size))) return true;
    __int128 d = (__int128)(uintptr_t)Q - (__int128)(uintptr_t)P;  // from P to Q
    if (d % size) return false;
    d /= size;
    Axes a;
    if (!a.gather(p_extent, p_stride, q_extent, q_stride)) return false;
    for (int i = 0;; ++i) {
        if (d >= a.span(a.ep, i, row) || -d >= a.span(a.eq, i, row)) return true;
        if (i == a.n || a.stride[i] == 0) return false;
        const __int128 s = a.stride[i], p = a.span(a.ep, i + 1, row), q = a.span(a.eq, i + 1, row);
        __int128 k = d / s, off = d % s;  // Q's entry j on this axis lies `off` behind P's entry j + k
        if (off < 0) off += s, --k;
        if (p <= s && off + q <= s) {
            d = off;
        } else if (q <= s && p <= off) {  // P's entry j + k + 1 lies s - off behind Q's entry j, and within its step
            d = off - s, ++k;
        } else {
            return false;
        }
        if (k >= a.ep[i] || -k >= a.eq[i]) return true;  // no two entries in one step
    }
}

}  // namespace

const char* clear_block_last_error(void) { return g_error.c_str(); }

int clear_block_rotary(const void* Q, void* Q_out, int Hq, const void* K, void* K_out, int Hk, const long long* strides, long long B, long long N,
                       int head_dim, int rot_dim, int interleaved, const void* positions, int position_bits, const long long* position_strides,
                       int n_axes, const double* freqs, float scale, int inverse, int dtype, void* stream)
{
    if (!known_dtype(dtype)) return invalid("dtype must be CLEAR_BF16 or CLEAR_F32");
    if (Hq < 1 || Hk < 0 || B < 0 || N < 0) return invalid("Hq must be >= 1, Hk, B and N >= 0");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim) return invalid("rot_dim must be even, >= 2 and <= head_dim");
    if (head_dim > 1024) return unsupported("head_dim must be <= 1024");
    if (Hq > 65536 || Hk > 65536) return unsupported("at most 65536 heads each");
    if (n_axes < 1 || n_axes > 4) return invalid("n_axes must be in [1, 4]");
    if (position_bits != 32 && position_bits != 64) return invalid("position_bits must be 32 or 64");
    if (!std::isfinite(scale)) return invalid("scale must be finite");
    if (B == 0 || N == 0) return CLEAR_OK;
    if (!Q || !Q_out || !strides || !positions || !position_strides || !freqs) return invalid("Q, Q_out, strides, positions, position_strides and freqs must be non-NULL");
    if ((K == nullptr) != (K_out == nullptr) || (K == nullptr) != (Hk == 0)) return invalid("K, K_out and Hk > 0 go together: all or none");
    const int size = size_of(dtype);
    if (!aligned(Q, size) || !aligned(Q_out, size) || !aligned(K, size) || !aligned(K_out, size) || !aligned(positions, position_bits / 8) || !aligned(freqs, 8))
        return invalid("pointers must be aligned to their elements");
    if (B > (1LL << 40) || N > (1LL << 40) / B) return unsupported("B * N must be <= 2^40");
    for (int i = 0; i < 3; ++i)
        if (position_strides[i] < 0) return invalid("position strides must be >= 0");
    // extents of the tensors; an output is its input, or apart from both inputs and from the other output
    const long long eq[3] = {B, Hq, N}, ek[3] = {B, Hk, N};
    for (int i = 0; i < 12; ++i) {
        const long long* const e = i < 6 ? eq : ek;
        if (i >= 6 && !K) break;
        if (strides[i] < 0) return invalid("strides must be >= 0");
        if (strides[i] > (1LL << 48)) return unsupported("strides must be <= 2^48");
        if (i % 6 >= 3 && strides[i] == 0 && e[i % 3] > 1) return invalid("an output's strides must be > 0");
    }
    const Span q = span_of(Q, eq, strides, 3, head_dim, size), qo = span_of(Q_out, eq, strides + 3, 3, head_dim, size);
    if (too_long(q) || too_long(qo)) return unsupported("tensor of more than 2^62 bytes");
    if (!rows_are_own(eq, strides + 3, head_dim)) return invalid("the rows of Q_out must not overlap");
    const bool q_in_place = Q == Q_out && std::equal(strides, strides + 3, strides + 3);
    bool k_in_place = true;
    if (!q_in_place && overlap(q, qo)) return invalid("Q_out must be Q itself or must not overlap it");
    if (K) {
        const Span k = span_of(K, ek, strides + 6, 3, head_dim, size), ko = span_of(K_out, ek, strides + 9, 3, head_dim, size);
        if (too_long(k) || too_long(ko)) return unsupported("tensor of more than 2^62 bytes");
        k_in_place = K == K_out && std::equal(strides + 6, strides + 9, strides + 9);
        if (!rows_are_own(ek, strides + 9, head_dim)) return invalid("the rows of K_out must not overlap");
        if (!k_in_place && overlap(k, ko)) return invalid("K_out must be K itself or must not overlap it");
        if (!q_in_place && (overlap(qo, k) || overlap(qo, ko))) return invalid("Q_out must not overlap K or K_out");
        if (!k_in_place && overlap(ko, q)) return invalid("K_out must not overlap Q");
        // (what is turned in place is written while the other is read; they may be slices of one tensor)
        if ((q_in_place || k_in_place) && !elements_apart(Q, eq, strides, K, ek, strides + 6, head_dim, size)) return invalid("Q and K must not share elements where one is turned in place");
    }
    RotaryArgs a = {};
    a.q = Q, a.k = K, a.q_out = Q_out, a.k_out = K_out;
    a.Hq = Hq, a.Hk = Hk;
    for (int i = 0; i < 12; ++i) a.st[i] = i < 6 || K ? strides[i] : 0;
    a.B = B, a.N = N;
    a.head_dim = head_dim, a.rot_dim = rot_dim;
    a.copy = rot_dim < head_dim && !(q_in_place && k_in_place);
    a.positions = positions;
    for (int i = 0; i < 3; ++i) a.ps[i] = position_strides[i];
    a.n_axes = n_axes;
    a.freqs = freqs;
    a.scale = scale;
    a.sign = inverse ? -1.f : 1.f;
    return launched(launch_rotary(a, interleaved != 0, position_bits == 64, dtype, (hipStream_t)stream), "rotary launch failed: ");
}

int clear_block_rotary_frequencies(double* freqs, int rot_dim, double theta, int scaling, double factor, double original_length, double slow, double fast)
{
    if (!freqs) return invalid("freqs is NULL");
    if (rot_dim < 2 || rot_dim % 2) return invalid("rot_dim must be even and >= 2");
    if (!(theta > 1) || !std::isfinite(theta)) return invalid("theta must be finite and > 1");
    if (scaling < CLEAR_ROPE_PLAIN || scaling > CLEAR_ROPE_PARTS) return invalid("unknown scaling");
    if (scaling != CLEAR_ROPE_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return invalid("factor must be finite and > 0");
    if (scaling == CLEAR_ROPE_BASE && rot_dim == 2) return unsupported("CLEAR_ROPE_BASE needs rot_dim > 2: with one pair there is no slowest beside the fastest");
    if (scaling == CLEAR_ROPE_PARTS && (!(original_length > 0) || !(slow >= 0) || !(fast > slow) || !std::isfinite(original_length) || !std::isfinite(fast)))
        return invalid("CLEAR_ROPE_PARTS needs original_length > 0 and fast > slow >= 0");
    if (scaling == CLEAR_ROPE_BASE) theta *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(theta, -2.0 * i / rot_dim);
        if (scaling == CLEAR_ROPE_LINEAR) f /= factor;
        if (scaling == CLEAR_ROPE_PARTS) {
            const double turns = original_length * f * 0.15915494309189533577;
            const double w = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
            f = f * (w + (1.0 - w) / factor);
        }
        freqs[i] = f;
    }
    return CLEAR_OK;
}

namespace {

int check_norm(long long groups, long long rows, int channels, const long long* strides, int n_strides, int dtype, int weight_dtype)
{
    if (!known_dtype(dtype) || !known_dtype(weight_dtype)) return invalid("dtype and weight_dtype must be CLEAR_BF16 or CLEAR_F32");
    if (groups < 0 || rows < 0) return invalid("groups and rows must be >= 0");
    if (channels < 1) return invalid("channels must be >= 1");
    if (channels > kNormMaxChannels) return unsupported("at most 16384 channels");
    if (groups > 0x7fffffffLL || rows > 0x7fffffffLL || groups * rows > 0x7fffffffLL) return unsupported("groups * rows must be < 2^31");
    if (!strides) return invalid("strides is NULL");
    for (int i = 0; i < n_strides; ++i) {
        if (strides[i] < 0) return invalid("strides must be >= 0");
        if (strides[i] > (1LL << 48)) return unsupported("strides must be <= 2^48");
    }
    return CLEAR_OK;
}

// An output may be `in` itself; else their ranges must be apart.  A row of an output is its own.
bool out_apart(const void* out, const long long* out_strides, const void* in, const long long* in_strides, const long long* extent, int channels, int size, bool may_be_same)
{
    if (may_be_same && out == in && out_strides[0] == in_strides[0] && out_strides[1] == in_strides[1]) return true;
    return !overlap(span_of(out, extent, out_strides, 2, channels, size), span_of(in, extent, in_strides, 2, channels, size));
}
bool rows_apart(const long long* strides, const long long* extent, int channels)
{
    if (extent[1] > 1 && strides[1] < channels) return false;
    if (extent[0] <= 1) return true;
    // groups one after the other, or interleaved with the rows (a transposed view)
    const __int128 rows = (__int128)(extent[1] - 1) * strides[1] + channels;
    return strides[0] >= rows || (strides[0] >= channels && (extent[1] == 1 || strides[1] >= (__int128)(extent[0] - 1) * strides[0] + channels));
}

}  // namespace

int clear_block_layer_norm(const void* X, const void* weight, const void* bias, void* Y, float* stats, long long groups, long long rows, int channels,
                           const long long* strides, int per_group, float eps, float weight_offset, int dtype, int weight_dtype, void* stream)
{
    const int rc = check_norm(groups, rows, channels, strides, 4, dtype, weight_dtype);
    if (rc != CLEAR_OK) return rc;
    if (!(eps >= 0) || !std::isfinite(eps) || !std::isfinite(weight_offset)) return invalid("eps must be finite and >= 0, weight_offset finite");
    if (groups == 0 || rows == 0) return CLEAR_OK;
    if (!X || !Y) return invalid("X and Y must be non-NULL");
    if (!aligned(X, size_of(dtype)) || !aligned(Y, size_of(dtype)) || !aligned(weight, size_of(weight_dtype)) || !aligned(bias, size_of(weight_dtype)) || !aligned(stats, 4))
        return invalid("pointers must be aligned to their elements");
    const long long extent[2] = {groups, rows};
    if (!rows_apart(strides + 2, extent, channels)) return invalid("the rows of Y must not overlap");
    if (!out_apart(Y, strides + 2, X, strides, extent, channels, size_of(dtype), true)) return invalid("Y must be X itself or must not overlap it");
    NormArgs a = {};
    a.x = X, a.w = weight, a.b = bias, a.y = Y, a.stats = stats;
    a.groups = (int)groups, a.rows = (int)rows, a.channels = channels;
    for (int i = 0; i < 4; ++i) a.st[i] = strides[i];
    a.per_group = per_group != 0;
    a.eps = eps, a.offset = weight_offset;
    return launched(launch_norm_forward(a, dtype, weight_dtype, (hipStream_t)stream), "layer norm launch failed: ");
}

int clear_block_layer_norm_backward(const void* dY, const void* X, const void* weight, const float* stats, void* dX, void* d_weight, void* d_bias,
                                    long long groups, long long rows, int channels, const long long* strides, int per_group, float weight_offset, int dtype,
                                    int weight_dtype, float* workspace, void* stream)
{
    const int rc = check_norm(groups, rows, channels, strides, 6, dtype, weight_dtype);
    if (rc != CLEAR_OK) return rc;
    if (!std::isfinite(weight_offset)) return invalid("weight_offset must be finite");
    const bool some = groups > 0 && rows > 0;  // (without rows dX has no elements, and may have no address)
    if (some && !dX && !d_weight && !d_bias) return invalid("one of dX, d_weight, d_bias must be non-NULL");
    if (some && (!dY || !X || !stats)) return invalid("dY, X and stats must be non-NULL");
    if (some && (d_weight || d_bias) && !workspace) return invalid("d_weight and d_bias need a workspace");
    if (per_group && groups > 65535) return unsupported("at most 65535 groups with a weight each");
    const int size = size_of(dtype), wsize = size_of(weight_dtype);
    if (!aligned(dY, size) || !aligned(X, size) || !aligned(dX, size) || !aligned(weight, wsize) || !aligned(d_weight, wsize) || !aligned(d_bias, wsize) ||
        !aligned(stats, 4) || !aligned(workspace, 4))
        return invalid("pointers must be aligned to their elements");
    if (some && dX) {
        const long long extent[2] = {groups, rows};
        if (!rows_apart(strides + 4, extent, channels)) return invalid("the rows of dX must not overlap");
        if (!out_apart(dX, strides + 4, dY, strides, extent, channels, size, true) || !out_apart(dX, strides + 4, X, strides + 2, extent, channels, size, false))
            return invalid("dX must be dY itself or must not overlap it, and must not overlap X");
    }
    if (!some && (!(d_weight || d_bias) || (per_group && groups == 0))) return CLEAR_OK;
    NormArgs a = {};
    a.x = X, a.w = weight, a.dy = dY, a.dx = dX, a.dw = d_weight, a.db = d_bias;
    a.stats = const_cast<float*>(stats);
    a.ws = workspace;
    a.groups = (int)groups, a.rows = (int)rows, a.channels = channels;
    for (int i = 0; i < 6; ++i) a.st[i] = strides[i];
    a.per_group = per_group != 0;
    a.offset = weight_offset;
    return launched(launch_norm_backward(a, dtype, weight_dtype, (hipStream_t)stream), "layer norm backward launch failed: ");
}

long long clear_block_layer_norm_workspace(long long groups, long long rows, int channels, int per_group)
{
    const long long none[4] = {};
    if (check_norm(groups, rows, channels, none, 4, CLEAR_F32, CLEAR_F32) != CLEAR_OK) return -1;
    return (long long)norm_partials(groups, rows, channels, per_group != 0) * (per_group ? groups : 1) * 2 * ((channels + 7) / 8 * 8);
}

int clear_block_adamw(int n_tensors, const clear_block_adamw_tensor* tensors, int dtype, int state_bits, double lr, double beta1, double beta2, double eps,
                      double weight_decay, long long step, const float* grad_scale, void* stream)
{
    if (!known_dtype(dtype)) return invalid("dtype must be CLEAR_BF16 or CLEAR_F32");
    if (state_bits != 32 && state_bits != 8) return invalid("state_bits must be 32 or 8");
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return invalid("n_tensors must be >= 0 and tensors non-NULL");
    if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1)) return invalid("beta1 and beta2 must be in [0, 1)");
    if (!std::isfinite(lr) || !(lr >= 0) || !std::isfinite(eps) || !(eps >= 0) || !std::isfinite(weight_decay) || !(weight_decay >= 0))
        return invalid("lr, eps and weight_decay must be finite and >= 0");
    if (step < 1) return invalid("step counts from 1");
    if (!aligned(grad_scale, 4)) return invalid("pointers must be aligned to their elements");
    const int size = size_of(dtype);
    for (int i = 0; i < n_tensors; ++i) {
        const clear_block_adamw_tensor& t = tensors[i];
        if (t.n < 0) return invalid("a tensor has a negative number of elements");
        if (t.n > (1LL << 35)) return unsupported("a tensor has more than 2^35 elements");
        if (t.n == 0 || !t.grad) continue;
        if (!t.param || !t.m || !t.v) return invalid("param, m and v of a tensor must be non-NULL");
        if (state_bits == 8 && (!t.m_scale || !t.v_scale)) return invalid("states of 8 bits need m_scale and v_scale");
        if (!aligned(t.param, size) || !aligned(t.grad, size) || !aligned(t.master, 4) || (state_bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))) ||
            !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))
            return invalid("pointers must be aligned to their elements");
    }
    AdamHyper h;
    h.beta1 = (float)beta1, h.one_minus_beta1 = (float)(1 - beta1);
    h.beta2 = (float)beta2, h.one_minus_beta2 = (float)(1 - beta2);
    h.keep = (float)(1 - lr * weight_decay);
    h.step_size = (float)(lr / (1 - std::pow(beta1, (double)step)));
    h.inv_root_correction = (float)(1 / std::sqrt(1 - std::pow(beta2, (double)step)));
    h.eps = (float)eps;
    h.grad_scale = grad_scale;
    return launched(launch_adamw(n_tensors, tensors, h, dtype, state_bits, (hipStream_t)stream), "AdamW launch failed: ");
}

int clear_block_adamw_decode(const void* m, const float* m_scale, const void* v, const float* v_scale, float* m_out, float* v_out, long long n, void* stream)
{
    if (n < 0) return invalid("n must be >= 0");
    if (n == 0) return CLEAR_OK;
    if (!m || !m_scale || !v || !v_scale || !m_out || !v_out) return invalid("every pointer must be non-NULL");
    if (!aligned(m_scale, 4) || !aligned(v_scale, 4) || !aligned(m_out, 4) || !aligned(v_out, 4)) return invalid("pointers must be aligned to their elements");
    return launched(launch_adamw_decode(m, m_scale, v, v_scale, m_out, v_out, n, (hipStream_t)stream), "AdamW decode launch failed: ");
}

namespace {

// A single row has no stride: what its tensor says is not looked at.
long long row_stride(long long rows, long long ld, int width) { return rows == 1 ? width : ld; }
// Sizes and row strides of the gated projection.
int check_gated(long long tokens, int channels, int hidden, const long long* ld, const int* width, int n_ld)
{
    if (tokens < 0 || channels < 1 || hidden < 1) return invalid("tokens must be >= 0, channels and hidden >= 1");
    if (channels % 8 || hidden % 8) return unsupported("channels and hidden must be multiples of 8");
    if (tokens > 0x7fffffffLL || channels >= (1 << 20) || hidden >= (1 << 20)) return unsupported("tokens must be < 2^31, channels and hidden < 2^20");
    for (int i = 0; i < n_ld; ++i) {
        if (ld[i] < width[i]) return invalid("a row stride is shorter than its row");
        if (ld[i] % 8 || ld[i] >= (1 << 20)) return unsupported("row strides must be multiples of 8 and < 2^20");
    }
    return CLEAR_OK;
}
Span rows_of(const void* p, long long rows, long long ld, int width, int size)
{
    return {(__int128)(uintptr_t)p, (__int128)(uintptr_t)p + ((__int128)(rows - 1) * ld + width) * size};
}

}  // namespace

int clear_block_gated_ff(const void* X, const void* Wg, const void* Wu, void* H, float* pre, long long tokens, int channels, int hidden, long long ld_x,
                         long long ld_gate, long long ld_up, long long ld_h, int activation, void* stream)
{
    ld_x = row_stride(tokens, ld_x, channels), ld_h = row_stride(tokens, ld_h, hidden);
    const long long ld[4] = {ld_x, ld_gate, ld_up, ld_h};
    const int width[4] = {channels, channels, channels, hidden};
    const int rc = check_gated(tokens, channels, hidden, ld, width, 4);
    if (rc != CLEAR_OK) return rc;
    if (activation < CLEAR_ACT_SILU || activation > CLEAR_ACT_GELU_ERF) return invalid("unknown activation");
    if (tokens == 0) return CLEAR_OK;
    if (!X || !Wg || !Wu || !H) return invalid("X, Wg, Wu and H must be non-NULL");
    if (!aligned(X, 16) || !aligned(Wg, 16) || !aligned(Wu, 16) || !aligned(H, 16) || !aligned(pre, 16)) return invalid("pointers must be 16-byte aligned");
    const Span h = rows_of(H, tokens, ld_h, hidden, 2);
    if (overlap(h, rows_of(X, tokens, ld_x, channels, 2)) || overlap(h, rows_of(Wg, hidden, ld_gate, channels, 2)) || overlap(h, rows_of(Wu, hidden, ld_up, channels, 2)))
        return invalid("H must not overlap an input");
    GatedArgs a = {};
    a.x = X, a.wg = Wg, a.wu = Wu, a.h = H, a.pre = pre;
    a.tokens = tokens, a.channels = channels, a.hidden = hidden, a.act = activation;
    a.ld_x = ld_x, a.ld_g = ld_gate, a.ld_u = ld_up, a.ld_h = ld_h;
    return launched(launch_gated_forward(a, (hipStream_t)stream), "gated projection launch failed: ");
}

int clear_block_gated_ff_backward(const void* dH, const void* X, const void* Wg, const void* Wu, const float* pre, void* dX, void* dWg, void* dWu, long long tokens,
                                  int channels, int hidden, const long long* strides, int activation, void* workspace, void* stream)
{
    if (!strides) return invalid("ld is NULL");
    const int width[7] = {hidden, channels, channels, channels, channels, channels, channels};
    long long ld[7];
    for (int i = 0; i < 7; ++i) ld[i] = i == 2 || i == 3 || i > 4 ? strides[i] : row_stride(tokens, strides[i], width[i]);  // dH, X and dX have a row for each token
    const int rc = check_gated(tokens, channels, hidden, ld, width, 7);
    if (rc != CLEAR_OK) return rc;
    if (activation < CLEAR_ACT_SILU || activation > CLEAR_ACT_GELU_ERF) return invalid("unknown activation");
    if ((dWg == nullptr) != (dWu == nullptr)) return invalid("dWg and dWu go together: both or neither");
    if (!dX && !dWg) return tokens > 0 ? invalid("one of dX and dWg, dWu must be non-NULL") : CLEAR_OK;  // (without tokens dX has no elements, and may have no address)
    if (tokens > 0 && (!dH || !X || !Wg || !Wu || !pre || !workspace)) return invalid("dH, X, Wg, Wu, pre and workspace must be non-NULL");
    if (!aligned(dH, 16) || !aligned(X, 16) || !aligned(Wg, 16) || !aligned(Wu, 16) || !aligned(pre, 16) || !aligned(dX, 16) || !aligned(dWg, 16) || !aligned(dWu, 16) ||
        !aligned(workspace, 16))
        return invalid("pointers must be 16-byte aligned");
    if (tokens > 0) {
        const Span in[4] = {rows_of(dH, tokens, ld[0], hidden, 2), rows_of(X, tokens, ld[1], channels, 2), rows_of(Wg, hidden, ld[2], channels, 2),
                            rows_of(Wu, hidden, ld[3], channels, 2)};
        const Span out[3] = {rows_of(dX, tokens, ld[4], channels, 2), rows_of(dWg, hidden, ld[5], channels, 2), rows_of(dWu, hidden, ld[6], channels, 2)};
        const bool have[3] = {dX != nullptr, dWg != nullptr, dWu != nullptr};
        for (int o = 0; o < 3; ++o)
            for (int i = 0; have[o] && i < 4; ++i)
                if (overlap(out[o], in[i])) return invalid("an output must not overlap an input");
        if (dX && dWg && (overlap(out[0], out[1]) || overlap(out[0], out[2]))) return invalid("dX must not overlap dWg or dWu");
    }
    if (dWg) {
        // (row-interleaved halves of one tensor are fine: their rows are apart)
        const bool same_stride = ld[5] == ld[6];
        const long long d = ((const char*)dWu - (const char*)dWg) / 2, off = same_stride ? ((d % ld[5]) + ld[5]) % ld[5] : 0;
        const bool interleaved = same_stride && off >= channels && off + channels <= ld[5];
        if (!interleaved && overlap(rows_of(dWg, hidden, ld[5], channels, 2), rows_of(dWu, hidden, ld[6], channels, 2))) return invalid("dWg must not overlap dWu");
    }
    GatedArgs a = {};
    a.dh = dH, a.x = X, a.wg = Wg, a.wu = Wu, a.pre = const_cast<float*>(pre), a.dx = dX, a.dwg = dWg, a.dwu = dWu;
    a.tokens = tokens, a.channels = channels, a.hidden = hidden, a.act = activation;
    a.ld_dh = ld[0], a.ld_x = ld[1], a.ld_g = ld[2], a.ld_u = ld[3], a.ld_dx = ld[4], a.ld_dwg = ld[5], a.ld_dwu = ld[6];
    a.ws = workspace;
    return launched(launch_gated_backward(a, (hipStream_t)stream), "gated projection backward launch failed: ");
}

long long clear_block_gated_ff_workspace(long long tokens, int channels, int hidden)
{
    if (check_gated(tokens, channels, hidden, nullptr, nullptr, 0) != CLEAR_OK) return -1;
    return (long long)gated_workspace_bytes(tokens, channels, hidden);
}
