// C ABI of the gated residual with its norms, the norm of gradients and the operands in 4 bits (include/clear_block.h): argument checks and launches.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>
#include <vector>

#include "block_checks.h"
#include "block_internal.h"

using namespace clear::block;

namespace {

constexpr long long kFar = 1LL << 48;

int check_residual(long long groups, long long rows, int channels, const long long* strides, int n_strides, int kind, int post, int dtype, int stream_dtype, int weight_dtype)
{
    if (!known_dtype(dtype) || !known_dtype(stream_dtype) || !known_dtype(weight_dtype)) return invalid("dtype, stream_dtype and weight_dtype must be CLEAR_BF16 or CLEAR_F32");
    if (dtype == CLEAR_F32 && stream_dtype == CLEAR_BF16) return unsupported("a stream in bf16 beside sublayers in fp32");
    if (kind != CLEAR_NORM_LAYER && kind != CLEAR_NORM_RMS) return invalid("kind must be CLEAR_NORM_LAYER or CLEAR_NORM_RMS");
    if (post < CLEAR_NORM_NONE || post > CLEAR_NORM_RMS) return invalid("unknown post norm");
    if (groups < 0 || rows < 0) return invalid("groups and rows must be >= 0");
    if (channels < 1) return invalid("channels must be >= 1");
    if (channels > kResidualMaxChannels) return unsupported("at most 8192 channels");
    if (groups > 0x7fffffffLL || rows > 0x7fffffffLL || groups * rows > 0x7fffffffLL) return unsupported("groups * rows must be < 2^31");
    if (!strides) return invalid("strides is NULL");
    for (int i = 0; i < n_strides; ++i) {
        if (strides[i] < 0) return invalid("strides must be >= 0");
        if (strides[i] > kFar) return unsupported("strides must be <= 2^48");
    }
    return CLEAR_OK;
}

struct Rows {
    const void* p;
    const long long* strides;
    int size;
};
// Whether output `out` lies apart from what is read and written beside it, or on `same`, whose place it may take.
bool apart(const Rows& out, const Rows* others, int n, const long long* extent, int channels, const Rows* same)
{
    const Span o = span_of(out.p, extent, out.strides, 2, channels, out.size);
    for (int i = 0; i < n; ++i) {
        if (!others[i].p) continue;
        if (&others[i] == same && out.p == same->p && out.size == same->size && out.strides[0] == same->strides[0] && out.strides[1] == same->strides[1]) continue;
        if (overlap(o, span_of(others[i].p, extent, others[i].strides, 2, channels, others[i].size))) return false;
    }
    return true;
}

}  // namespace

int clear_block_residual_norm(const void* X, const void* Y, const void* gate, const void* weight, const void* bias, const void* post_weight, void* R, void* H, float* stats,
                              long long groups, long long rows, int channels, const long long* strides, int gate_per_group, int per_group, int kind, int post, float eps,
                              float residual_scale, float weight_offset, float post_offset, int dtype, int stream_dtype, int weight_dtype, void* stream)
{
    const int rc = check_residual(groups, rows, channels, strides, 8, kind, post, dtype, stream_dtype, weight_dtype);
    if (rc != CLEAR_OK) return rc;
    if (!(eps >= 0) || !std::isfinite(eps) || !std::isfinite(residual_scale) || !std::isfinite(weight_offset) || !std::isfinite(post_offset))
        return invalid("eps must be finite and >= 0, scale and offsets finite");
    if (post_weight && post == CLEAR_NORM_NONE) return invalid("post_weight without a post norm");
    if (groups == 0 || rows == 0) return CLEAR_OK;
    if (!X || !Y || !R || !H) return invalid("X, Y, R and H must be non-NULL");
    const int size = size_of(dtype), ssize = size_of(stream_dtype), wsize = size_of(weight_dtype);
    if (!aligned(X, ssize) || !aligned(R, ssize) || !aligned(Y, size) || !aligned(H, size) || !aligned(gate, wsize) || !aligned(weight, wsize) || !aligned(bias, wsize) ||
        !aligned(post_weight, wsize) || !aligned(stats, 4))
        return invalid("pointers must be aligned to their elements");
    const long long extent[2] = {groups, rows};
    const Rows in[4] = {{X, strides, ssize}, {Y, strides + 2, size}, {R, strides + 4, ssize}, {H, strides + 6, size}};
    for (const Rows& t : in)
        if (too_long(span_of(t.p, extent, t.strides, 2, channels, t.size))) return unsupported("tensor of more than 2^62 bytes");
    if (!rows_apart(strides + 4, extent, channels) || !rows_apart(strides + 6, extent, channels)) return invalid("the rows of R and of H must not overlap");
    const Rows beside_r[3] = {in[0], in[1], in[3]}, beside_h[2] = {in[0], in[1]};
    if (!apart(in[2], beside_r, 3, extent, channels, &beside_r[0])) return invalid("R must be X itself or must not overlap it, and must not overlap Y and H");
    if (!apart(in[3], beside_h, 2, extent, channels, &beside_h[1])) return invalid("H must be Y itself or must not overlap it, and must not overlap X");
    ResidualArgs a = {};
    a.x = X, a.y = Y, a.gate = gate, a.w = weight, a.b = bias, a.pw = post_weight, a.r = R, a.h = H, a.stats = stats;
    a.groups = (int)groups, a.rows = (int)rows, a.channels = channels;
    for (int i = 0; i < 8; ++i) a.st[i] = strides[i];
    a.per_group = per_group != 0, a.gate_per_group = gate_per_group != 0, a.kind = kind, a.post = post;
    a.eps = eps, a.scale = residual_scale, a.offset = weight_offset, a.post_offset = post_offset;
    return launched(launch_residual_forward(a, dtype, stream_dtype, weight_dtype, (hipStream_t)stream), "residual norm launch failed: ");
}

int clear_block_residual_norm_backward(const void* dR, const void* dH, const void* X, const void* Y, const void* gate, const void* weight, const void* post_weight, const float* stats,
                                       void* dX, void* dY, void* d_gate, void* d_weight, void* d_bias, void* d_post_weight, long long groups, long long rows, int channels,
                                       const long long* strides, int gate_per_group, int per_group, int kind, int post, float residual_scale, float weight_offset,
                                       float post_offset, int dtype, int stream_dtype, int weight_dtype, float* workspace, void* stream)
{
    const int rc = check_residual(groups, rows, channels, strides, 12, kind, post, dtype, stream_dtype, weight_dtype);
    if (rc != CLEAR_OK) return rc;
    if (!std::isfinite(residual_scale) || !std::isfinite(weight_offset) || !std::isfinite(post_offset)) return invalid("scale and offsets must be finite");
    if ((post_weight || d_post_weight) && post == CLEAR_NORM_NONE) return invalid("post_weight without a post norm");
    if ((d_gate && !gate) || (d_weight && !weight) || (d_post_weight && !post_weight)) return invalid("the gradient of a vector that is NULL");
    const bool some = groups > 0 && rows > 0, sums = d_gate || d_weight || d_bias || d_post_weight;
    if (some && !dX && !dY && !sums) return invalid("one of the gradients must be non-NULL");
    if (some && (!dH || !X || !Y || !stats)) return invalid("dH, X, Y and stats must be non-NULL");
    if (some && sums && !workspace) return invalid("the vectors' gradients need a workspace");
    if ((per_group || gate_per_group) && groups > 65535) return unsupported("at most 65535 groups with a vector each");
    const int size = size_of(dtype), ssize = size_of(stream_dtype), wsize = size_of(weight_dtype);
    if (!aligned(dR, ssize) || !aligned(X, ssize) || !aligned(dX, ssize) || !aligned(dH, size) || !aligned(Y, size) || !aligned(dY, size) || !aligned(gate, wsize) ||
        !aligned(weight, wsize) || !aligned(post_weight, wsize) || !aligned(d_gate, wsize) || !aligned(d_weight, wsize) || !aligned(d_bias, wsize) || !aligned(d_post_weight, wsize) ||
        !aligned(stats, 4) || !aligned(workspace, 4))
        return invalid("pointers must be aligned to their elements");
    if (some) {
        const long long extent[2] = {groups, rows};
        const Rows all[6] = {{dR, strides, ssize}, {dH, strides + 2, size}, {X, strides + 4, ssize}, {Y, strides + 6, size}, {dX, strides + 8, ssize}, {dY, strides + 10, size}};
        for (const Rows& t : all)
            if (t.p && too_long(span_of(t.p, extent, t.strides, 2, channels, t.size))) return unsupported("tensor of more than 2^62 bytes");
        if ((dX && !rows_apart(strides + 8, extent, channels)) || (dY && !rows_apart(strides + 10, extent, channels))) return invalid("the rows of dX and of dY must not overlap");
        const Rows beside_x[5] = {all[0], all[1], all[2], all[3], all[5]}, beside_y[4] = {all[0], all[1], all[2], all[3]};
        if (dX && !apart(all[4], beside_x, 5, extent, channels, &beside_x[0])) return invalid("dX must be dR itself or must not overlap it, and must not overlap another tensor");
        if (dY && !apart(all[5], beside_y, 4, extent, channels, &beside_y[1])) return invalid("dY must be dH itself or must not overlap it, and must not overlap another tensor");
    }
    if (!some && !sums) return CLEAR_OK;  // (dX and dY have no elements)
    ResidualArgs a = {};
    a.x = X, a.y = Y, a.gate = gate, a.w = weight, a.pw = post_weight, a.dr = dR, a.dh = dH, a.dx = dX, a.dy = dY;
    a.dgate = d_gate, a.dw = d_weight, a.db = d_bias, a.dpw = d_post_weight;
    a.stats = const_cast<float*>(stats), a.ws = workspace;
    a.groups = (int)groups, a.rows = (int)rows, a.channels = channels;
    for (int i = 0; i < 12; ++i) a.st[i] = strides[i];
    a.per_group = per_group != 0, a.gate_per_group = gate_per_group != 0, a.kind = kind, a.post = post;
    a.scale = residual_scale, a.offset = weight_offset, a.post_offset = post_offset;
    if (groups == 0) {  // vectors of no groups have no elements; shared ones have gradients of 0
        if (a.gate_per_group) a.dgate = nullptr;
        if (a.per_group) a.dw = a.db = nullptr;
        a.gate_per_group = a.per_group = 0;
        if (!a.dgate && !a.dw && !a.db && !a.dpw) return CLEAR_OK;
    }
    return launched(launch_residual_backward(a, dtype, stream_dtype, weight_dtype, (hipStream_t)stream), "residual norm backward launch failed: ");
}

long long clear_block_residual_norm_workspace(long long groups, long long rows, int channels, int gate_per_group, int per_group)
{
    const long long none[12] = {};
    if (check_residual(groups, rows, channels, none, 12, CLEAR_NORM_LAYER, CLEAR_NORM_NONE, CLEAR_F32, CLEAR_F32, CLEAR_F32) != CLEAR_OK) return -1;
    const long long sets = gate_per_group || per_group ? groups : 1;
    return (long long)residual_partials(groups, rows, channels, sets) * sets * 4 * ((channels + 7) / 8 * 8);
}

namespace {

int check_grads(int n_tensors, const clear_block_grad* tensors)
{
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return invalid("n_tensors must be >= 0 and tensors non-NULL");
    for (int i = 0; i < n_tensors; ++i) {
        const clear_block_grad& t = tensors[i];
        if (!known_dtype(t.dtype)) return invalid("dtype must be CLEAR_BF16 or CLEAR_F32");
        if (t.n < 0) return invalid("a tensor has a negative number of elements");
        if (t.n > (1LL << 35)) return unsupported("a tensor has more than 2^35 elements");
        if (!aligned(t.data, size_of(t.dtype))) return invalid("pointers must be aligned to their elements");
    }
    return CLEAR_OK;
}

}  // namespace

long long clear_block_grad_norm_workspace(int n_tensors, const clear_block_grad* tensors)
{
    return check_grads(n_tensors, tensors) == CLEAR_OK ? grad_norm_partials(n_tensors, tensors) * 8 : -1;
}

namespace {

int check_norm(int n_tensors, const clear_block_grad* tensors, int kind, double max_norm, bool factor, const float* unscale, const float* norm, const float* factor_out, const void* workspace)
{
    const int rc = check_grads(n_tensors, tensors);
    if (rc != CLEAR_OK) return rc;
    if (kind != CLEAR_GRAD_NORM_2 && kind != CLEAR_GRAD_NORM_MAX) return invalid("kind must be CLEAR_GRAD_NORM_2 or CLEAR_GRAD_NORM_MAX");
    if (factor && !(max_norm >= 0)) return invalid("max_norm must be >= 0");
    if (!aligned(unscale, 4) || !aligned(norm, 4) || !aligned(factor_out, 4) || !aligned(workspace, 8)) return invalid("pointers must be aligned to their elements");
    if (!workspace && grad_norm_partials(n_tensors, tensors) > 0) return invalid("workspace must be non-NULL");
    return CLEAR_OK;
}
// Whether no two tensors, which are written, share memory with each other or with the scalars and partials that other workgroups read or write meanwhile.
struct Beside {
    const void* p;
    long long bytes;
};
int check_apart(int n_tensors, const clear_block_grad* tensors, std::initializer_list<Beside> beside) noexcept
{
    try {
        std::vector<std::pair<uintptr_t, uintptr_t>> spans;
        spans.reserve(n_tensors + beside.size());
        for (int i = 0; i < n_tensors; ++i)
            if (tensors[i].data && tensors[i].n > 0) spans.emplace_back((uintptr_t)tensors[i].data, (uintptr_t)tensors[i].data + (uintptr_t)tensors[i].n * size_of(tensors[i].dtype));
        for (const Beside& b : beside)
            if (b.p && b.bytes > 0) spans.emplace_back((uintptr_t)b.p, (uintptr_t)b.p + (uintptr_t)b.bytes);
        std::sort(spans.begin(), spans.end());
        for (size_t i = 1; i < spans.size(); ++i)
            if (spans[i].first < spans[i - 1].second) return invalid("gradients share memory with each other, or with a scalar or the workspace");
    } catch (...) {
        return fail(CLEAR_ERR_ALLOC, "out of host memory");
    }
    return CLEAR_OK;
}

}  // namespace

int clear_block_grad_norm(int n_tensors, const clear_block_grad* tensors, int kind, double max_norm, const float* unscale, float* norm, float* factor, void* workspace, void* stream)
{
    const int rc = check_norm(n_tensors, tensors, kind, max_norm, factor != nullptr, unscale, norm, factor, workspace);
    if (rc != CLEAR_OK) return rc;
    if (!norm && !factor) return invalid("norm or factor must be non-NULL");
    const GradFactor f = {kind, max_norm, unscale, norm, factor};
    return launched(launch_grad_norm(n_tensors, tensors, f, workspace, (hipStream_t)stream), "gradient norm launch failed: ");
}

int clear_block_grad_clip(int n_tensors, const clear_block_grad* tensors, int kind, double max_norm, const float* unscale, float* norm, float* factor, void* workspace, void* stream)
{
    int rc = check_norm(n_tensors, tensors, kind, max_norm, true, unscale, norm, factor, workspace);
    if (rc != CLEAR_OK) return rc;
    const Beside partials = {workspace, grad_norm_partials(n_tensors, tensors) * 8};
    if ((rc = check_apart(n_tensors, tensors, {{unscale, 4}, {norm, 4}, {factor, 4}, partials})) != CLEAR_OK) return rc;
    const GradFactor f = {kind, max_norm, unscale, norm, factor};
    return launched(launch_grad_clip(n_tensors, tensors, f, workspace, (hipStream_t)stream), "gradient clipping launch failed: ");
}

int clear_block_grad_scale(int n_tensors, const clear_block_grad* tensors, const float* factor, void* stream)
{
    int rc = check_grads(n_tensors, tensors);
    if (rc != CLEAR_OK) return rc;
    if (!factor || !aligned(factor, 4)) return invalid("factor must be a pointer to a float");
    if ((rc = check_apart(n_tensors, tensors, {{factor, 4}})) != CLEAR_OK) return rc;
    return launched(launch_grad_scale(n_tensors, tensors, factor, (hipStream_t)stream), "gradient scaling launch failed: ");
}

namespace {

constexpr int kMxMaxChannels = 1 << 20;

int check_mx(long long rows, int channels)
{
    if (rows < 0 || channels < 1) return invalid("rows must be >= 0 and channels >= 1");
    if (channels % 32) return unsupported("channels must be a multiple of 32");
    if (channels > kMxMaxChannels || rows > 0x7fffffffLL) return unsupported("channels must be <= 2^20 and rows < 2^31");
    return CLEAR_OK;
}
// Codes and scales of `rows` rows: [rows] of ld bytes, [groups] of ld_scales bytes.
int check_mx_operand(const void* codes, const void* scales, long long ld, long long ld_scales, long long rows, int channels)
{
    if (!codes || !scales) return invalid("codes and scales must be non-NULL");
    if (!aligned(codes, 16) || !aligned(scales, 8)) return invalid("codes must be 16-byte, scales 8-byte aligned");
    if (ld < channels / 2) return invalid("a row of codes is longer than its stride");
    if (ld % 16 || ld > kMxMaxChannels) return unsupported("strides of codes must be multiples of 16 and <= 2^20");
    if (channels > 256 && ld_scales < rows * 8) return invalid("a group of scales is longer than its stride");
    if (ld_scales < 0 || ld_scales % 8 || ld_scales > (1LL << 35)) return unsupported("strides of scales must be multiples of 8, >= 0 and <= 2^35");
    return CLEAR_OK;
}
Span piece(const void* p, long long count, long long ld, long long width)
{
    return {(__int128)(uintptr_t)p, (__int128)(uintptr_t)p + (__int128)(count - 1) * ld + width};
}
Span codes_span(const void* p, long long rows, long long ld, int channels) { return piece(p, rows, ld, channels / 2); }
Span scales_span(const void* p, long long rows, long long ld, int channels) { return piece(p, (channels + 255) / 256, ld, rows * 8); }
// A single row has no stride, nor has a single group of scales: what their tensors say is not looked at.
long long mx_row(long long rows, long long ld, int width) { return rows == 1 ? (width + 15) / 16 * 16 : ld; }
long long mx_group(int channels, long long ld, long long rows) { return channels <= 256 ? rows * 8 : ld; }

}  // namespace

int clear_block_mx_quantize(const void* X, void* codes, void* scales, long long rows, int channels, long long ld_x, long long ld_codes, long long ld_scales, int dtype, void* stream)
{
    int rc = check_mx(rows, channels);
    if (rc != CLEAR_OK) return rc;
    if (!known_dtype(dtype)) return invalid("dtype must be CLEAR_BF16 or CLEAR_F32");
    if (rows == 0) return CLEAR_OK;
    if (rows == 1) ld_x = channels;
    ld_codes = mx_row(rows, ld_codes, channels / 2), ld_scales = mx_group(channels, ld_scales, rows);
    if ((rc = check_mx_operand(codes, scales, ld_codes, ld_scales, rows, channels)) != CLEAR_OK) return rc;
    if (!X || !aligned(X, size_of(dtype))) return invalid("X must be non-NULL and aligned to its elements");
    if (ld_x < 0) return invalid("strides must be >= 0");
    if (ld_x > (1LL << 32)) return unsupported("the row stride of X must be <= 2^32");
    const Span x = piece(X, rows, ld_x * size_of(dtype), (long long)channels * size_of(dtype)), c = codes_span(codes, rows, ld_codes, channels), s = scales_span(scales, rows, ld_scales, channels);
    if (overlap(x, c) || overlap(x, s) || overlap(c, s)) return invalid("X, codes and scales must not overlap");
    MxArgs a = {};
    a.x = X, a.codes_out = codes, a.scales_out = scales, a.rows = rows, a.channels = channels, a.ld_x = ld_x, a.ld_codes = ld_codes, a.ld_scales = ld_scales;
    return launched(launch_mx_quantize(a, dtype, (hipStream_t)stream), "quantisation launch failed: ");
}

int clear_block_mx_dequantize(const void* codes, const void* scales, void* Y, long long rows, int channels, long long ld_codes, long long ld_scales, long long ld_y, int dtype, void* stream)
{
    int rc = check_mx(rows, channels);
    if (rc != CLEAR_OK) return rc;
    if (!known_dtype(dtype)) return invalid("dtype must be CLEAR_BF16 or CLEAR_F32");
    if (rows == 0) return CLEAR_OK;
    if (rows == 1) ld_y = channels;
    ld_codes = mx_row(rows, ld_codes, channels / 2), ld_scales = mx_group(channels, ld_scales, rows);
    if ((rc = check_mx_operand(codes, scales, ld_codes, ld_scales, rows, channels)) != CLEAR_OK) return rc;
    if (!Y || !aligned(Y, size_of(dtype))) return invalid("Y must be non-NULL and aligned to its elements");
    if (ld_y < channels) return invalid("a row stride is shorter than its row");
    if (ld_y > (1LL << 32)) return unsupported("the row stride of Y must be <= 2^32");
    const Span y = piece(Y, rows, ld_y * size_of(dtype), (long long)channels * size_of(dtype));
    if (overlap(y, codes_span(codes, rows, ld_codes, channels)) || overlap(y, scales_span(scales, rows, ld_scales, channels))) return invalid("Y must not overlap codes or scales");
    MxArgs a = {};
    a.codes = codes, a.scales = scales, a.y = Y, a.rows = rows, a.channels = channels, a.ld_codes = ld_codes, a.ld_scales = ld_scales, a.ld_y = ld_y;
    return launched(launch_mx_dequantize(a, dtype, (hipStream_t)stream), "dequantisation launch failed: ");
}

int clear_block_mx_linear(const void* X, const void* X_scales, const void* W, const void* W_scales, const void* bias, void* Y, long long tokens, int channels, int outputs,
                          const long long* strides, int x_dtype, int bias_dtype, int out_dtype, void* workspace, void* stream)
{
    int rc = check_mx(tokens, channels);
    if (rc != CLEAR_OK) return rc;
    if (outputs < 1) return invalid("outputs must be >= 1");
    if (outputs > kMxMaxChannels) return unsupported("outputs must be <= 2^20");
    if (!X_scales && !known_dtype(x_dtype)) return invalid("x_dtype must be CLEAR_BF16 or CLEAR_F32 where X is not in 4 bits");
    if ((bias && !known_dtype(bias_dtype)) || !known_dtype(out_dtype)) return invalid("bias_dtype and out_dtype must be CLEAR_BF16 or CLEAR_F32");
    if (tokens == 0) return CLEAR_OK;
    if (!X || !Y || !strides) return invalid("X, Y and strides must be non-NULL");
    long long ld_x = strides[0], ld_xs = strides[1], ld_w = mx_row(outputs, strides[2], channels / 2), ld_ws = mx_group(channels, strides[3], outputs), ld_y = strides[4];
    if (tokens == 1) ld_y = outputs;
    if ((rc = check_mx_operand(W, W_scales, ld_w, ld_ws, outputs, channels)) != CLEAR_OK) return rc;
    const int out_size = size_of(out_dtype);
    Span x[2];
    if (X_scales) {
        ld_x = mx_row(tokens, ld_x, channels / 2), ld_xs = mx_group(channels, ld_xs, tokens);
        if ((rc = check_mx_operand(X, X_scales, ld_x, ld_xs, tokens, channels)) != CLEAR_OK) return rc;
        x[0] = codes_span(X, tokens, ld_x, channels), x[1] = scales_span(X_scales, tokens, ld_xs, channels);
    } else {
        if (tokens == 1) ld_x = channels;
        if (!aligned(X, size_of(x_dtype))) return invalid("X must be aligned to its elements");
        if (ld_x < 0) return invalid("strides must be >= 0");
        if (ld_x > (1LL << 32)) return unsupported("the row stride of X must be <= 2^32");
        x[0] = x[1] = piece(X, tokens, ld_x * size_of(x_dtype), (long long)channels * size_of(x_dtype));
    }
    if (!aligned(Y, out_size) || !aligned(bias, bias ? size_of(bias_dtype) : 1) || !aligned(workspace, 16)) return invalid("Y and bias must be aligned to their elements, the workspace to 16 bytes");
    if (ld_y < outputs) return invalid("a row stride is shorter than its row");
    if (ld_y > (1LL << 32)) return unsupported("the row stride of Y must be <= 2^32");
    if (!workspace && mx_linear_workspace_bytes(tokens, channels, outputs, X_scales != nullptr) > 0) return invalid("workspace must be non-NULL");
    const Span y = piece(Y, tokens, ld_y * out_size, (long long)outputs * out_size);
    if (overlap(y, x[0]) || overlap(y, x[1]) || overlap(y, codes_span(W, outputs, ld_w, channels)) || overlap(y, scales_span(W_scales, outputs, ld_ws, channels)) ||
        (bias && overlap(y, piece(bias, 1, 0, (long long)outputs * size_of(bias_dtype)))))
        return invalid("Y must not overlap an input");
    MxLinearArgs a = {};
    a.x = X, a.xs = X_scales, a.w = W, a.ws = W_scales, a.bias = bias, a.y = Y;
    a.tokens = tokens, a.channels = channels, a.outputs = outputs;
    a.ld_x = ld_x, a.ld_xs = ld_xs, a.ld_w = ld_w, a.ld_ws = ld_ws, a.ld_y = ld_y;
    a.x_dtype = x_dtype, a.bias_dtype = bias_dtype, a.out_dtype = out_dtype;
    a.workspace = workspace;
    return launched(launch_mx_linear(a, (hipStream_t)stream), "4-bit product launch failed: ");
}

long long clear_block_mx_linear_workspace(long long tokens, int channels, int outputs, int quantized)
{
    if (check_mx(tokens, channels) != CLEAR_OK) return -1;
    if (outputs < 1 || outputs > kMxMaxChannels) return unsupported("outputs must be in [1, 2^20]"), -1;
    return (long long)mx_linear_workspace_bytes(tokens, channels, outputs, quantized != 0);
}
