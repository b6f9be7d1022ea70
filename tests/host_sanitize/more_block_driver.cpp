// Drives the C entry points of the gated residual with its norms, the norm of gradients and the operands in 4 bits under the host sanitizers: arguments of every kind, refused and accepted, with launchers
// that check what they are given instead of launching.
#include <cassert>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <string>
#include <vector>

#include "../../paper_2412_16112_amd/csrc/block_internal.h"

static int launches = 0;
static std::string reason;

namespace clear {
namespace block {
int fail(int code, const char* what, const char* why) noexcept
{
    reason = std::string(what) + why;
    assert(code != CLEAR_OK && !reason.empty());
    return code;
}
static bool at(const void* p, int to) { return ((uintptr_t)p & (to - 1)) == 0; }
hipError_t launch_residual_forward(const ResidualArgs& a, int dtype, int stream_dtype, int, hipStream_t)
{
    ++launches;
    assert(a.x && a.y && a.r && a.h && a.groups > 0 && a.rows > 0 && a.channels > 0 && a.channels <= kResidualMaxChannels);
    assert(dtype == CLEAR_BF16 || stream_dtype == CLEAR_F32);
    assert(a.kind == CLEAR_NORM_LAYER || a.kind == CLEAR_NORM_RMS);
    assert(a.post != CLEAR_NORM_NONE || !a.pw);
    for (int i = 0; i < 8; ++i) assert(a.st[i] >= 0);
    return hipSuccess;
}
hipError_t launch_residual_backward(const ResidualArgs& a, int, int, int, hipStream_t)
{
    ++launches;
    assert(a.dx || a.dy || a.dgate || a.dw || a.db || a.dpw);
    assert(a.groups > 0 || (!a.per_group && !a.gate_per_group));
    if (a.groups > 0 && a.rows > 0) assert(a.dh && a.x && a.y && a.stats && ((!a.dgate && !a.dw && !a.db && !a.dpw) || a.ws));
    return hipErrorInvalidValue;  // (an error of a launch is reported, not thrown)
}
int residual_partials(long long groups, long long rows, int, long long sets) { return groups * rows == 0 || sets == 0 ? 0 : 256; }
hipError_t launch_grad_norm(int n, const clear_block_grad* t, const GradFactor& f, void*, hipStream_t)
{
    ++launches;
    for (int i = 0; i < n; ++i) assert(t[i].n >= 0 && t[i].n <= 1LL << 35 && at(t[i].data, t[i].dtype == CLEAR_F32 ? 4 : 2));
    assert(f.norm || f.factor);
    return hipSuccess;
}
hipError_t launch_grad_clip(int n, const clear_block_grad* t, const GradFactor&, void*, hipStream_t)
{
    ++launches;
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j) {
            const char *p = (const char*)t[i].data, *q = (const char*)t[j].data;
            const long long a = t[i].n * (t[i].dtype == CLEAR_F32 ? 4 : 2), b = t[j].n * (t[j].dtype == CLEAR_F32 ? 4 : 2);
            assert(!p || !q || a == 0 || b == 0 || p + a <= q || q + b <= p);
        }
    return hipSuccess;
}
hipError_t launch_grad_scale(int n, const clear_block_grad* t, const float* factor, hipStream_t stream)
{
    assert(factor && at(factor, 4));
    return launch_grad_clip(n, t, GradFactor{}, nullptr, stream);
}
long long grad_norm_partials(int n, const clear_block_grad* t)
{
    long long all = 0;
    for (int i = 0; i < n; ++i) all += t[i].data && t[i].n;
    return all;
}
hipError_t launch_mx_quantize(const MxArgs& a, int, hipStream_t)
{
    ++launches;
    assert(a.rows > 0 && a.channels > 0 && a.channels % 32 == 0 && a.ld_codes % 16 == 0 && a.ld_scales % 8 == 0 && a.ld_codes >= a.channels / 2 && at(a.codes_out, 16) && at(a.scales_out, 8));
    return hipSuccess;
}
hipError_t launch_mx_dequantize(const MxArgs& a, int, hipStream_t)
{
    ++launches;
    assert(a.rows > 0 && a.channels % 32 == 0 && a.ld_codes % 16 == 0 && a.ld_y >= a.channels && at(a.codes, 16) && at(a.scales, 8));
    return hipSuccess;
}
hipError_t launch_mx_linear(const MxLinearArgs& a, hipStream_t)
{
    ++launches;
    assert(a.tokens > 0 && a.outputs > 0 && a.channels % 32 == 0 && a.ld_w % 16 == 0 && a.ld_w <= 1 << 20 && a.ld_y >= a.outputs && at(a.w, 16) && at(a.ws, 8));
    assert(!a.xs || (a.ld_x % 16 == 0 && a.ld_x <= 1 << 20 && at(a.x, 16) && at(a.xs, 8)));
    return hipSuccess;
}
size_t mx_linear_workspace_bytes(long long tokens, int channels, int, bool quantized) { return quantized ? 0 : (size_t)tokens * channels; }
}  // namespace block
}  // namespace clear

static uint64_t state = 12345;
static uint64_t draw()
{
    state = state * 6364136223846793005ULL + 1442695040888963407ULL;
    return state >> 20;
}
static long long pick(std::vector<long long> of) { return of[draw() % of.size()]; }
static long long usual(long long value) { return draw() % 6 ? value : pick({-1, 0, 1, 7, value + 1, value + 8, value * 2, 1LL << 31, (1LL << 31) - 1, 1LL << 32, 1LL << 48, (1LL << 48) + 1, LLONG_MAX, LLONG_MIN}); }
static int small(long long value) { return (int)(draw() % 6 ? value : pick({-1, 0, 1, 31, 32, 33, 8192, 8193, 1 << 20, (1 << 20) + 32, INT_MAX, INT_MIN})); }
static float number() { return draw() % 8 ? 1.f : (draw() % 2 ? NAN : INFINITY); }
static char* place(int n) { return draw() % 9 ? (char*)((uintptr_t)(n + 1) << 44) + (draw() % 12 ? 0 : draw() % 64) : draw() % 2 ? nullptr : (char*)((uintptr_t)(draw() % 20 + 1) << 44); }

int main()
{
    for (int round = 0; round < 60000; ++round) {
        const long long groups = usual(pick({1, 2, 5})), rows = usual(pick({1, 10, 300}));
        const int C = small(pick({1, 64, 256, 2432}));
        std::vector<long long> st;
        for (int i = 0; i < 6; ++i) st.push_back(usual((long long)C * pick({1, 10, 300}))), st.push_back(usual(C));
        const int kind = (int)pick({0, 1, 1, 2, 2, 3}), post = (int)pick({-1, 0, 0, 1, 2, 3}), dt = (int)pick({0, 0, 1, 2}), sd = (int)pick({0, 1, 1, 2}), wd = (int)pick({0, 1, -1});
        clear_block_residual_norm(place(0), place(1), place(2), place(3), place(4), place(5), place(6), place(7), (float*)place(8), groups, rows, C, draw() % 20 ? st.data() : nullptr, draw() % 2, draw() % 2, kind,
                                  post, number(), number(), number(), number(), dt, sd, wd, nullptr);
        clear_block_residual_norm_backward(place(0), place(1), place(2), place(3), place(4), place(5), place(6), (float*)place(7), place(8), place(9), place(10), place(11), place(12), place(13), groups, rows, C,
                                           draw() % 20 ? st.data() : nullptr, draw() % 2, draw() % 2, kind, post, number(), number(), number(), dt, sd, wd, (float*)place(14), nullptr);
        clear_block_residual_norm_workspace(groups, rows, C, draw() % 2, draw() % 2);

        std::vector<clear_block_grad> g;
        const int n = (int)(draw() % 6);
        for (int i = 0; i < n; ++i) g.push_back({place(i), usual(pick({0, 5, 1000})), draw() % 30 ? (int)(draw() % 2) : 2});
        const int count = draw() % 20 ? n : -1;
        const double bound = draw() % 8 ? 1.0 : draw() % 2 ? NAN : -1.0;
        clear_block_grad_norm_workspace(count, g.data());
        clear_block_grad_norm(count, g.data(), (int)pick({0, 0, 1, 2}), bound, (float*)place(16), (float*)place(17), (float*)place(18), place(19), nullptr);
        clear_block_grad_clip(count, g.data(), (int)pick({0, 0, 1, 2}), bound, (float*)place(16), (float*)place(17), (float*)place(18), place(19), nullptr);
        clear_block_grad_scale(count, g.data(), (float*)place(18), nullptr);

        const long long tokens = usual(pick({1, 10, 300}));
        const int K = small(pick({32, 256, 2432})), F = small(pick({1, 33, 1000}));
        const long long lx = usual(draw() % 2 ? K : K / 2), lxs = usual(tokens > 0 && tokens < 1000 ? tokens * 8 : 8), lw = usual(K / 2), lws = usual(F > 0 && F < 5000 ? F * 8LL : 8), ly = usual(F);
        clear_block_mx_quantize(place(0), place(1), place(2), tokens, K, lx, usual(K / 2), lxs, dt, nullptr);
        clear_block_mx_dequantize(place(1), place(2), place(0), tokens, K, usual(K / 2), lxs, usual(K), dt, nullptr);
        const long long five[5] = {lx, lxs, lw, lws, ly};
        clear_block_mx_linear(place(0), place(1), place(2), place(3), place(4), place(5), tokens, K, F, draw() % 20 ? five : nullptr, dt, wd, sd, place(6), nullptr);
        clear_block_mx_linear_workspace(tokens, K, F, draw() % 2);
    }
    assert(launches > 1000);
    std::printf("clean under the sanitizers, %d launches\n", launches);
    return 0;
}
