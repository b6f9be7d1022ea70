// Drives the C entry points of the operators around the attention under the host sanitizers: arguments of every kind, refused and accepted, with launchers that
// check what they are given instead of launching.
#include <cassert>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <string>
#include <vector>

#include "../../paper_2412_16112_amd/csrc/block_internal.h"

static int launches = 0;

namespace clear {
namespace block {
hipError_t launch_rotary(const RotaryArgs& a, bool, bool, int, hipStream_t)
{
    ++launches;
    assert(a.q && a.q_out && a.Hq > 0 && a.B > 0 && a.N > 0 && a.rot_dim <= a.head_dim && a.n_axes >= 1 && a.n_axes <= 4);
    assert((a.k == nullptr) == (a.Hk == 0));
    return hipSuccess;
}
hipError_t launch_norm_forward(const NormArgs& a, int, int, hipStream_t)
{
    ++launches;
    assert(a.x && a.y && a.groups > 0 && a.rows > 0 && a.channels > 0 && a.channels <= kNormMaxChannels);
    return hipSuccess;
}
hipError_t launch_norm_backward(const NormArgs& a, int, int, hipStream_t)
{
    ++launches;
    assert(a.dx || a.dw || a.db);
    return hipErrorInvalidValue;  // (an error of a launch is reported, not thrown)
}
int norm_partials(long long groups, long long rows, int, int) { return groups * rows == 0 ? 0 : 256; }
hipError_t launch_gated_forward(const GatedArgs& a, hipStream_t)
{
    ++launches;
    assert(a.tokens > 0 && a.channels % 8 == 0 && a.hidden % 8 == 0 && a.ld_x >= a.channels && a.ld_h >= a.hidden);
    return hipSuccess;
}
hipError_t launch_gated_backward(const GatedArgs& a, hipStream_t)
{
    ++launches;
    assert(a.dx || a.dwg);
    return hipSuccess;
}
size_t gated_workspace_bytes(long long tokens, int, int hidden) { return (size_t)tokens * hidden * 4; }
hipError_t launch_adamw(int n, const clear_block_adamw_tensor* t, const AdamHyper& h, int, int, hipStream_t)
{
    ++launches;
    for (int i = 0; i < n; ++i) assert(t[i].n >= 0);
    assert(std::isfinite(h.step_size) && std::isfinite(h.inv_root_correction));
    return hipSuccess;
}
hipError_t launch_adamw_decode(const void*, const float*, const void*, const float*, float*, float*, long long n, hipStream_t)
{
    ++launches;
    assert(n > 0);
    return hipSuccess;
}
}  // namespace block
}  // namespace clear

static unsigned long long state = 88172645463325252ULL;
static unsigned long long next()
{
    state ^= state << 13;
    state ^= state >> 7;
    return state ^= state << 17;
}
template <typename T>
static T pick(const std::vector<T>& v) { return v[next() % v.size()]; }
static const void* place()
{
    static const std::vector<unsigned long long> some = {0, 0x100000000, 0x200000000, 0x300000000, 0x400000000, 0x500000002, 0x600000001, 0x100000010, ~0ULL - 15, 0x7fffffffff00};
    return (const void*)pick(some);
}
static void* out() { return const_cast<void*>(place()); }
static long long extent() { return pick<long long>({-1, 0, 1, 2, 7, 64, 1000, 1LL << 20, 1LL << 31, 1LL << 40, LLONG_MAX, LLONG_MIN}); }
static int small() { return pick<int>({-8, 0, 1, 2, 7, 8, 64, 72, 128, 1000, 4096, 16384, 16385, 1 << 20, INT_MAX, INT_MIN}); }
static double real() { return pick<double>({0, 1, 0.9, 1e-8, -1, 1e300, INFINITY, -INFINITY, NAN}); }

int main()
{
    int status[6] = {};
    const auto count = [&](int s) {
        if (s < 0 || s > 5) abort();
        ++status[s];
        if (s != CLEAR_OK && std::string(clear_block_last_error()).empty()) abort();
    };
    for (int turn = 0; turn < 200000; ++turn) {
        long long st[12];
        for (long long& v : st) v = pick<long long>({0, 1, 64, 640, 2560, 4096, 1LL << 30, 1LL << 48, LLONG_MAX, -1, -64});
        const bool sane = next() & 1;  // half of the turns get sizes that go together
        if (sane) {
            const long long plain[12] = {640, 64, 64, 640, 64, 64, 640, 64, 64, 640, 64, 64};
            std::copy(plain, plain + 12, st);
        }
        const long long B = sane ? 2 : extent(), N = sane ? 1 : extent();
        const void* const q = sane ? (void*)0x100000000 : place();
        count(clear_block_rotary(q, sane ? (void*)0x200000000 : out(), sane ? 10 : small(), sane ? nullptr : place(), sane ? nullptr : out(), sane ? 0 : small(), next() % 50 ? st : nullptr, B, N,
                                 sane ? 64 : small(), sane ? 32 : small(), (int)(next() & 1), sane ? (void*)0x700000000 : place(), sane ? 32 : small(), st, sane ? 2 : small(),
                                 (const double*)(sane ? (void*)0x800000000 : place()), sane ? 1.f : (float)real(), 0, sane ? 1 : small(), nullptr));
        count(clear_block_layer_norm(q, place(), place(), sane ? (void*)0x900000000 : out(), (float*)out(), sane ? 2 : extent(), sane ? 10 : extent(), sane ? 64 : small(), st, (int)(next() & 1),
                                     sane ? 1e-6f : (float)real(), sane ? 0.f : (float)real(), sane ? 1 : small(), sane ? 0 : small(), nullptr));
        count(clear_block_layer_norm_backward(q, place(), place(), (const float*)place(), out(), out(), out(), sane ? 2 : extent(), sane ? 10 : extent(), sane ? 64 : small(), st, (int)(next() & 1),
                                              0.f, sane ? 1 : small(), sane ? 0 : small(), (float*)out(), nullptr));
        (void)clear_block_layer_norm_workspace(extent(), extent(), small(), (int)(next() & 1));
        const long long ld[7] = {sane ? 128 : extent(), sane ? 64 : extent(), sane ? 64 : extent(), sane ? 64 : extent(), sane ? 64 : extent(), sane ? 64 : extent(), sane ? 64 : extent()};
        count(clear_block_gated_ff(q, sane ? (void*)0x200000000 : place(), sane ? (void*)0x300000000 : place(), sane ? (void*)0x400000000 : out(), (float*)out(), sane ? 9 : extent(),
                                   sane ? 64 : small(), sane ? 128 : small(), ld[1], ld[2], ld[3], ld[0], sane ? 2 : small(), nullptr));
        count(clear_block_gated_ff_backward(q, place(), place(), place(), (const float*)place(), out(), out(), out(), sane ? 9 : extent(), sane ? 64 : small(), sane ? 128 : small(),
                                            next() % 50 ? ld : nullptr, sane ? 1 : small(), out(), nullptr));
        (void)clear_block_gated_ff_workspace(extent(), small(), small());
        std::vector<clear_block_adamw_tensor> t(next() % 4);
        for (auto& e : t) e = {out(), place(), (float*)(next() & 1 ? nullptr : out()), out(), out(), (float*)out(), (float*)out(), sane ? 1000 : extent()};
        count(clear_block_adamw(next() % 20 ? (int)t.size() : small() & INT_MIN, t.data(), sane ? 0 : small(), pick<int>({8, 32, 16}), sane ? 1e-3 : real(), sane ? 0.9 : real(),
                                sane ? 0.99 : real(), sane ? 1e-8 : real(), sane ? 0.0 : real(), sane ? 3 : extent(), (const float*)(next() & 1 ? nullptr : place()), nullptr));
        count(clear_block_adamw_decode(place(), (const float*)place(), place(), (const float*)place(), (float*)out(), (float*)out(), extent(), nullptr));
        double f[64];
        count(clear_block_rotary_frequencies(next() % 20 ? f : nullptr, pick<int>({2, 64, 128, 7, 0, -2}), sane ? 500.0 : real(), pick<int>({0, 1, 2, 3, 4, -1}), sane ? 4.0 : real(),
                                             sane ? 100.0 : real(), sane ? 1.0 : real(), sane ? 32.0 : real()));
    }
    printf("%d launches, statuses %d %d %d %d %d %d: clean under the sanitizers\n", launches, status[0], status[1], status[2], status[3], status[4], status[5]);
    return launches > 100000 && status[0] && status[1] && status[2] && status[4] ? 0 : 1;
}
