// Rotary positions for the queries and keys of a block in one launch.  Memory-bound: every element is read and written once.
//
// A thread takes one unit of channels of one token and goes through a range of the heads: its angles (fp64 products and
// reduction to a turn, then fp32 sine and cosine) are formed once for all of them.  A unit is 16 bytes of a head's row, or of each half of
// the turned channels where a pair lies half of them apart; units past the turned channels are copies.  Neighbouring threads take
// neighbouring units, then neighbouring tokens.  16 896 tokens x 48 heads of 128 channels, bf16: 91 us, 4.6 TB/s; 8 314 x 76 heads of 64, fp32: 63 us, 5.1 TB/s; 16 tokens x 40
// heads: 6.6 us.
#include <algorithm>

#include "block_internal.h"

namespace clear {
namespace block {
namespace {

constexpr int kThreads = 256;
constexpr int kHeadsInFlight = 8;

template <typename T>
struct Vec;
template <>
struct Vec<__bf16> {
    static constexpr int n = 8;
    typedef bf16x8 type;
    typedef bf16x8_any any;
};
template <>
struct Vec<float> {
    static constexpr int n = 4;
    typedef f32x4 type;
    typedef f32x4_any any;
};

// The first `count` of the elements at p (all of them where count is no less).
template <typename T>
__device__ __forceinline__ typename Vec<T>::type load_some(const T* p, int count)
{
    typename Vec<T>::type v;
    if (count >= Vec<T>::n) return *(const typename Vec<T>::any*)p;
#pragma unroll
    for (int j = 0; j < Vec<T>::n; ++j) v[j] = j < count ? p[j] : (T)0.f;
    return v;
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, int count, const typename Vec<T>::type& v)
{
    if (count >= Vec<T>::n) {
        *(typename Vec<T>::any*)p = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < Vec<T>::n; ++j)
        if (j < count) p[j] = v[j];
}

// FULL: every unit has all of its channels.
template <typename T, bool INTERLEAVED, typename P, bool FULL>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a, long long token_first, long long n_threads, int units, int turned_units, int heads_each)
{
    constexpr int V = Vec<T>::n, PAIRS = INTERLEAVED ? V / 2 : V;
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (id >= n_threads) return;
    const unsigned of = (unsigned)id / (unsigned)units;  // (a launch has fewer than 2^31 threads)
    const int u = (int)((unsigned)id - of * units);
    const long long token = token_first + of;
    const long long b = token / a.N, n = token - b * a.N;
    const int half = a.rot_dim / 2;
    const bool turn = u < turned_units;
    // first channel, number of channels and, for the half layout, the distance to the other channel of a pair
    const int c0 = turn ? (INTERLEAVED ? V : PAIRS) * u : a.rot_dim + V * (u - turned_units);
    const int count = FULL ? V : turn ? (INTERLEAVED ? a.rot_dim - c0 : half - c0) : a.head_dim - c0;
    float cs[PAIRS], sn[PAIRS];
    if (turn) {
        double at[4];
#pragma unroll
        for (int ax = 0; ax < 4; ++ax) at[ax] = ax < a.n_axes ? (double)((const P*)a.positions)[ax * a.ps[0] + b * a.ps[1] + n * a.ps[2]] : 0.0;
        const int i0 = PAIRS * u;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            double angle = 0.0;
            if (i0 + i < half) {
#pragma unroll
                for (int ax = 0; ax < 4; ++ax)
                    if (ax < a.n_axes) angle += at[ax] * a.freqs[(long long)ax * half + i0 + i];
            }
            angle *= 0.15915494309189533577;  // 1 / (2 pi)
            const float part = (float)(angle - rint(angle));  // of a turn, in [-1/2, 1/2]
            float s, c;
            sincospif(2.f * part, &s, &c);
            cs[i] = c * a.scale;
            sn[i] = s * a.scale * a.sign;
        }
    }
    const int heads = a.Hq + a.Hk;
    const int h0 = blockIdx.y * heads_each, h1 = min(h0 + heads_each, heads);
    const long long in_q = b * a.st[0] + n * a.st[2], out_q = b * a.st[3] + n * a.st[5];
    const long long in_k = b * a.st[6] + n * a.st[8], out_k = b * a.st[9] + n * a.st[11];
    for (int hb = h0; hb < h1; hb += kHeadsInFlight) {
        typename Vec<T>::type x[kHeadsInFlight], y[kHeadsInFlight];
#pragma unroll
        for (int i = 0; i < kHeadsInFlight; ++i) {
            const int h = hb + i;
            if (h < h1) {
                const T* const p = (h < a.Hq ? (const T*)a.q + in_q + h * a.st[1] : (const T*)a.k + in_k + (h - a.Hq) * a.st[7]) + c0;
                x[i] = load_some<T>(p, count);
                if (!INTERLEAVED && turn) y[i] = load_some<T>(p + half, count);
            }
        }
#pragma unroll
        for (int i = 0; i < kHeadsInFlight; ++i) {
            const int h = hb + i;
            if (h < h1) {
                T* const p = (h < a.Hq ? (T*)a.q_out + out_q + h * a.st[4] : (T*)a.k_out + out_k + (h - a.Hq) * a.st[10]) + c0;
                if (turn) {
#pragma unroll
                    for (int j = 0; j < PAIRS; ++j) {
                        if (INTERLEAVED) {
                            const float e = (float)x[i][2 * j], o = (float)x[i][2 * j + 1];
                            x[i][2 * j] = (T)(e * cs[j] - o * sn[j]);
                            x[i][2 * j + 1] = (T)(e * sn[j] + o * cs[j]);
                        } else {
                            const float e = (float)x[i][j], o = (float)y[i][j];
                            x[i][j] = (T)(e * cs[j] - o * sn[j]);
                            y[i][j] = (T)(e * sn[j] + o * cs[j]);
                        }
                    }
                    if (!INTERLEAVED) store_some<T>(p + half, count, y[i]);
                }
                store_some<T>(p, count, x[i]);
            }
        }
    }
}

template <typename T, bool INTERLEAVED, typename P>
hipError_t launch(const RotaryArgs& a, hipStream_t stream)
{
    constexpr int V = Vec<T>::n, PAIRS = INTERLEAVED ? V / 2 : V;
    const int turned = (a.rot_dim / 2 + PAIRS - 1) / PAIRS, units = turned + (a.copy ? (a.head_dim - a.rot_dim + V - 1) / V : 0);
    const bool full = a.rot_dim / 2 % PAIRS == 0 && (!a.copy || (a.head_dim - a.rot_dim) % V == 0);
    const long long tokens = a.B * a.N;
    const int heads = a.Hq + a.Hk;
    // All heads of a token in one thread, so that its angles are formed once; fewer where that would leave CUs without work (under
    // 8 workgroups a CU), down to the heads whose loads are in flight together.
    const long long blocks = (tokens * units + kThreads - 1) / kThreads;
    const int groups = (heads + kHeadsInFlight - 1) / kHeadsInFlight;
    const int split = (int)std::min<long long>(groups, std::max<long long>(1, 2048 / std::max<long long>(1, blocks)));
    const int heads_each = (groups + split - 1) / split * kHeadsInFlight;
    const long long most = 0x7fffffffLL / 2 / units;  // tokens a launch can have
    for (long long first = 0; first < tokens; first += most) {
        const long long n = std::min(most, tokens - first) * units;
        const dim3 grid((unsigned)((n + kThreads - 1) / kThreads), (heads + heads_each - 1) / heads_each);
        if (full)
            rotary_kernel<T, INTERLEAVED, P, true><<<grid, dim3(kThreads), 0, stream>>>(a, first, n, units, turned, heads_each);
        else
            rotary_kernel<T, INTERLEAVED, P, false><<<grid, dim3(kThreads), 0, stream>>>(a, first, n, units, turned, heads_each);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch(const RotaryArgs& a, bool interleaved, bool wide, hipStream_t stream)
{
    if (interleaved) return wide ? launch<T, true, long long>(a, stream) : launch<T, true, int>(a, stream);
    return wide ? launch<T, false, long long>(a, stream) : launch<T, false, int>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, bool interleaved, bool wide_positions, int dtype, hipStream_t stream)
{
    return dtype == CLEAR_BF16 ? launch<__bf16>(a, interleaved, wide_positions, stream) : launch<float>(a, interleaved, wide_positions, stream);
}

}  // namespace block
}  // namespace clear
