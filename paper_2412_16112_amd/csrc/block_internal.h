// Launchers of the operators around the attention (block_api.cpp calls them with checked arguments) and the vector types
// that their kernels share.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/clear_block.h"

namespace clear {
namespace block {

// ---- rotary positions
struct RotaryArgs {
    const void *q, *k;
    void *q_out, *k_out;
    int Hq, Hk;
    long long st[12];  // (batch, head, token) of q, q_out, k, k_out
    long long B, N;
    int head_dim, rot_dim, copy;  // copy: the channels from rot_dim on are copied
    const void* positions;
    long long ps[3];
    int n_axes;
    const double* freqs;
    float scale, sign;
};
hipError_t launch_rotary(const RotaryArgs& a, bool interleaved, bool wide_positions, int dtype, hipStream_t stream);

// ---- layer norm
constexpr int kNormMaxChannels = 16384;
struct NormArgs {
    const void *x, *w, *b, *dy;
    void *y, *dx, *dw, *db;
    float *stats, *ws;
    int groups, rows, channels;
    long long st[6];  // forward: (group, row) of x, y; backward: of dy, x, dx
    int per_group;
    float eps, offset;
};
hipError_t launch_norm_forward(const NormArgs& a, int dtype, int weight_dtype, hipStream_t stream);
hipError_t launch_norm_backward(const NormArgs& a, int dtype, int weight_dtype, hipStream_t stream);
int norm_partials(long long groups, long long rows, int channels, int per_group);  // workgroups whose sums of d_weight and d_bias a set is joined from

// ---- gated feed-forward projection
struct GatedArgs {
    const void *x, *wg, *wu, *dh;
    void *h, *dx, *dwg, *dwu;
    float* pre;
    long long tokens;
    int channels, hidden, act;
    long long ld_x, ld_g, ld_u, ld_h, ld_dh, ld_dx, ld_dwg, ld_dwu;
    void* ws;
};
hipError_t launch_gated_forward(const GatedArgs& a, hipStream_t stream);
hipError_t launch_gated_backward(const GatedArgs& a, hipStream_t stream);
size_t gated_workspace_bytes(long long tokens, int channels, int hidden);

// ---- AdamW
constexpr int kAdamTensors = 56;  // as many descriptors as fit the 4 KB of a launch's arguments
constexpr int kAdamBlock = 256;   // elements that share a scale of 8-bit states
struct AdamHyper {
    float beta1, one_minus_beta1, beta2, one_minus_beta2, keep, step_size, inv_root_correction, eps;
    const float* grad_scale;
};
hipError_t launch_adamw(int n, const clear_block_adamw_tensor* tensors, const AdamHyper& h, int dtype, int state_bits, hipStream_t stream);
hipError_t launch_adamw_decode(const void* m, const float* ms, const void* v, const float* vs, float* m_out, float* v_out, long long n,
                               hipStream_t stream);

// ---- device types.  Callers' tensors need the alignment of their elements only: global memory takes a wide access at any
// address, and the types say so to the compiler.
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8), aligned(2))) __bf16 bf16x8_any;
typedef __attribute__((ext_vector_type(4), aligned(2))) __bf16 bf16x4_any;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;

// 8 elements as two fours, the second GAP elements behind the first (4: side by side); of the first 4 .. 8 the first n exist, of the second those that are then left
// (n - GAP).  Elements that do not exist are 0 / are not written.
template <typename T>
struct Chunk8;
template <>
struct Chunk8<__bf16> {
    bf16x8 v;
    template <int GAP = 4>
    __device__ __forceinline__ void load(const __bf16* p, int n)
    {
        if constexpr (GAP == 4) {
            if (n >= 8) {
                v = *(const bf16x8_any*)p;
                return;
            }
        }
        const bf16x4 lo = four(p, n), hi = four(p + GAP, n - GAP);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = lo[j], v[4 + j] = hi[j];
    }
    __device__ __forceinline__ float get(int j) const { return (float)v[j]; }
    template <int GAP = 4>
    static __device__ __forceinline__ void store(__bf16* p, int n, const float (&x)[8])
    {
        static_assert(GAP == 4, "rows of bf16 are stored in eights");
        bf16x8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (__bf16)x[j];
        if (n >= 8) {
            *(bf16x8_any*)p = o;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) p[j] = o[j];
        }
    }
    static __device__ __forceinline__ bf16x4 four(const __bf16* p, int n)
    {
        bf16x4 x;
        if (n >= 4) {
            x = *(const bf16x4_any*)p;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = j < n ? p[j] : (__bf16)0.f;
        }
        return x;
    }
};
template <>
struct Chunk8<float> {
    f32x4 lo, hi;
    template <int GAP = 4>
    __device__ __forceinline__ void load(const float* p, int n)
    {
        lo = four(p, n);
        hi = four(p + GAP, n - GAP);
    }
    __device__ __forceinline__ float get(int j) const { return j < 4 ? lo[j & 3] : hi[j & 3]; }
    template <int GAP = 4>
    static __device__ __forceinline__ void store(float* p, int n, const float (&x)[8])
    {
        store_four(p, n, f32x4{x[0], x[1], x[2], x[3]});
        store_four(p + GAP, n - GAP, f32x4{x[4], x[5], x[6], x[7]});
    }
    static __device__ __forceinline__ f32x4 four(const float* p, int n)
    {
        f32x4 x;
        if (n >= 4) {
            x = *(const f32x4_any*)p;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = j < n ? p[j] : 0.f;
        }
        return x;
    }
    static __device__ __forceinline__ void store_four(float* p, int n, f32x4 x)
    {
        if (n >= 4) {
            *(f32x4_any*)p = x;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < n) p[j] = x[j];
        }
    }
};

// join over the wave's values, in every lane (exchanges inside rows of 16 lanes, then between rows: no LDS).
template <typename F>
__device__ __forceinline__ float wave_reduce(float x, F&& join)
{
    const auto beside = [](float v, auto ctrl) {
        constexpr int c = ctrl;
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), c, 0xf, 0xf, true));
    };
    x = join(x, beside(x, std::integral_constant<int, 0xb1>{}));   // lane ^ 1
    x = join(x, beside(x, std::integral_constant<int, 0x4e>{}));   // lane ^ 2
    x = join(x, beside(x, std::integral_constant<int, 0x141>{}));  // the other half of 8 lanes
    x = join(x, beside(x, std::integral_constant<int, 0x140>{}));  // the other half of 16
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = join(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return join(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float wave_sum(float x)
{
    return wave_reduce(x, [](float a, float b) { return a + b; });
}

}  // namespace block
}  // namespace clear
