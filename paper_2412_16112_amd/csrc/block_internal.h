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

// How a row's chunks lie in it: `whole`: all lanes have all 8 elements of theirs; `tiny`: the row has less than 8.
struct RowForm {
    bool whole, tiny;
};

// 8 elements of a row, one piece of 8 (GAP 4) or two of 4, the second GAP elements behind the first.  From the chunk's place on, the row has n elements left.  A piece that
// reaches past the end is taken further in front, so that it ends with the row; its elements that belong to the lane before are not the lane's own().  So a lane has one
// load for a piece and no branch but for having none, and nothing waits for a load where it is asked for.
template <int GAP>
struct Piece {
    static __device__ __forceinline__ int first(int j) { return GAP == 4 || j < 4 ? 0 : GAP; }                        // of element j's piece
    static __device__ __forceinline__ int back(int j, int n) { return max((GAP == 4 ? 8 : 4) - (n - first(j)), 0); }  // how far it is taken in front
    static __device__ __forceinline__ int in(int j) { return GAP == 4 ? j : j & 3; }                                  // element j's place in it
    // Where element j is, from the chunk's place, and whether it is the lane's own.
    static __device__ __forceinline__ int at(int j, int n, RowForm form) { return first(j) + in(j) - (form.whole || form.tiny ? 0 : back(j, n)); }
    static __device__ __forceinline__ bool own(int j, int n, RowForm form)
    {
        if (form.whole) return true;
        if (form.tiny) return first(j) + in(j) < n;
        return n > first(j) && in(j) >= back(j, n);
    }
};

template <typename T>
struct Chunk8;
template <>
struct Chunk8<__bf16> {
    bf16x8 v;
    template <int GAP>
    __device__ __forceinline__ void load(const __bf16* p, int n, RowForm form)
    {
        typedef Piece<GAP> P;
        if (form.tiny) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = P::own(j, n, form) ? p[P::at(j, n, form)] : (__bf16)0.f;
        } else if (GAP == 4 && form.whole) {
            v = *(const bf16x8_any*)p;
        } else if (GAP == 4) {
            v = bf16x8{};
            if (n > 0) v = *(const bf16x8_any*)(p + P::at(0, n, form));
        } else {
            bf16x4 lo = {}, hi = {};
            if (form.whole) {
                lo = *(const bf16x4_any*)p;
                hi = *(const bf16x4_any*)(p + GAP);
            } else {
                if (n > 0) lo = *(const bf16x4_any*)(p + P::at(0, n, form));
                if (n > GAP) hi = *(const bf16x4_any*)(p + P::at(4, n, form));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = lo[j], v[4 + j] = hi[j];
        }
    }
    template <int GAP>
    __device__ __forceinline__ void clear_others(int n, RowForm form)  // elements that are not the lane's own: 0
    {
        if (form.whole) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = Piece<GAP>::own(j, n, form) ? v[j] : (__bf16)0.f;
    }
    __device__ __forceinline__ float get(int j) const { return (float)v[j]; }
    template <int GAP>
    static __device__ __forceinline__ void store(__bf16* p, int n, RowForm form, const float (&x)[8])
    {
        static_assert(GAP == 4, "rows of bf16 are stored in eights");
        typedef Piece<GAP> P;
        bf16x8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (__bf16)x[j];
        if (form.whole || P::back(0, n) == 0) {
            *(bf16x8_any*)p = o;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (P::own(j, n, form)) p[P::at(j, n, form)] = o[j];
        }
    }
};
template <>
struct Chunk8<float> {
    f32x4 lo, hi;
    template <int GAP>
    __device__ __forceinline__ void load(const float* p, int n, RowForm form)
    {
        typedef Piece<GAP> P;
        if (form.tiny) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = P::own(j, n, form) ? p[P::at(j, n, form)] : 0.f;
                hi[j] = P::own(4 + j, n, form) ? p[P::at(4 + j, n, form)] : 0.f;
            }
        } else if (form.whole) {
            lo = *(const f32x4_any*)p;
            hi = *(const f32x4_any*)(p + GAP);
        } else {
            lo = hi = f32x4{};
            if (n > 0) lo = *(const f32x4_any*)(p + P::at(0, n, form));
            if (n > P::first(4)) hi = *(const f32x4_any*)(p + P::at(4, n, form));
        }
    }
    template <int GAP>
    __device__ __forceinline__ void clear_others(int n, RowForm form)
    {
        if (form.whole) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            lo[j] = Piece<GAP>::own(j, n, form) ? lo[j] : 0.f;
            hi[j] = Piece<GAP>::own(4 + j, n, form) ? hi[j] : 0.f;
        }
    }
    __device__ __forceinline__ float get(int j) const { return j < 4 ? lo[j & 3] : hi[j & 3]; }
    template <int GAP>
    static __device__ __forceinline__ void store(float* p, int n, RowForm form, const float (&x)[8])
    {
        typedef Piece<GAP> P;
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            if (form.whole || P::back(h, n) == 0) {
                *(f32x4_any*)(p + P::first(h) + P::in(h)) = f32x4{x[h], x[h + 1], x[h + 2], x[h + 3]};
            } else {
#pragma unroll
                for (int j = h; j < h + 4; ++j)
                    if (P::own(j, n, form)) p[P::at(j, n, form)] = x[j];
            }
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
