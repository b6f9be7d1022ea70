// The AdamW step over many tensors in one launch.  Memory-bound: parameter, gradient and states are read once, parameter and
// states written once.  113 M elements: 589 us in bf16 with fp32 masters and states (28 bytes an element, 5.4 TB/s), 345 in fp32 with states of 8 bits (16 bytes, 5.3 TB/s).
//
// A wave takes groups of 256 elements, 4 a lane, which is also the block that shares a scale where states have 8 bits: its largest magnitude is
// then a maximum over the wave.  A workgroup takes kGroups groups for each of its waves, of one tensor; it finds its tensor by bisection in the table of first
// workgroups, which comes with the launch's arguments together with the pointers (nothing is copied to the device beforehand).
//
// Every operation is rounded for itself (no contraction to fma), so that the stored codes of 8 bits, where a last bit can turn a
// rounding, follow from the formulas alone.
#include <algorithm>

#include "block_internal.h"

namespace clear {
namespace block {
namespace {

#pragma clang fp contract(off)

constexpr int kThreads = 256, kWaves = kThreads / 64, kGroups = 4;
constexpr int kChunk = kAdamBlock * kWaves * kGroups;  // elements of a workgroup

struct Launch {
    struct Tensor {
        void* param;
        const void* grad;
        float* master;
        void *m, *v;
        float *m_scale, *v_scale;
        long long n;
    } t[kAdamTensors];
    unsigned first[kAdamTensors + 1];  // first workgroup of each tensor
    int n;
    AdamHyper h;
};
static_assert(sizeof(Launch) <= 4096, "the arguments of a launch are at most 4 KB");

typedef __attribute__((ext_vector_type(4), aligned(1))) signed char i8x4_any;
typedef __attribute__((ext_vector_type(4), aligned(1))) unsigned char u8x4_any;

// 4 consecutive elements as floats, of which the first n exist (the others are 0).
__device__ __forceinline__ f32x4 load4(const float* p, long long n)
{
    if (n >= 4) return *(const f32x4_any*)p;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j < n) v[j] = p[j];
    return v;
}
__device__ __forceinline__ f32x4 load4(const __bf16* p, long long n)
{
    bf16x4 r = {(__bf16)0.f, (__bf16)0.f, (__bf16)0.f, (__bf16)0.f};
    if (n >= 4) {
        r = *(const bf16x4_any*)p;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) r[j] = p[j];
    }
    return f32x4{(float)r[0], (float)r[1], (float)r[2], (float)r[3]};
}
template <typename C, typename CV>
__device__ __forceinline__ f32x4 load_codes(const C* p, long long n)
{
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n >= 4) {
        const CV c = *(const CV*)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)c[j];
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) v[j] = (float)p[j];
    }
    return v;
}
template <typename V, typename E>
__device__ __forceinline__ void store4(E* p, long long n, const f32x4& x)
{
    V o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = (E)x[j];
    if (n >= 4) {
        *(V*)p = o;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) p[j] = o[j];
    }
}
__device__ __forceinline__ void store4(float* p, long long n, const f32x4& x) { store4<f32x4_any>(p, n, x); }
__device__ __forceinline__ void store4(__bf16* p, long long n, const f32x4& x) { store4<bf16x4_any>(p, n, x); }

__device__ __forceinline__ float decode_m(float code, float scale)
{
    const float t = code * (1.f / 127.f);
    return t * fabsf(t) * scale;
}
__device__ __forceinline__ float decode_v(float code, float scale)
{
    float t = code * (1.f / 255.f);
    t = t * t;
    return t * t * scale;
}

// The largest of 4 magnitudes over the wave; NaN if any is NaN.
__device__ __forceinline__ float wave_top(const f32x4& x)
{
    float top = 0.f, bad = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        top = fmaxf(top, fabsf(x[j]));
        bad = x[j] != x[j] ? 1.f : bad;
    }
    return __any(bad != 0.f) ? __builtin_nanf("") : wave_reduce(top, [](float a, float b) { return fmaxf(a, b); });
}

// Root of a share of the scale in steps, rounded for itself at every operation: what the stored code is the nearest integer of.
template <bool FOURTH>
__device__ __forceinline__ float steps_exact(float x, float top)
{
    const float root = sqrtf(x / top);
    return FOURTH ? sqrtf(root) * 255.f : root * 127.f;
}
// Codes of the 4 magnitudes x under the scale top, as floats.  A division and two or four roots to the last bit for each element would bound the step (540 us
// at 113 M parameters, where its bytes take 350): the hardware's reciprocal and roots are off by under 1e-4 of a step, and decide unless the
// result lies within 3e-4 of half a step, which sends 4 in 100 waves to the exact form.
template <bool FOURTH>
__device__ __forceinline__ f32x4 encode(const f32x4& x, float top)
{
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
    if (top > 0x1p-100f) {  // (the reciprocal of less may overflow)
        const float inverse = __builtin_amdgcn_rcpf(top);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float root = __builtin_amdgcn_sqrtf(x[j] * inverse);
            float s = FOURTH ? __builtin_amdgcn_sqrtf(root) * 255.f : root * 127.f;
            if (fabsf(s - floorf(s) - 0.5f) < 3e-4f) s = steps_exact<FOURTH>(x[j], top);
            c[j] = rintf(s);
        }
    } else if (top > 0.f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = rintf(steps_exact<FOURTH>(x[j], top));
    }
    return c;
}

// Codes of the 4 elements and the scale of their block.
__device__ __forceinline__ f32x4 encode_m(const f32x4& x, float* scale)
{
    const float top = wave_top(x);
    const bool fine = top < INFINITY;
    *scale = fine ? top : __builtin_nanf("");
    f32x4 c = encode<false>(f32x4{fabsf(x[0]), fabsf(x[1]), fabsf(x[2]), fabsf(x[3])}, top);
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = fine ? copysignf(c[j], x[j]) : 0.f;
    return c;
}
__device__ __forceinline__ f32x4 encode_v(const f32x4& x, float* scale)
{
    const float top = wave_top(x);
    const bool fine = top < INFINITY;
    *scale = fine ? top : __builtin_nanf("");
    f32x4 c = encode<true>(x, top);
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = !fine ? 0.f : x[j] > 0.f ? fmaxf(c[j], 1.f) : c[j];
    return c;
}

// A wave's groups: block, block + kWaves, ... of tensor t.  FULL: every one has all of its 256 elements (in the other form each access asks how many there are).
template <typename T, bool EIGHT, bool FULL>
__device__ __forceinline__ void adamw_groups(const Launch::Tensor& t, const AdamHyper& h, long long block, int lane)
{
    const float scale = h.grad_scale ? *h.grad_scale : 1.f;
    f32x4 p[kGroups], g[kGroups], m[kGroups], v[kGroups];
    float ms[kGroups], vs[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const long long at = (block + i * kWaves) * kAdamBlock + 4 * lane, left = FULL ? 4 : t.n - at;
        const bool any = FULL || (block + i * kWaves) * kAdamBlock < t.n;
        p[i] = t.master ? load4(t.master + at, left) : load4((const T*)t.param + at, left);
        g[i] = load4((const T*)t.grad + at, left);
        if (EIGHT) {
            m[i] = load_codes<signed char, i8x4_any>((const signed char*)t.m + at, left);
            v[i] = load_codes<unsigned char, u8x4_any>((const unsigned char*)t.v + at, left);
            ms[i] = any ? t.m_scale[block + i * kWaves] : 0.f;
            vs[i] = any ? t.v_scale[block + i * kWaves] : 0.f;
        } else {
            m[i] = load4((const float*)t.m + at, left);
            v[i] = load4((const float*)t.v + at, left);
        }
    }
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const long long at = (block + i * kWaves) * kAdamBlock + 4 * lane, left = FULL ? 4 : t.n - at;
        if (!FULL && (block + i * kWaves) * kAdamBlock >= t.n) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gr = h.grad_scale ? g[i][j] * scale : g[i][j];
            float mm = EIGHT ? decode_m(m[i][j], ms[i]) : m[i][j], vv = EIGHT ? decode_v(v[i][j], vs[i]) : v[i][j];
            mm = mm * h.beta1 + gr * h.one_minus_beta1;
            vv = vv * h.beta2 + (gr * gr) * h.one_minus_beta2;
            const float denominator = sqrtf(vv) * h.inv_root_correction + h.eps;
            p[i][j] = p[i][j] * h.keep - (mm / denominator) * h.step_size;
            m[i][j] = mm;
            v[i][j] = vv;
        }
        if (EIGHT) {
            if (!FULL) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j >= left) m[i][j] = v[i][j] = 0.f;  // (what lies past the tensor's end has no say in the scale)
            }
            float s;
            const f32x4 mc = encode_m(m[i], &s);
            if (lane == 0) t.m_scale[block + i * kWaves] = s;
            const f32x4 vc = encode_v(v[i], &s);
            if (lane == 0) t.v_scale[block + i * kWaves] = s;
            store4<i8x4_any>((signed char*)t.m + at, left, mc);
            store4<u8x4_any>((unsigned char*)t.v + at, left, vc);
        } else {
            store4((float*)t.m + at, left, m[i]);
            store4((float*)t.v + at, left, v[i]);
        }
        if (t.master) store4(t.master + at, left, p[i]);
        store4((T*)t.param + at, left, p[i]);
    }
}

template <typename T, bool EIGHT>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const Launch l)
{
    int lo = 0, hi = l.n;  // first[lo] <= blockIdx.x < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (l.first[mid] <= blockIdx.x) lo = mid; else hi = mid;
    }
    const Launch::Tensor& t = l.t[lo];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const long long block = (long long)(blockIdx.x - l.first[lo]) * (kWaves * kGroups) + wave;
    if ((block + (kGroups - 1) * kWaves + 1) * kAdamBlock <= t.n)
        adamw_groups<T, EIGHT, true>(t, l.h, block, lane);
    else
        adamw_groups<T, EIGHT, false>(t, l.h, block, lane);
}

__global__ void __launch_bounds__(kThreads) adamw_decode_kernel(const signed char* m, const float* ms, const unsigned char* v, const float* vs, float* m_out,
                                                                float* v_out, long long n)
{
    f32x4 mc[kGroups], vc[kGroups];
    float sm[kGroups], sv[kGroups];
    const long long first = (long long)blockIdx.x * kChunk + 4 * threadIdx.x;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const long long at = first + 4 * kThreads * i, left = n - at;
        mc[i] = load_codes<signed char, i8x4_any>(m + at, left);
        vc[i] = load_codes<unsigned char, u8x4_any>(v + at, left);
        sm[i] = left > 0 ? ms[at / kAdamBlock] : 0.f;
        sv[i] = left > 0 ? vs[at / kAdamBlock] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const long long at = first + 4 * kThreads * i, left = n - at;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            mc[i][j] = decode_m(mc[i][j], sm[i]);
            vc[i][j] = decode_v(vc[i][j], sv[i]);
        }
        if (left > 0) {
            store4(m_out + at, left, mc[i]);
            store4(v_out + at, left, vc[i]);
        }
    }
}

}  // namespace

hipError_t launch_adamw(int n, const clear_block_adamw_tensor* tensors, const AdamHyper& h, int dtype, int state_bits, hipStream_t stream)
{
    // A launch takes as many tensors as its arguments hold, and 2^32 - 1 threads; a tensor has at most half of them.
    constexpr unsigned kMostBlocks = 0xffffffffu / kThreads;
    auto kernel = dtype == CLEAR_BF16 ? (state_bits == 8 ? adamw_kernel<__bf16, true> : adamw_kernel<__bf16, false>)
                                      : (state_bits == 8 ? adamw_kernel<float, true> : adamw_kernel<float, false>);
    Launch l;
    l.h = h;
    l.n = 0;
    unsigned blocks = 0;
    auto flush = [&]() -> hipError_t {
        if (l.n == 0) return hipSuccess;
        l.first[l.n] = blocks;
        kernel<<<dim3(blocks), dim3(kThreads), 0, stream>>>(l);
        l.n = 0;
        blocks = 0;
        return hipGetLastError();
    };
    for (int i = 0; i < n; ++i) {
        if (!tensors[i].grad || tensors[i].n == 0) continue;
        const long long need = (tensors[i].n + kChunk - 1) / kChunk;
        if (l.n == kAdamTensors || blocks + need > kMostBlocks) {
            const hipError_t e = flush();
            if (e != hipSuccess) return e;
        }
        const clear_block_adamw_tensor& t = tensors[i];
        l.t[l.n] = {t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.n};
        l.first[l.n++] = blocks;
        blocks += (unsigned)need;
    }
    return flush();
}

hipError_t launch_adamw_decode(const void* m, const float* ms, const void* v, const float* vs, float* m_out, float* v_out, long long n,
                               hipStream_t stream)
{
    const long long each = kChunk, most = 1LL << 23;  // workgroups of a launch
    for (long long first = 0; first < n; first += most * each) {
        const long long left = std::min(n - first, most * each);
        adamw_decode_kernel<<<dim3((unsigned)((left + each - 1) / each)), dim3(kThreads), 0, stream>>>(
            (const signed char*)m + first, ms + first / kAdamBlock, (const unsigned char*)v + first, vs + first / kAdamBlock, m_out + first, v_out + first, left);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace block
}  // namespace clear
