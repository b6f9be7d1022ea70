// The norm of all gradients of a model with the factor that clips it, and the scaling of all gradients in place.  Memory-bound: every gradient is read once for the norm, and read
// and written once where it is scaled.
//
// 113 M bf16 gradients 40 us (5.6 TB/s) and 4 for the factor; 98 MB of bf16 matrices and fp32 vectors clipped 58 (24 and 34, the second reading from the memory side's cache).  (Ranges of chunks a workgroup with the next
// chunk's loads ahead: the same for the norm, scaling 10 % slower.)
//
// Squares are formed and added in fp64: they can neither overflow nor vanish, sums of 10^8 of them lose nothing, and the vector unit has the rate (a bf16 gradient's conversion and fma beside 2 bytes
// of memory).  The largest magnitude is the largest of the values' bits without their signs, as whole numbers: a NaN is larger than everything.
//
// A workgroup takes chunks of kChunkBytes in turn; it finds a chunk's tensor by bisection in the table of first chunks, which comes with the launch's arguments together with the
// pointers.  Its sum is one partial; the partials are added by one workgroup in a fixed order.
#include <algorithm>

#include "block_internal.h"

namespace clear {
namespace block {
namespace {

constexpr int kThreads = 256, kTensors = 160, kLoads = 4, kChunkBytes = kThreads * 16 * kLoads;
constexpr int kMostBlocks = 1024;  // workgroups of a launch: 4 a CU (113 M bf16 gradients 47 us; 2048 51, 4096 52)

struct Launch {
    void* data[kTensors];
    long long n[kTensors];
    unsigned first[kTensors + 1];  // first chunk of each tensor; chunks altogether
    unsigned char wide[kTensors];  // fp32
    int count;
};
static_assert(sizeof(Launch) + 96 <= 4096, "the arguments of a launch are at most 4 KB");

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(4), aligned(2))) unsigned u32x4_any2;
typedef __attribute__((ext_vector_type(4), aligned(4))) unsigned u32x4_any4;

struct Place {
    int tensor;
    long long at;  // of the chunk's first element
};
__device__ __forceinline__ Place place_of(const Launch& l, unsigned chunk)
{
    int lo = 0, hi = l.count;  // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (l.first[mid] <= chunk) lo = mid; else hi = mid;
    }
    return {lo, (long long)(chunk - l.first[lo]) * (kChunkBytes / (l.wide[lo] ? 4 : 2))};
}

// What is added to a sum of squares, or held against a largest magnitude.
struct Squares {
    typedef double Sum;
    static __device__ __forceinline__ void add(Sum& s, float x) { s = __builtin_fma((double)x, (double)x, s); }
    static __device__ __forceinline__ Sum join(Sum a, Sum b) { return a + b; }
    static __device__ __forceinline__ double value(Sum s) { return s; }
};
struct Largest {
    typedef unsigned Sum;
    static __device__ __forceinline__ void add(Sum& s, float x) { s = max(s, __float_as_uint(x) & 0x7fffffffu); }
    static __device__ __forceinline__ Sum join(Sum a, Sum b) { return max(a, b); }
    static __device__ __forceinline__ double value(Sum s) { return (double)__uint_as_float(s); }
};

__device__ __forceinline__ float low(unsigned pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(unsigned pair) { return __uint_as_float(pair & 0xffff0000u); }

template <typename T>
__device__ __forceinline__ u32x4 load16(const T* p)
{
    if constexpr (sizeof(T) == 4) return *(const u32x4_any4*)p;
    else return *(const u32x4_any2*)p;
}

// The pieces of 16 bytes of a chunk that `left` elements are left for, kLoads a thread, 0 where there are none; FULL: all of them.  What is left behind the last whole piece is
// the threads' own, one element each: its index, or -1.
template <bool FULL, typename T>
__device__ __forceinline__ void load_chunk(u32x4 (&v)[kLoads], const T* p, long long left)
{
    constexpr int EACH = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int at = (i * kThreads + threadIdx.x) * EACH;
        if (!FULL) v[i] = u32x4{};
        if (FULL || at + EACH <= left) v[i] = load16(p + at);
    }
}
template <typename T>
__device__ __forceinline__ int own_element(long long left)
{
    constexpr int EACH = 16 / sizeof(T);
    return (int)threadIdx.x < (int)(left % EACH) ? (int)(left / EACH) * EACH + (int)threadIdx.x : -1;
}

template <typename K, bool FULL, typename T>
__device__ __forceinline__ void add_chunk(typename K::Sum (&s)[4], const T* p, long long left)
{
    u32x4 v[kLoads];
    load_chunk<FULL>(v, p, left);
    const int own = FULL ? -1 : own_element<T>(left);
    const float last = own >= 0 ? (float)p[own] : 0.f;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) {
                K::add(s[j], __uint_as_float(v[i][j]));
            } else {
                K::add(s[j], low(v[i][j]));
                K::add(s[j], high(v[i][j]));
            }
        }
    if (!FULL) K::add(s[0], last);
}
// f(the chunk's first element, elements left from there on, whether the chunk is full) with the tensor's type.
template <typename F>
__device__ __forceinline__ void with_chunk(const Launch& l, unsigned chunk, F&& f)
{
    const Place at = place_of(l, chunk);
    const long long left = l.n[at.tensor] - at.at;
    if (l.wide[at.tensor]) {
        float* const p = (float*)l.data[at.tensor] + at.at;
        if (left >= kChunkBytes / 4) f(p, left, std::true_type{}); else f(p, left, std::false_type{});
    } else {
        __bf16* const p = (__bf16*)l.data[at.tensor] + at.at;
        if (left >= kChunkBytes / 2) f(p, left, std::true_type{}); else f(p, left, std::false_type{});
    }
}

template <typename K>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const Launch l, double* partials)
{
    typename K::Sum s[4] = {};
    const unsigned chunks = l.first[l.count];
    for (unsigned chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        with_chunk(l, chunk, [&](auto* p, long long left, auto full) { add_chunk<K, full>(s, p, left); });
    }
    __shared__ typename K::Sum part[kThreads];
    part[threadIdx.x] = K::join(K::join(s[0], s[1]), K::join(s[2], s[3]));
    for (int half = kThreads / 2; half > 0; half /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < half) part[threadIdx.x] = K::join(part[threadIdx.x], part[threadIdx.x + half]);
    }
    if (threadIdx.x == 0) partials[blockIdx.x] = K::value(part[0]);
}

// The factor from the partials, in every thread of a workgroup; `gives`: this one writes it and the norm down.  The order of the sum is the same wherever it is formed.
__device__ __forceinline__ float factor_of(const double* partials, long long n, const GradFactor& f, bool gives)
{
    __shared__ double part[kThreads];
    const bool squares = f.kind == CLEAR_GRAD_NORM_2;
    auto join = [&](double a, double b) { return squares ? a + b : a > b || a != a ? a : b; };
    double s = 0;
#pragma unroll 4
    for (long long i = threadIdx.x; i < n; i += kThreads) s = join(s, partials[i]);
    part[threadIdx.x] = s;
    for (int half = kThreads / 2; half > 0; half /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < half) part[threadIdx.x] = join(part[threadIdx.x], part[threadIdx.x + half]);
    }
    __syncthreads();
    const double unscale = f.unscale ? (double)*f.unscale : 1.0;
    const double norm = (squares ? sqrt(part[0]) : part[0]) * fabs(unscale);
    const float factor = (float)(unscale * (norm > f.max_norm ? f.max_norm / norm : norm != norm ? norm : 1.0));
    if (gives && threadIdx.x == 0) {
        if (f.norm) *f.norm = (float)norm;
        if (f.factor) *f.factor = factor;
    }
    return factor;
}
__global__ void __launch_bounds__(kThreads) grad_factor_kernel(const double* partials, long long n, GradFactor f) { factor_of(partials, n, f, true); }

__device__ __forceinline__ unsigned pair_of(float lo, float hi)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_bit_cast(unsigned, bf16x2{(__bf16)lo, (__bf16)hi});
}

template <bool FULL, typename T>
__device__ __forceinline__ void scale_chunk(T* p, long long left, float factor)
{
    constexpr int EACH = 16 / sizeof(T);
    u32x4 v[kLoads];
    load_chunk<FULL>(v, p, left);
    const int own = FULL ? -1 : own_element<T>(left);
    if (own >= 0) p[own] = (T)((float)p[own] * factor);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int at = (i * kThreads + threadIdx.x) * EACH;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4)
                v[i][j] = __float_as_uint(__uint_as_float(v[i][j]) * factor);
            else
                v[i][j] = pair_of(low(v[i][j]) * factor, high(v[i][j]) * factor);
        }
        if (FULL || at + EACH <= left) {
            if constexpr (sizeof(T) == 4) *(u32x4_any4*)(p + at) = v[i];
            else *(u32x4_any2*)(p + at) = v[i];
        }
    }
}

// A factor of 1 changes nothing: nothing is read.
__device__ __forceinline__ void scale_all(const Launch& l, float factor)
{
    if (factor == 1.f) return;
    const unsigned chunks = l.first[l.count];
    for (unsigned chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x)
        with_chunk(l, chunk, [&](auto* p, long long left, auto full) { scale_chunk<full>(p, left, factor); });
}
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const Launch l, const float* factor) { scale_all(l, *factor); }
// Clipping: every workgroup forms the factor for itself, which a launch of its own and the wait for it would cost more than: 26 small tensors 6.8 us, norm and scaling apart 12.4.  It reads all partials for that, at most 8 KB
// for each launch of the norm (160 tensors), from the caches: work that grows with the square of the launches.  Tensors of 25 000 fp32, clipped, and norm and scaling apart: 160 11 us and 22, 1000 (7 launches) 89 and 115, 3000
// (19 launches) 374 and 375.
__global__ void __launch_bounds__(kThreads) grad_clip_kernel(const Launch l, const double* partials, long long n, GradFactor f, int gives)
{
    scale_all(l, factor_of(partials, n, f, gives && blockIdx.x == 0));
}

long long chunks_of(const clear_block_grad& t) { return (t.n * (t.dtype == CLEAR_F32 ? 4 : 2) + kChunkBytes - 1) / kChunkBytes; }
bool skipped(const clear_block_grad& t) { return !t.data || t.n == 0; }

// give(launch, its chunks) for as many tensors at a time as the arguments hold (a tensor has at most 2^23 chunks, a launch fewer than 2^31).
template <typename F>
hipError_t each_launch(int n, const clear_block_grad* tensors, F&& give)
{
    Launch l;
    l.count = 0;
    long long chunks = 0;
    auto flush = [&]() -> hipError_t {
        if (l.count == 0) return hipSuccess;
        l.first[l.count] = (unsigned)chunks;
        const hipError_t e = give(l, chunks);
        l.count = 0;
        chunks = 0;
        return e;
    };
    for (int i = 0; i < n; ++i) {
        const clear_block_grad& t = tensors[i];
        if (skipped(t)) continue;
        if (l.count == kTensors) {
            const hipError_t e = flush();
            if (e != hipSuccess) return e;
        }
        l.data[l.count] = t.data;
        l.n[l.count] = t.n;
        l.wide[l.count] = t.dtype == CLEAR_F32;
        l.first[l.count++] = (unsigned)chunks;
        chunks += chunks_of(t);
    }
    return flush();
}
unsigned blocks_of(long long chunks) { return (unsigned)std::min<long long>(chunks, kMostBlocks); }

}  // namespace

long long grad_norm_partials(int n, const clear_block_grad* tensors)
{
    long long partials = 0;
    (void)each_launch(n, tensors, [&](const Launch&, long long chunks) {
        partials += blocks_of(chunks);
        return hipSuccess;
    });
    return partials;
}

static hipError_t launch_partials(int n, const clear_block_grad* tensors, int kind, void* workspace, hipStream_t stream, long long* partials)
{
    *partials = 0;
    return each_launch(n, tensors, [&](const Launch& l, long long chunks) {
        const unsigned blocks = blocks_of(chunks);
        double* const to = (double*)workspace + *partials;
        *partials += blocks;
        if (kind == CLEAR_GRAD_NORM_2)
            grad_norm_kernel<Squares><<<dim3(blocks), dim3(kThreads), 0, stream>>>(l, to);
        else
            grad_norm_kernel<Largest><<<dim3(blocks), dim3(kThreads), 0, stream>>>(l, to);
        return hipGetLastError();
    });
}

hipError_t launch_grad_norm(int n, const clear_block_grad* tensors, const GradFactor& f, void* workspace, hipStream_t stream)
{
    long long partials;
    const hipError_t e = launch_partials(n, tensors, f.kind, workspace, stream, &partials);
    if (e != hipSuccess) return e;
    grad_factor_kernel<<<dim3(1), dim3(kThreads), 0, stream>>>((const double*)workspace, partials, f);
    return hipGetLastError();
}

hipError_t launch_grad_clip(int n, const clear_block_grad* tensors, const GradFactor& f, void* workspace, hipStream_t stream)
{
    long long partials;
    hipError_t e = launch_partials(n, tensors, f.kind, workspace, stream, &partials);
    if (e != hipSuccess) return e;
    if (partials == 0) {  // nothing to clip: the norm is 0
        grad_factor_kernel<<<dim3(1), dim3(kThreads), 0, stream>>>((const double*)workspace, partials, f);
        return hipGetLastError();
    }
    int gives = 1;
    return each_launch(n, tensors, [&](const Launch& l, long long chunks) {
        grad_clip_kernel<<<dim3(blocks_of(chunks)), dim3(kThreads), 0, stream>>>(l, (const double*)workspace, partials, f, gives);
        gives = 0;
        return hipGetLastError();
    });
}

hipError_t launch_grad_scale(int n, const clear_block_grad* tensors, const float* factor, hipStream_t stream)
{
    return each_launch(n, tensors, [&](const Launch& l, long long chunks) {
        grad_scale_kernel<<<dim3(blocks_of(chunks)), dim3(kThreads), 0, stream>>>(l, factor);
        return hipGetLastError();
    });
}

}  // namespace block
}  // namespace clear
