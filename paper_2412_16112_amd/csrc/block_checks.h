// Argument checks that the C entry points of the operators around the attention share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/clear_block.h"

namespace clear {
namespace block {

// Notes the reason of a failure for clear_block_last_error and returns the code.  Nothing leaves a C entry point as an exception: a message that cannot be stored is dropped.
int fail(int code, const char* what, const char* why = "") noexcept;
inline int invalid(const char* what) noexcept { return fail(CLEAR_ERR_INVALID_ARG, what); }
inline int unsupported(const char* what) noexcept { return fail(CLEAR_ERR_UNSUPPORTED, what); }
inline int launched(hipError_t e, const char* what) noexcept { return e == hipSuccess ? CLEAR_OK : fail(CLEAR_ERR_HIP, what, hipGetErrorString(e)); }

inline bool known_dtype(int dtype) { return dtype == CLEAR_BF16 || dtype == CLEAR_F32; }
inline int size_of(int dtype) { return dtype == CLEAR_BF16 ? 2 : 4; }
inline bool aligned(const void* p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }

// Byte range [first, last) that a strided tensor spans.
struct Span {
    __int128 first, last;
};
inline Span span_of(const void* p, const long long* extent, const long long* stride, int axes, long long row, int size)
{
    __int128 last = row;
    for (int i = 0; i < axes; ++i) last += (__int128)(extent[i] - 1) * stride[i];
    return {(__int128)(uintptr_t)p, (__int128)(uintptr_t)p + last * size};
}
inline bool overlap(const Span& a, const Span& b) { return a.first < b.last && b.first < a.last; }
inline bool too_long(const Span& a) { return a.last > ((__int128)1 << 62); }

// An output may be `in` itself; else their ranges must be apart.  A row of an output is its own.
inline bool out_apart(const void* out, const long long* out_strides, const void* in, const long long* in_strides, const long long* extent, int channels, int size, bool may_be_same)
{
    if (may_be_same && out == in && out_strides[0] == in_strides[0] && out_strides[1] == in_strides[1]) return true;
    return !overlap(span_of(out, extent, out_strides, 2, channels, size), span_of(in, extent, in_strides, 2, channels, size));
}
inline bool rows_apart(const long long* strides, const long long* extent, int channels)
{
    if (extent[1] > 1 && strides[1] < channels) return false;
    if (extent[0] <= 1) return true;
    // groups one after the other, or interleaved with the rows (a transposed view)
    const __int128 rows = (__int128)(extent[1] - 1) * strides[1] + channels;
    return strides[0] >= rows || (strides[0] >= channels && (extent[1] == 1 || strides[1] >= (__int128)(extent[0] - 1) * strides[0] + channels));
}

}  // namespace block
}  // namespace clear
