// What the kernels that multiply tiles of matrices share: loads from memory to LDS, where a row's pieces lie there, the order of the tiles.
#pragma once
#include <mutex>

#include "block_internal.h"

namespace clear {
namespace block {

typedef __attribute__((ext_vector_type(4))) int i32x4;

template <int N>
using Int = std::integral_constant<int, N>;
#define INLINED __attribute__((always_inline))

// f(Int<FROM>{}), ..., f(Int<TO - 1>{}), in order.
template <int FROM, int TO, typename F>
__device__ __forceinline__ void each_of(F& f)
{
    if constexpr (FROM < TO) {
        f(Int<FROM>{});
        each_of<FROM + 1, TO>(f);
    }
}

// ---- buffer loads to LDS ------------------------------------------------------------------------------------------------
// A buffer descriptor bounds a load: what lies at or past `bytes` reads as 0 and nothing past it is touched.
__device__ __forceinline__ i32x4 buffer_of(const void* base, long long bytes)
{
    const unsigned long long b = (unsigned long long)base;
    const int size = bytes < 0 ? 0 : (int)(bytes < 0x7fffffffLL ? bytes : 0x7fffffffLL);
    return i32x4{__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32)), __builtin_amdgcn_readfirstlane(size), 0x00020000};
}
constexpr unsigned kOutside = 0x80000000u;  // an offset past every buffer
// 16 bytes a lane from buffer + voff to LDS at lds + OFFSET + 16 * lane (lds: wave-uniform); counted by vmcnt.  The whole offset is in the vector register, which
// the bounds check looks at.  The compiler puts no wait states into asm: the load needs one after the write of M0, written here, and five after a vector
// instruction that wrote its descriptor, which settled() puts behind the making of descriptors once for all of their loads.
template <int OFFSET>
__device__ __forceinline__ void load_to_lds(const i32x4& buffer, unsigned voff, unsigned lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(buffer), "n"(OFFSET) : "memory", "m0", "scc");
}
__device__ __forceinline__ void settled(i32x4& a, i32x4& b) { asm volatile("s_nop 4" : "+s"(a), "+s"(b)); }
// The buffer `bytes` further on, by scalar instructions (no wait states).
__device__ __forceinline__ void move(i32x4& buffer, unsigned bytes)
{
    const unsigned long long b = ((unsigned long long)(unsigned)buffer[1] << 32 | (unsigned)buffer[0]) + bytes;
    buffer[0] = (int)b;
    buffer[1] = (int)(b >> 32);
}

// Where the 16-byte chunks of a row of a tile lie in LDS: chunk c of row r of STEP elements of 2 bytes in slot c ^ turn_of(r).
template <int STEP>
__device__ __forceinline__ int turn_of(int row)
{
    return STEP == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
}
// Workgroups are dealt to the 8 XCDs in turn, each with its own L2: every XCD gets a contiguous range of an order that goes through the tiles in bands of 4
// of B, so that the 32 tiles in flight on it are 4 x 8 and share 12 operand tiles instead of 30 and more.
__device__ __forceinline__ void tile_of(unsigned id, unsigned n, int tiles_a, int tiles_b, int* tile_a, int* tile_b)
{
    constexpr unsigned XCDS = 8, BAND = 4;
    const unsigned x = id % XCDS, each = n / XCDS, more = n % XCDS;
    const unsigned at = x * each + min(x, more) + id / XCDS;
    const unsigned band = at / (BAND * tiles_a), in = at - band * (BAND * tiles_a);
    const unsigned width = min(BAND, (unsigned)tiles_b - band * BAND);
    *tile_a = (int)(in / width);
    *tile_b = (int)(band * BAND + in % width);
}

// A kernel's limit of dynamic LDS is raised once for each device (it belongs to the device's copy of the kernel).
struct LdsLimit {
    static constexpr int kDevices = 64;
    std::once_flag once[kDevices];
    hipError_t result[kDevices] = {};
    hipError_t ensure(const void* kernel, int bytes)
    {
        int device = 0;
        const hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess) return e;
        if (device < 0 || device >= kDevices) return hipErrorInvalidDevice;
        std::call_once(once[device], [&] { result[device] = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
        return result[device];
    }
};

}  // namespace block
}  // namespace clear
