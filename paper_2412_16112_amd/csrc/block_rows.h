// How a team of waves holds a row of channels, for the kernels that norm rows (block_norm.hip, block_residual.hip).
#pragma once
#include "block_internal.h"

namespace clear {
namespace block {

__host__ __device__ constexpr int padded(int channels) { return (channels + 7) & ~7; }  // channels of a partial sum: whole chunks

// Where chunk i of a lane is, and how its elements lie there.
template <typename T, int TEAM, int CH, bool WHOLE>
struct Layout {
    static constexpr bool FOURS = sizeof(T) == 4;
    static constexpr int GAP = FOURS ? 256 * TEAM : 4;
    static __device__ __forceinline__ int first(int lane, int i) { return (FOURS ? 4 : 8) * lane + 512 * TEAM * i; }
    typedef Piece<GAP> P;
    static __device__ __forceinline__ RowForm form(int channels, int i) { return {WHOLE || i + 1 < CH, TEAM * CH == 1 && channels < 8}; }
};

typedef __attribute__((address_space(3))) float* shared_float;
typedef __attribute__((address_space(3))) f32x4* shared_f32x4;
__device__ __forceinline__ void put_four(float* to, f32x4 x) { *(f32x4_any*)to = x; }
__device__ __forceinline__ void put_four(shared_float to, f32x4 x) { *(shared_f32x4)to = x; }  // (at multiples of 16 bytes)

// Sums over a team.  `slots`: N floats for each wave of the workgroup; every wave of the workgroup calls it.  With one barrier: the next call must be given other
// slots, and the one after that may have these again.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&x)[N], float (*slots)[N], int wave)
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
    if (TEAM == 1) return;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) slots[wave][i] = x[i];
    }
    __syncthreads();
    const int first = wave / TEAM * TEAM;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < TEAM; ++w) x[i] += slots[first + w][i];
    }
}

}  // namespace block
}  // namespace clear
