// Operands in 4 bits: rows of numbers to codes of 4 bits with a scale for every 32 channels, back, and the product of two such matrices on the scaled matrix instructions.
//
// A code is a sign, two bits of exponent and one of fraction: 0, 0.5, 1, 1.5, 2, 3, 4, 6.  A block of 32 channels of a row shares a scale, the power of two at which its largest
// magnitude lies in [4, 8): 2^e, e = max(floor(log2 max |x|) - 2, -127), stored as e + 127; a code is the nearest to x / 2^e, halfway the one whose fraction is 0, and over 6 it is 6.  Scales lie in
// groups of 8 blocks (256 channels, a stage of the product's contraction): [groups][rows][8], so that a tile's scales of a stage are one piece of memory.
#include <algorithm>
#include <type_traits>

#include "block_tiles.h"

namespace clear {
namespace block {
namespace {

constexpr int kGroup = 256;  // channels of a group of scales, and of a stage of the contraction
typedef __attribute__((ext_vector_type(4), aligned(2))) int i32x4_any2;
typedef __attribute__((ext_vector_type(4), aligned(4))) int i32x4_any4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

int groups_of(int channels) { return (channels + kGroup - 1) / kGroup; }

// ---- to 4 bits and back ---------------------------------------------------------------------------------------------------
// Memory-bound: 16 717 x 2 432 bf16 17 us there (5.9 TB/s), 19 back (5.3); 65 536 x 4 096 117 and 120 (four or eight rows a lane: 3 to 10 % slower).  A lane has 8 channels (4 lanes a block, half a
// wave a group), kQuantRows rows one after the other; a workgroup the same group of kQuantRows x 8 rows, whose scales are one piece.
constexpr int kQuantRows = 2;

__device__ __forceinline__ unsigned top_of_block(unsigned bits)  // the largest of 4 neighbouring lanes
{
    bits = max(bits, (unsigned)__builtin_amdgcn_update_dpp(0, (int)bits, 0xb1, 0xf, 0xf, true));
    return max(bits, (unsigned)__builtin_amdgcn_update_dpp(0, (int)bits, 0x4e, 0xf, 0xf, true));
}
// Stored exponent of a block by the bits of its largest magnitude (a NaN's or an infinity's make it 255, which stands for NaN).
__device__ __forceinline__ int exponent_of(unsigned top) { return top >= 0x7f800000u ? 255 : max((int)(top >> 23) - 2, 0); }

// 2^-(e - 127) of a stored exponent, exact; what it makes too small for a float is far below half of the least code.
__device__ __forceinline__ float up_of(int e) { return __uint_as_float((unsigned)(254 - min(e, 253)) << 23); }

template <typename T>
__global__ void __launch_bounds__(256) mx_quantize_kernel(const MxArgs a)
{
    const int group = blockIdx.x, half = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long first = (long long)blockIdx.y * (8 * kQuantRows) + half;
    const int c = group * kGroup + 8 * lane;
    const bool in = c < a.channels;  // (channels come in blocks of 32)
    Chunk8<T> v[kQuantRows];
#pragma unroll
    for (int i = 0; i < kQuantRows; ++i) {
        const long long row = first + 8 * i;
        v[i].template load<4>((const T*)a.x + row * a.ld_x + c, in && row < a.rows ? 8 : 0, RowForm{false, false});
    }
#pragma unroll
    for (int i = 0; i < kQuantRows; ++i) {
        const long long row = first + 8 * i;
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i].get(j)) & 0x7fffffffu);
        top = top_of_block(top);
        const int e = exponent_of(top);
        const float up = up_of(e);
        unsigned codes = 0;
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = v[i].get(j) * up;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, s[0], s[1], 1.f, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, s[2], s[3], 1.f, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, s[4], s[5], 1.f, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, s[6], s[7], 1.f, 3);
        if (row < a.rows) {
            if (in) *(unsigned*)((unsigned char*)a.codes_out + row * a.ld_codes + c / 2) = e == 255 ? 0 : codes;
            if ((lane & 3) == 0) ((unsigned char*)a.scales_out)[group * a.ld_scales + row * 8 + (lane >> 2)] = (unsigned char)e;  // (0 behind the last block)
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) mx_dequantize_kernel(const MxArgs a)
{
    const int group = blockIdx.x, half = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long first = (long long)blockIdx.y * (8 * kQuantRows) + half;
    const int c = group * kGroup + 8 * lane;
    if (c >= a.channels) return;
    unsigned codes[kQuantRows];
    int e[kQuantRows];
#pragma unroll
    for (int i = 0; i < kQuantRows; ++i) {
        const long long row = first + 8 * i;
        codes[i] = 0, e[i] = 0;
        if (row < a.rows) {
            codes[i] = *(const unsigned*)((const unsigned char*)a.codes + row * a.ld_codes + c / 2);
            e[i] = ((const unsigned char*)a.scales)[group * a.ld_scales + row * 8 + (lane >> 2)];
        }
    }
#pragma unroll
    for (int i = 0; i < kQuantRows; ++i) {
        const long long row = first + 8 * i;
        if (row >= a.rows) break;
        const float scale = __uint_as_float(e[i] == 0 ? 0x00400000u : e[i] == 255 ? 0x7fc00000u : (unsigned)e[i] << 23);
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // sign, exponent and fraction put where a float has them, 2^126 too small: 0.5 is a subnormal float there, as it is a subnormal code
            const unsigned code = codes[i] >> (4 * j);
            const float size = __uint_as_float((code & 7) << 22) * 0x1p126f;
            o[j] = __uint_as_float(__float_as_uint(size) | (code & 8) << 28) * scale;
        }
        Chunk8<T>::template store<4>((T*)a.y + row * a.ld_y + c, 8, RowForm{true, false}, o);
    }
}

// ---- the product ------------------------------------------------------------------------------------------------------------
// Y = X W^T + bias: A are the rows of W (the contiguous axis of the output), B those of X.  A stage is 256 of the contraction: 128 bytes of codes and 8 of scales a row.  Lane l of an
// instruction (32 x 32 outputs, 64 of the contraction) has row l % 32 and block l / 32 of two; as a sum has no order, instruction s of a stage takes blocks s and 4 + s of its 8, so that a lane's four
// scales are four neighbouring bytes, of which the instruction names the s-th.
//
// The largest tile is 256 x 256 for 8 waves of 64 x 128, one workgroup a CU.  A workgroup goes on to further tiles, the next one's first stage under way during the epilogue, and stores past the caches (16 717 x
// 2 432 x 9 728 246 us with a workgroup a tile, 213 to 235 now by the part's clock).  16 384 x 16 384 x 8 192: 960 us, 4.6 PFLOP/s, the matrix pipe busy 67 % at 1.63 GHz: the part is at
// its power limit, and 4 waves of 128 x 128, which read a third less from LDS, take the same 1.75 us a stage (and 10 us more for a tile's end).  With 2 432 channels, ten stages, 48 % at 1.9 GHz: a tile's end, whose 128 KB
// all CUs store at about the same time, costs 5 us beside 17 of stages.  Tried without gain: all of the next tile's first stages asked for before the epilogue (- 4 %), lines fetched to L2 two stages ahead (- 8 %), loads
// all in one slot or a quarter of them early, wave priorities around the barrier (all within 2 %).

typedef const __attribute__((address_space(3))) i32x4* lds_i32x4_ptr;
typedef const __attribute__((address_space(3))) int* lds_int_ptr;
typedef const __attribute__((address_space(3))) f32x4* lds_f32x4_ptr;

// 4 bytes a lane, as load_to_lds.
template <int OFFSET>
__device__ __forceinline__ void load_word_to_lds(const i32x4& buffer, unsigned voff, unsigned lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(buffer), "n"(OFFSET) : "memory", "m0", "scc");
}
__device__ __forceinline__ void move_far(i32x4& buffer, long long bytes)
{
    const unsigned long long b = ((unsigned long long)(unsigned)buffer[1] << 32 | (unsigned)buffer[0]) + (unsigned long long)bytes;
    buffer[0] = (int)b;
    buffer[1] = (int)(b >> 32);
}

// A tile: WA x WB waves of NA x NB blocks of 32 x 32, RING stages.
template <int WA, int WB, int NA, int NB, int RING>
struct Shape {
    static constexpr int TA = 32 * NA * WA, TB = 32 * NB * WB, WAVES = WA * WB, THREADS = 64 * WAVES;
    static constexpr int A_BYTES = TA * 128, B_BYTES = TB * 128;
    static constexpr int A_LOADS = A_BYTES / 1024 / WAVES, B_LOADS = B_BYTES / 1024 / WAVES;  // instructions a wave, 1 KB each: 8 rows
    static constexpr int CODE_LOADS = A_LOADS + B_LOADS, LOADS = CODE_LOADS + 2;                 // and one each for A's scales and B's, of 32 rows
    static constexpr int SCALE_BYTES = WAVES * 256, STAGE = A_BYTES + B_BYTES + 2 * SCALE_BYTES, RING_BYTES = RING * STAGE;
    static constexpr int LDS = RING_BYTES + WAVES * 256;  // (the bias of each wave's outputs)
    static_assert(NA == 2, "a wave has 64 outputs, one a lane");
    static_assert(TA <= 32 * WAVES && TB <= 32 * WAVES, "one load a wave for each operand's scales");
    static_assert(A_BYTES / 1024 % WAVES == 0 && B_BYTES / 1024 % WAVES == 0, "the waves share the loads of a stage evenly");
    static_assert(RING >= 2 && LDS <= 160 * 1024);
};

struct TileArgs {
    const unsigned char *w, *ws, *x, *xs;
    long long ld_w, ld_ws, ld_x, ld_xs;
    const void* bias;
    void* out;
    long long ld_out, rows_b;  // rows_b: tokens
    int rows_a, depth;         // outputs, channels
    int tiles_a, tiles_b, bias_bf16, out_bf16;
    unsigned tiles;
    float* parts;     // where the contraction is split: fp32 [gridDim.y][rows_b][ld_parts], to be joined; else null
    int ld_parts;
};

// The bias of an output, 0 where it has none.
__device__ __forceinline__ float bias_of(const TileArgs& t, int at)
{
    if (!t.bias || at >= t.rows_a) return 0.f;
    return t.bias_bf16 ? (float)((const __bf16*)t.bias)[at] : ((const float*)t.bias)[at];
}

// Its bits as they lie in memory, 0 where the contraction is split (nothing waits for them here).
typedef const __attribute__((address_space(4))) TileArgs* tile_args_ptr;
__device__ __forceinline__ unsigned bias_bits(tile_args_ptr t, int at)
{
    if (t->parts || !t->bias || at >= t->rows_a) return 0;
    return t->bias_bf16 ? ((const unsigned short*)t->bias)[at] : ((const unsigned*)t->bias)[at];
}

// Both operands in 4 bits (format 4); byte S of a lane's scales is that of its block.
template <int S>
__device__ __forceinline__ f32x16 product(i32x4 a, i32x4 b, f32x16 c, int scale_a, int scale_b)
{
    const i32x8 wide_a = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wide_b = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide_a, wide_b, c, 4, 4, S, scale_a, S, scale_b);
}

// A lane's or wave's number, or the kernel's arguments, as if they were new.  What a tile needs of them once is formed anew for each tile: kept in registers through all tiles, it would cost
// the loop its own.
__device__ __forceinline__ int anew(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}
__device__ __forceinline__ int anew_scalar(int wave)
{
    asm volatile("" : "+s"(wave));
    return wave;
}
__device__ __forceinline__ tile_args_ptr args_anew()
{
    tile_args_ptr p = (tile_args_ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}
// A product's result is wanted here.  (The compiler keeps the scaled products, unlike the plain ones, no nearer to their places than their data does: it moves a whole stage's down past the barrier
// and the branch behind it, with all operands kept in registers until then.)
__device__ __forceinline__ void stay_here(f32x16& x) { asm volatile("" : "+v"(x)); }

template <int WA, int WB, int NA, int NB, int RING>
__global__ void __launch_bounds__(64 * WA * WB, 2) mx_tile_kernel(const TileArgs t)  // (two waves a SIMD, 256 registers: with more the compiler takes the products' results to accumulation registers and back)
{
    typedef Shape<WA, WB, NA, NB, RING> S;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds_bytes[];
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)lds_bytes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wa = wave % WA, wb = wave / WA;
    const int steps_all = (t.depth + kGroup - 1) / kGroup;
    const int it_first = (int)((long long)steps_all * blockIdx.y / gridDim.y), it_end = (int)((long long)steps_all * (blockIdx.y + 1) / gridDim.y);
    const int steps = it_end - it_first;  // of this part of the contraction
    const int plain = min(t.depth / kGroup, it_end) - it_first;  // those of them that the contraction's end does not cut short
    const int rest = min(t.depth - (it_end - 1) * kGroup, kGroup);  // channels of the last step

    // ---- loads of a stage: codes of A, codes of B, scales of both.  A lane's offsets stay as they are from stage to stage and the buffers move on.
    i32x4 buf_a, buf_b, buf_sa, buf_sb;
    unsigned voff[S::CODE_LOADS], lds_to = lds;
    const unsigned voff_s = threadIdx.x * 4;  // (both operands' scales: lane by lane, as they lie)
    int aimed = 0;                            // the step that buffers and offsets are for
    auto row_of = [](int n, int l) INLINED { return n * 8 + l / 8; };
    auto chunk_of = [&](int n, int l) INLINED { return (l % 8) ^ turn_of<64>(row_of(n, l)); };
    auto place_of = [](int i, int w) INLINED { return i < S::A_LOADS ? w * S::A_LOADS + i : w * S::B_LOADS + i - S::A_LOADS; };
    // Of a step that the contraction's end cuts short: the chunks behind it are not loaded.
    auto cut = [&]() INLINED {
        const int l = anew(lane), v = anew_scalar(wave);
#pragma unroll
        for (int i = 0; i < S::CODE_LOADS; ++i)
            if (chunk_of(place_of(i, v), l) * 32 >= rest) voff[i] = kOutside;
    };
    int a_first, rows_b;
    long long b_first;
    const long long ld_ws = t.ld_ws, ld_xs = t.ld_xs;
    auto begin = [&](unsigned id) INLINED {  // buffers and offsets of a tile's first step
        const tile_args_ptr q = args_anew();
        const int l = anew(lane), v = anew_scalar(wave);
        int tile_a, tile_b;
        tile_of(id, q->tiles, q->tiles_a, q->tiles_b, &tile_a, &tile_b);
        a_first = tile_a * S::TA, b_first = (long long)tile_b * S::TB;
        const int rows_a = min(q->rows_a - a_first, S::TA);
        rows_b = (int)min(q->rows_b - b_first, (long long)S::TB);
        const int left = (q->depth - it_first * kGroup) / 2;  // bytes of a row of codes
        const long long ld_w = q->ld_w, ld_x = q->ld_x;
        buf_a = buffer_of(q->w + a_first * ld_w + it_first * (kGroup / 2), (rows_a - 1) * ld_w + left);
        buf_b = buffer_of(q->x + b_first * ld_x + it_first * (kGroup / 2), (rows_b - 1) * ld_x + left);
        buf_sa = buffer_of(q->ws + it_first * ld_ws + a_first * 8LL, rows_a * 8);
        buf_sb = buffer_of(q->xs + it_first * ld_xs + b_first * 8, rows_b * 8);
        settled(buf_a, buf_b);
        settled(buf_sa, buf_sb);
#pragma unroll
        for (int i = 0; i < S::CODE_LOADS; ++i) {
            const int n = place_of(i, v);
            voff[i] = (unsigned)(row_of(n, l) * (int)(i < S::A_LOADS ? ld_w : ld_x) + chunk_of(n, l) * 16);
        }
        lds_to = lds;
        aimed = 0;
        if (plain == 0) cut();
    };
    // (A buffer that moves on along its rows keeps its length, which is still short of the row behind the last: what it lets through behind the last row's part of the step, no lane's
    // offset reaches.)
    auto advance = [&](unsigned stage) INLINED {  // to the next step, whose place in LDS is `stage`; behind the last one nothing is read
        lds_to = lds + stage;
        move(buf_a, kGroup / 2);
        move(buf_b, kGroup / 2);
        move_far(buf_sa, ld_ws);
        move_far(buf_sb, ld_xs);
        if (++aimed >= plain) {
            if (aimed < steps)
                cut();
            else
                buf_a[2] = buf_b[2] = buf_sa[2] = buf_sb[2] = 0;
        }
    };
    auto load = [&](auto i) INLINED {
        if constexpr (i < S::A_LOADS)
            load_to_lds<i * 1024>(buf_a, voff[i], lds_to + wave * (S::A_LOADS * 1024));
        else if constexpr (i < S::CODE_LOADS)
            load_to_lds<S::A_BYTES + (i - S::A_LOADS) * 1024>(buf_b, voff[i], lds_to + wave * (S::B_LOADS * 1024));
        else if constexpr (i == S::CODE_LOADS)
            load_word_to_lds<S::A_BYTES + S::B_BYTES>(buf_sa, voff_s, lds_to + wave * 256);
        else
            load_word_to_lds<S::A_BYTES + S::B_BYTES + S::SCALE_BYTES>(buf_sb, voff_s, lds_to + wave * 256);
    };

    // ---- operand reads: of 32 rows block 4 h + s of a stage, h = lane / 32: one address for each s, the blocks of 32 rows at constant distances
    constexpr int SLOTS = 4;
    auto rows_address = [&](int first, int s) INLINED { return (unsigned)((first + (lane & 31)) * 128 + (((4 * (lane >> 5) + s) ^ turn_of<64>(lane)) << 4)); };
    unsigned a_zero[SLOTS], b_zero[SLOTS], a_at[SLOTS], b_at[SLOTS], sa_at = 0, sb_at = 0;  // in stage 0, and in the present one
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
        a_zero[i] = lds + rows_address(32 * NA * wa, i);
        b_zero[i] = lds + S::A_BYTES + rows_address(32 * NB * wb, i);
    }
    const unsigned s_zero = lds + S::A_BYTES + S::B_BYTES + (lane & 31) * 8 + (lane >> 5) * 4;
    auto enter = [&](unsigned stage) INLINED {
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) a_at[i] = a_zero[i] + stage, b_at[i] = b_zero[i] + stage;
        sa_at = s_zero + stage + 32 * NA * wa * 8;
        sb_at = s_zero + stage + S::SCALE_BYTES + 32 * NB * wb * 8;
    };
    i32x4 a[2][NA], b[2][NB];
    int sa[NA], sb[NB], sa_next[NA], sb_next[NB];
    constexpr int CODES = NA + NB;
    // Read n of slot s: codes in the order of first use (a[0], b[0], the rest of a, the rest of b); then the scales, where s is a stage's first.
    auto read = [&](auto into, auto s, auto n) INLINED {
        if constexpr (n >= CODES + NA) {
            sb_next[n - CODES - NA] = *(lds_int_ptr)(size_t)(sb_at + (n - CODES - NA) * 256);
        } else if constexpr (n >= CODES) {
            sa_next[n - CODES] = *(lds_int_ptr)(size_t)(sa_at + (n - CODES) * 256);
        } else if constexpr (n == 0 || (n >= 2 && n <= NA)) {
            constexpr int i = n == 0 ? 0 : n - 1;
            a[into][i] = *(lds_i32x4_ptr)(size_t)(a_at[s] + i * 4096);
        } else {
            constexpr int j = n == 1 ? 0 : n - NA;
            b[into][j] = *(lds_i32x4_ptr)(size_t)(b_at[s] + j * 4096);
        }
    };
    auto take_scales = [&](unsigned mask) INLINED {
#pragma unroll
        for (int i = 0; i < NA; ++i) sa[i] = sa_next[i] & mask;
#pragma unroll
        for (int j = 0; j < NB; ++j) sb[j] = sb_next[j] & mask;
    };

    f32x16 acc[NA][NB];

    // ---- the loop, as in the gated projection: a stage is 4 slots; in each the operands of the next slot are read beside the products of this one, across the barrier too; loads take half of
    // a stage's last slot and half of the next one's first.
    constexpr int PRODUCTS = NA * NB, READ_IN = PRODUCTS * 3 / 4, EARLY = S::LOADS / 2;
    // Products of slot `of`; beside them the reads of slot s of the stage entered (not where s is SLOTS), and loads first .. last - 1.
    auto slot = [&](auto of, auto s, auto first, auto last) INLINED {
        constexpr int from = of % 2, reads = s == 0 ? 2 * CODES : CODES;
        auto one = [&](auto n) INLINED {
            if constexpr (s < SLOTS && n < READ_IN) {
                auto next = [&](auto r) INLINED { read(Int<1 - from>{}, s, r); };
                each_of<n * reads / READ_IN, (n + 1) * reads / READ_IN>(next);
            }
            __builtin_amdgcn_sched_barrier(0);
            acc[n % NA][n / NA] = product<of>(a[from][n % NA], b[from][n / NA], acc[n % NA][n / NA], sa[n % NA], sb[n / NA]);
            stay_here(acc[n % NA][n / NA]);
            __builtin_amdgcn_sched_barrier(0);
            each_of<first + n * (last - first) / PRODUCTS, first + (n + 1) * (last - first) / PRODUCTS>(load);
            __builtin_amdgcn_sched_barrier(0);
        };
        each_of<0, PRODUCTS>(one);
    };
    // All but `more` of this wave's loads have arrived and its reads are done; after the barrier everybody's.
    auto settle = [](auto more) INLINED {
        constexpr int n = more;
        static_assert(n < 64, "vmcnt is 6 bits");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((n & 15) | 7 << 4 | (n >> 4) << 14);  // lgkmcnt 0, expcnt unconstrained
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto slots = [&](auto loads) INLINED {
        auto one = [&](auto s) INLINED { slot(s, Int<s + 1>{}, Int<EARLY>{}, Int<(s == 0 && loads ? S::LOADS : EARLY)>{}); };
        each_of<0, SLOTS - 1>(one);
    };
    const unsigned tiles = t.tiles;
    unsigned id = blockIdx.x;
    begin(id);
    each_of<0, S::LOADS>(load);
    int stores = 0;  // that this wave has under way since
    while (true) {
#pragma unroll
        for (int i = 1; i < RING; ++i) {
            advance(i * S::STAGE);
            if (i + 1 < RING)
                each_of<0, S::LOADS>(load);
            else
                each_of<0, EARLY>(load);
        }
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        // (the stores of the tile before lie between the first stage's loads and those of the others: they need not have arrived)
        constexpr int BEHIND = (RING - 2) * S::LOADS + EARLY;
        constexpr int NARROW = 4 * NB, WIDE = 8 * NB;  // of a whole tile's outputs in bf16, in fp32
        if (stores == WIDE)
            settle(Int<BEHIND + WIDE>{});
        else if (stores == NARROW)
            settle(Int<BEHIND + NARROW>{});
        else
            settle(Int<BEHIND>{});
        const unsigned bias_raw = bias_bits(args_anew(), a_first + 32 * NA * wa + lane);  // (asked for here, where it delays nothing)
        enter(0);
        auto next = [&](auto r) INLINED { read(Int<0>{}, Int<0>{}, r); };
        each_of<0, 2 * CODES>(next);
        unsigned stage = 0;
        for (int it = 0; it + 1 < steps; ++it) {
            const unsigned next_stage = stage + S::STAGE == S::RING_BYTES ? 0 : stage + S::STAGE;
            take_scales(~0u);
            slots(std::true_type{});
            settle(Int<(RING - 2) * S::LOADS>{});
            advance(stage);
            enter(next_stage);
            __builtin_amdgcn_sched_barrier(0);
            slot(Int<SLOTS - 1>{}, Int<0>{}, Int<0>{}, Int<EARLY>{});
            stage = next_stage;
        }
        // (what lies behind a row's last scale is whatever it is: there the codes are 0, and so are the scales made)
        const int blocks = min(max(rest / 32 - 4 * (lane >> 5), 0), 4);
        take_scales(blocks == 4 ? ~0u : (1u << 8 * blocks) - 1);
        slots(std::false_type{});
        slot(Int<SLOTS - 1>{}, Int<SLOTS>{}, Int<0>{}, Int<0>{});
        settle(Int<0>{});  // (nothing may still be on its way to this workgroup's LDS, which is used again)

        *(__attribute__((address_space(3))) float*)(size_t)(lds + S::RING_BYTES + wave * 256 + 4 * lane) = __uint_as_float(args_anew()->bias_bf16 ? bias_raw << 16 : bias_raw);
        // the next tile's first stage is loaded beside the epilogue, which has the rest of LDS
        const int out_a = a_first, out_rows = rows_b;
        const long long out_b = b_first;
        id += gridDim.x;
        const bool more = id < tiles;
        if (more) {
            begin(id);
            each_of<0, S::LOADS>(load);
        }
        // epilogue: register r of acc[i][j] is A row 8 (r / 4) + 4 (lane / 32) + r % 4 and B row lane % 32 of the two blocks.  Outputs go through a part of LDS of the wave's own, so that
        // neighbouring lanes store neighbouring 16 bytes of a row.
        constexpr int OWN = (S::RING_BYTES - S::STAGE) / S::WAVES / 16 * 16;
        const tile_args_ptr q = args_anew();
        const int l = anew(lane), v = anew_scalar(wave), va = v % WA, vb = v / WA, out_width = q->rows_a;
        const unsigned own = lds + S::STAGE + v * OWN, bias = lds + S::RING_BYTES + v * 256;
        const int first = out_a + 32 * NA * va;
        // BIASED: the bias is added.  WHOLE: the tile has all of its outputs, which needs no looking at each (half of the epilogue's instructions).
        auto store = [&](auto type, auto whole, auto biased, decltype(type)* to, long long ld) INLINED {
            typedef decltype(type) T;
            typedef T four __attribute__((ext_vector_type(4)));
            constexpr int PER = 16 / (int)sizeof(T), BYTES = 32 * NA * (int)sizeof(T), PITCH = BYTES + 16, LANES = BYTES / 16, ROWS = 64 / LANES;
            constexpr int FIT = OWN / (32 * PITCH), TOGETHER = FIT >= NB ? NB : FIT >= 2 && NB % 2 == 0 ? 2 : 1;
            static_assert(FIT >= 1, "a block fits");
            const int c = first + l % LANES * PER, in = 32 * NB * vb + l / LANES;  // this lane's outputs in its first row, and that in the tile
            T* o = to + (out_b + in) * ld + c;
            auto some = [&](auto k) INLINED {
                constexpr int j0 = k * TOGETHER;
                auto put_block = [&](auto n) INLINED {
                    auto put = [&](auto g) INLINED {
                        f32x4 x;
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[r] = acc[g / 4][j0 + n][4 * (g % 4) + r];
                        if constexpr (biased) x += *(lds_f32x4_ptr)(size_t)(bias + (8 * g + 4 * (l >> 5)) * 4);
                        *(__attribute__((address_space(3))) four*)(size_t)(own + (unsigned)((32 * n + (l & 31)) * PITCH + (8 * g + 4 * (l >> 5)) * (int)sizeof(T))) =
                            __builtin_convertvector(x, four);
                    };
                    each_of<0, 4 * NA>(put);
                };
                each_of<0, TOGETHER>(put_block);
                asm volatile("" ::: "memory");  // (a wave's LDS instructions are executed in order)
#pragma unroll
                for (int i = 0; i < TOGETHER * 32 / ROWS; ++i, o += ROWS * ld) {
                    const i32x4 x = *(lds_i32x4_ptr)(size_t)(own + (unsigned)((i * ROWS + l / LANES) * PITCH + l % LANES * 16));
                    auto put = [&] {  // (rows of any length: at any address that its elements allow)
                        if constexpr (sizeof(T) == 2) __builtin_nontemporal_store(x, (i32x4_any2*)o);
                        else __builtin_nontemporal_store(x, (i32x4_any4*)o);
                    };
                    if constexpr (whole) {
                        put();
                    } else if (in + 32 * j0 + i * ROWS < out_rows && c < out_width) {
                        if (c + PER <= out_width) {
                            put();
                        } else {
                            typedef T piece __attribute__((ext_vector_type(PER)));
                            const piece v = __builtin_bit_cast(piece, x);
#pragma unroll
                            for (int e = 0; e < PER - 1; ++e)
                                if (c + e < out_width) o[e] = v[e];
                        }
                    }
                }
                asm volatile("" ::: "memory");
            };
            each_of<0, NB / TOGETHER>(some);
        };
        const bool wide = q->parts || !q->out_bf16, whole = out_a + S::TA <= out_width && out_rows == S::TB, biased = q->bias && !q->parts;
        stores = !whole ? 0 : wide ? WIDE : NARROW;
        auto store_as = [&](auto type, decltype(type)* to, long long ld) INLINED {
            if (!whole) store(type, std::false_type{}, std::true_type{}, to, ld);
            else if (biased) store(type, std::true_type{}, std::true_type{}, to, ld);
            else store(type, std::true_type{}, std::false_type{}, to, ld);
        };
        if (wide)
            store_as(0.f, q->parts ? q->parts + blockIdx.y * q->rows_b * q->ld_parts : (float*)q->out, q->parts ? q->ld_parts : q->ld_out);
        else
            store_as((__bf16)0.f, (__bf16*)q->out, q->ld_out);
        if (!more) break;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 3 << 14);  // lgkmcnt 0: the epilogue's part of LDS is read
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
}

// The sum of the parts of a split contraction, in order, and the bias to the output; 4 outputs a thread.
__global__ void __launch_bounds__(256) mx_join_kernel(const TileArgs t, int parts, long long n)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= n) return;
    const int each = t.ld_parts / 4;
    const long long row = id / each, plane = t.rows_b * t.ld_parts;
    const int c = (int)(id - row * each) * 4;
    const float* const from = t.parts + row * t.ld_parts + c;
    f32x4 s = *(const f32x4*)from;
#pragma unroll 4
    for (int p = 1; p < parts; ++p) s += *(const f32x4*)(from + p * plane);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c + e >= t.rows_a) break;
        const float y = s[e] + bias_of(t, c + e);
        if (t.out_bf16) ((__bf16*)t.out)[row * t.ld_out + c + e] = (__bf16)y;
        else ((float*)t.out)[row * t.ld_out + c + e] = y;
    }
}

// ---- few tokens -----------------------------------------------------------------------------------------------------------
// Up to 16 MT tokens: bound by the one reading of the weights.  A workgroup takes 16 outputs and all of the contraction, its 8 or 16 waves every 8th or 16th group of it: weights go straight from memory
// to the operand registers.  Lane l of an instruction (16 x 16 outputs, 128 of the contraction) has row l % 16 and block l / 16 of four; instruction s of two takes blocks s, 2 + s, 4 + s and 6 + s of a
// group, so that a lane's codes of a group are 32 neighbouring bytes and its scales two.  The waves' sums are added in order in LDS.
// One token at 4 096 x 11 264: 7.7 us a launch in a graph (3.2 TB/s, of which some 3 us are a launch's start and end); three or four groups ahead in place of two 10.
template <int S>
__device__ __forceinline__ f32x4 few_product(i32x4 a, i32x4 b, f32x4 c, int scale_a, int scale_b)
{
    const i32x8 wide_a = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wide_b = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide_a, wide_b, c, 4, 4, S, scale_a, S, scale_b);
}
// Tokens that come as numbers and are at most kDirect go to 4 bits here: a wave takes the channels of its groups, 4 a lane, and its operands go through LDS.  (A launch of its own for that takes 3 us and
// as many of the host's: one token at 4 096 x 11 264 10 us from Python, 15 with it.)
constexpr int kDirect = 4;
template <int N>
struct alignas(16) DirectGroup {
    unsigned short codes[N][64];  // (a lane's 4 codes; read 16 bytes at a time, which alignment each of a wave's groups has: 144 bytes of one token, 544 of four)
    unsigned char scales[N][8];
};
static_assert(sizeof(DirectGroup<1>) % 16 == 0 && sizeof(DirectGroup<kDirect>) % 16 == 0);
template <typename T>
struct FourOf;
template <>
struct FourOf<__bf16> {
    typedef bf16x4_any type;
};
template <>
struct FourOf<float> {
    typedef f32x4_any type;
};
template <typename T, int N>
__device__ __forceinline__ void load_direct(f32x4 (&v)[N], const T* x, long long ld_x, int tokens, int c, int channels)
{
#pragma unroll
    for (int m = 0; m < N; ++m)
        v[m] = m < tokens && c < channels ? __builtin_convertvector(*(const typename FourOf<T>::type*)(x + m * ld_x + c), f32x4) : f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int N>
__device__ __forceinline__ void direct_group(DirectGroup<N>* to, const f32x4 (&v)[N], int tokens, int lane)
{
#pragma unroll
    for (int m = 0; m < N; ++m) {
        if (m >= tokens) break;
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(v[m][j]) & 0x7fffffffu);
        top = top_of_block(top);
        top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xf, 0xf, true));  // (the other four lanes of the block's eight)
        const int e = exponent_of(top);
        const f32x4 s = v[m] * up_of(e);
        unsigned codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, s[0], s[1], 1.f, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, s[2], s[3], 1.f, 1);
        to->codes[m][lane] = e == 255 ? 0 : (unsigned short)codes;
        if ((lane & 7) == 0) to->scales[m][lane >> 3] = (unsigned char)e;
    }
}

// T: of the tokens, of which there are N at most, or void where they come in 4 bits.
template <int MT, typename T, int N, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) mx_few_kernel(const TileArgs t)
{
    constexpr bool DIRECT = !std::is_void<T>::value;
    static_assert(!DIRECT || MT == 1);
    constexpr int AHEAD = 2;  // groups whose loads are in flight together
    __shared__ f32x4 part[WAVES][MT][64];
    __shared__ DirectGroup<N> direct[DIRECT ? WAVES : 1][DIRECT ? AHEAD : 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, block = 2 * (lane >> 4);
    const int f0 = blockIdx.x * 16;
    const int f = min(f0 + (lane & 15), t.rows_a - 1);
    const unsigned char* const w = t.w + f * t.ld_w + block * 16;
    const unsigned char* const ws = t.ws + f * 8LL + block;
    const unsigned char *x[MT], *xs[MT];
    if (!DIRECT) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const long long token = min((long long)(16 * m + (lane & 15)), t.rows_b - 1);
            x[m] = t.x + token * t.ld_x + block * 16;
            xs[m] = t.xs + token * 8 + block;
        }
    }
    // this thread's four outputs of the end, whose bias is asked for here, where it delays nothing (of several tokens that are numbers, behind the sums: registers)
    const int c = f0 + 4 * (lane >> 4);
    f32x4 bias = {0.f, 0.f, 0.f, 0.f};
    auto load_bias = [&] {
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = bias_of(t, c + e);
    };
    if (N == 1 && wave < MT) load_bias();
    f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int groups = (t.depth + kGroup - 1) / kGroup;
    for (int g0 = wave; g0 < groups; g0 += WAVES * AHEAD) {
        // (One token is read first: it comes from near and goes to 4 bits while the weights are on their way: 4 096 x 11 264 8.9 -> 7.7 us.  Of several, the registers for that would cost more: 11.3 -> 14.0.)
        f32x4 v[DIRECT ? AHEAD : 1][N];
        auto load_tokens = [&](int i) {
            if constexpr (DIRECT) load_direct<T>(v[i], (const T*)t.x, t.ld_x, (int)t.rows_b, (g0 + WAVES * i) * kGroup + 4 * lane, t.depth);
        };
        if constexpr (DIRECT && N == 1) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) load_tokens(i);
            __builtin_amdgcn_sched_barrier(0);
        }
        i32x4 a[AHEAD][2], b[AHEAD][MT][2];
        int sa[AHEAD], sb[AHEAD][MT];
        const i32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int g = g0 + WAVES * i, left = t.depth - g * kGroup - block * 32;  // channels from this lane's first block on
            const int mask = left >= 64 ? 0xffff : left > 0 ? 0xff : 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                a[i][k] = left > 32 * k ? *(const i32x4*)(w + (long long)g * (kGroup / 2) + 16 * k) : zero;
                if (!DIRECT) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) b[i][m][k] = left > 32 * k ? *(const i32x4*)(x[m] + (long long)g * (kGroup / 2) + 16 * k) : zero;
                }
            }
            sa[i] = left > 0 ? *(const unsigned short*)(ws + g * t.ld_ws) & mask : 0;
            if (!DIRECT) {
#pragma unroll
                for (int m = 0; m < MT; ++m) sb[i][m] = left > 0 ? *(const unsigned short*)(xs[m] + g * t.ld_xs) & mask : 0;
            }
        }
        if constexpr (DIRECT) {
            if constexpr (N == 1) __builtin_amdgcn_sched_barrier(0);
            const int token = lane & 15;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if constexpr (N > 1) load_tokens(i);
                direct_group(&direct[wave][i], v[i], (int)t.rows_b, lane);
            }
            asm volatile("" ::: "memory");  // (a wave's LDS instructions are executed in order)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const DirectGroup<N>& d = direct[wave][i];
                const bool in = token < (int)t.rows_b;
#pragma unroll
                for (int k = 0; k < 2; ++k) b[i][0][k] = in ? *(const i32x4*)((const unsigned char*)d.codes[token & (N - 1)] + 16 * (block + k)) : zero;
                sb[i][0] = in ? *(const unsigned short*)(d.scales[token & (N - 1)] + block) : 0;
            }
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                acc[m] = few_product<0>(a[i][0], b[i][m][0], acc[m], sa[i], sb[i][m]);
                acc[m] = few_product<1>(a[i][1], b[i][m][1], acc[m], sa[i], sb[i][m]);
            }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) part[wave][m][lane] = acc[m];
    __syncthreads();
    // register r of lane l: output 4 (l / 16) + r, token l % 16
    if (wave >= MT) return;
    f32x4 s = part[0][wave][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) s += part[v][wave][lane];
    if (N > 1) load_bias();
    s += bias;
    const long long token = 16 * wave + (lane & 15);
    if (token >= t.rows_b) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c + e >= t.rows_a) break;
        if (t.out_bf16) ((__bf16*)t.out)[token * t.ld_out + c + e] = (__bf16)s[e];
        else ((float*)t.out)[token * t.ld_out + c + e] = s[e];
    }
}

template <int MT, typename T, int N>
hipError_t launch_few(const TileArgs& t, hipStream_t stream)
{
    // Where a CU has one workgroup and 8 waves more than a turn's work, 16: 11 264 x 4 096 11.4 -> 8.2 us; at 4 096 x 11 264 7.7 -> 10.5, at 2 048 x 2 048 and 16 tokens 3.8 -> 4.0.
    const dim3 grid((t.rows_a + 15) / 16);
    if (grid.x <= 256 && groups_of(t.depth) > 8 * MT) mx_few_kernel<MT, T, N, 16><<<grid, dim3(64 * 16), 0, stream>>>(t);
    else mx_few_kernel<MT, T, N, 8><<<grid, dim3(64 * 8), 0, stream>>>(t);
    return hipGetLastError();
}

template <int WA, int WB, int NA, int NB, int RING>
hipError_t launch_tiles(TileArgs t, int parts, hipStream_t stream)
{
    typedef Shape<WA, WB, NA, NB, RING> S;
    t.tiles_a = (t.rows_a + S::TA - 1) / S::TA;
    const long long tiles_b = (t.rows_b + S::TB - 1) / S::TB;
    if (tiles_b > 0x7fffffffLL || tiles_b * t.tiles_a > 0xffff0000LL) return hipErrorInvalidValue;  // (outputs that no memory holds)
    t.tiles_b = (int)tiles_b;
    if (parts == 1) t.parts = nullptr;
    static LdsLimit limit;
    const hipError_t allowed = limit.ensure((const void*)mx_tile_kernel<WA, WB, NA, NB, RING>, S::LDS);
    if (allowed != hipSuccess) return allowed;
    t.tiles = (unsigned)(tiles_b * t.tiles_a);
    const unsigned resident = 256 * (S::LDS <= 80 * 1024 ? 2 : 1);  // workgroups that the CUs hold: a multiple of 8, so that a workgroup's tiles are its XCD's
    mx_tile_kernel<WA, WB, NA, NB, RING><<<dim3(std::min(t.tiles, resident), parts), dim3(S::THREADS), S::LDS, stream>>>(t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    const long long n = t.rows_b * (t.ld_parts / 4), blocks = (n + 255) / 256;
    if (blocks > 0xffffffffLL / 256) return hipErrorInvalidValue;
    mx_join_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(t, parts, n);
    return hipGetLastError();
}

// Form, tile shape and number of parts that the contraction is split into, by the time that they are expected to take with weights from memory: where no CU has two tiles, a part's steps (256 of the
// contraction) and what a tile costs beside; else rounds of as many tiles as the chip holds at once.  The constants, in us, were fitted to 3000 timings at 8 to 3000 tokens and eleven shapes of 608 x 3000 to
// 4096 x 11264: the chosen form takes 0.5 % longer than the best of them on average, at most 11 %.  (77 tokens at 4096 x 11264: 64 x 64 12.5 us, 64 x 128 12.1, 128 x 128 14.3; at 4096 x 4096 8.2, 9.2 and 11.9; 333 at
// 2432 x 7297 13.8, 12.6 and 11.7; 1000 at 2432 x 9728 39.9, 29.6 and 31.0, 256 x 256 25.6.)  One shape for the whole product: a last round of few tiles takes as long as a full one (tokens in 4 bits at 2432 x 9728: 1500
// 25.7 us, 2000 37.3, 3000 48.8, 4608 71.4; at 4096 x 11264 1000 28.4, 1500, which are 264 tiles, 55.2, 2000 57.6).
enum TileShape { kLarge, kPair, kDeep, kSmall, kFlat, kFew };  // kPair: two workgroups a CU, kDeep: one with four stages in flight
struct Cost {
    int outputs, tokens;                 // of a tile
    int at_once;                         // tiles that the chip holds
    double step_alone, tile_alone;       // where it holds more than a tile a CU and has not to
    double step, round, start;
} constexpr kCosts[] = {
    {256, 256, 256, 0, 0, 1.34, 7.4, -1.3}, {128, 128, 512, 0.88, 3.6, 1.03, 1.6, 3.6}, {128, 128, 256, 0, 0, 0.52, 3.0, 1.7}, {64, 64, 512, 0.25, 3.3, 0.41, 1.3, 4.5}, {64, 128, 512, 0.44, 4.0, 0.65, 1.3, 3.6},
};
struct Plan {
    TileShape shape;
    int parts;
};
Plan plan_of(long long tokens, int channels, int outputs)
{
    const auto up = [](long long x, long long by) { return (x + by - 1) / by; };
    // (few tokens, here and in tiles: 8 at 2432 x 9728 6.5 and 7.3, at 4096 x 11264 8.5 and 9.2; 32 at 4096 x 4096 6.6 and 8.2, at 2432 x 7297 6.4 and 7.4, at 2432 x 9728 12.8 and 7.5)
    if (tokens <= 16 || (tokens <= 32 && (long long)channels * outputs <= 20 << 20)) return {kFew, 1};
    const long long steps = groups_of(channels);
    Plan best = {kLarge, 1};
    double best_us = 0;
    for (int parts = 1; parts <= 8 && (parts == 1 || steps >= 3 * parts); ++parts) {
        const double each = (double)up(steps, parts);
        // (the parts are written and read once more)
        const double join = parts == 1 ? 0 : 3.7 + (1.35 * parts - 0.1) * tokens * outputs * 4 / 4e6;
        for (int i = kLarge; i <= kFlat; ++i) {
            const Cost& c = kCosts[i];
            const long long tiles = up(outputs, c.outputs) * up(tokens, c.tokens) * parts;
            const double us = join + (tiles <= 256 && c.at_once > 256 ? each * c.step_alone + c.tile_alone : up(tiles, c.at_once) * (each * c.step + c.round) + c.start);
            if (best_us == 0 || us < best_us) best_us = us, best = {(TileShape)i, parts};
        }
    }
    return best;
}

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t codes_bytes(long long tokens, int channels) { return rounded((size_t)tokens * channels / 2); }
size_t scales_bytes(long long tokens, int channels) { return rounded((size_t)groups_of(channels) * tokens * 8); }
int parts_pitch(int outputs) { return (outputs + 3) / 4 * 4; }

}  // namespace

hipError_t launch_mx_quantize(const MxArgs& a, int dtype, hipStream_t stream)
{
    // (a launch has at most 65535 workgroups along its grid's second axis, of 8 kQuantRows rows each)
    constexpr long long each = 8 * kQuantRows, most = 65535 * each;
    for (long long first = 0; first < a.rows; first += most) {
        MxArgs b = a;
        b.rows = std::min(a.rows - first, most);
        b.x = (const char*)a.x + first * a.ld_x * (dtype == CLEAR_BF16 ? 2 : 4);
        b.codes_out = (char*)a.codes_out + first * a.ld_codes;
        b.scales_out = (char*)a.scales_out + first * 8;
        const dim3 grid(groups_of(a.channels), (unsigned)((b.rows + each - 1) / each));
        if (dtype == CLEAR_BF16) mx_quantize_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(b);
        else mx_quantize_kernel<float><<<grid, dim3(256), 0, stream>>>(b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_mx_dequantize(const MxArgs& a, int dtype, hipStream_t stream)
{
    constexpr long long each = 8 * kQuantRows, most = 65535 * each;
    for (long long first = 0; first < a.rows; first += most) {
        MxArgs b = a;
        b.rows = std::min(a.rows - first, most);
        b.codes = (const char*)a.codes + first * a.ld_codes;
        b.scales = (const char*)a.scales + first * 8;
        b.y = (char*)a.y + first * a.ld_y * (dtype == CLEAR_BF16 ? 2 : 4);
        const dim3 grid(groups_of(a.channels), (unsigned)((b.rows + each - 1) / each));
        if (dtype == CLEAR_BF16) mx_dequantize_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(b);
        else mx_dequantize_kernel<float><<<grid, dim3(256), 0, stream>>>(b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// The tokens in 4 bits, unless they come so, then the parts of a split contraction.
size_t mx_linear_workspace_bytes(long long tokens, int channels, int outputs, bool quantized)
{
    if (tokens == 0 || (!quantized && tokens <= kDirect)) return 0;
    const int parts = plan_of(tokens, channels, outputs).parts;
    return (quantized ? 0 : codes_bytes(tokens, channels) + scales_bytes(tokens, channels)) + (parts > 1 ? (size_t)parts * tokens * parts_pitch(outputs) * 4 : 0);
}

hipError_t launch_mx_linear(const MxLinearArgs& a, hipStream_t stream)
{
    TileArgs t = {};
    t.w = (const unsigned char*)a.w, t.ws = (const unsigned char*)a.ws, t.x = (const unsigned char*)a.x, t.xs = (const unsigned char*)a.xs;
    t.ld_w = a.ld_w, t.ld_ws = a.ld_ws, t.ld_x = a.ld_x, t.ld_xs = a.ld_xs;
    t.bias = a.bias, t.bias_bf16 = a.bias_dtype == CLEAR_BF16;
    t.out = a.y, t.ld_out = a.ld_y, t.out_bf16 = a.out_dtype == CLEAR_BF16;
    t.rows_a = a.outputs, t.rows_b = a.tokens, t.depth = a.channels;
    if (!a.xs && a.tokens <= kDirect) {
        const bool half = a.x_dtype == CLEAR_BF16;
        if (a.tokens == 1) return half ? launch_few<1, __bf16, 1>(t, stream) : launch_few<1, float, 1>(t, stream);
        return half ? launch_few<1, __bf16, kDirect>(t, stream) : launch_few<1, float, kDirect>(t, stream);
    }
    unsigned char* ws = (unsigned char*)a.workspace;
    if (!a.xs) {
        MxArgs q = {};
        q.x = a.x, q.ld_x = a.ld_x;
        q.codes_out = ws, q.ld_codes = a.channels / 2;
        q.scales_out = ws + codes_bytes(a.tokens, a.channels), q.ld_scales = a.tokens * 8;
        q.rows = a.tokens, q.channels = a.channels;
        const hipError_t e = launch_mx_quantize(q, a.x_dtype, stream);
        if (e != hipSuccess) return e;
        t.x = ws, t.ld_x = q.ld_codes, t.xs = (const unsigned char*)q.scales_out, t.ld_xs = q.ld_scales;
        ws += codes_bytes(a.tokens, a.channels) + scales_bytes(a.tokens, a.channels);
    }
    const Plan p = plan_of(a.tokens, a.channels, a.outputs);
    t.parts = (float*)ws, t.ld_parts = parts_pitch(a.outputs);
    switch (p.shape) {
    case kFew: return a.tokens <= 16 ? launch_few<1, void, 1>(t, stream) : launch_few<2, void, 1>(t, stream);
    case kLarge: return launch_tiles<4, 2, 2, 4, 2>(t, p.parts, stream);
    case kPair: return launch_tiles<2, 2, 2, 2, 2>(t, p.parts, stream);
    case kDeep: return launch_tiles<2, 2, 2, 2, 4>(t, p.parts, stream);
    case kSmall: return launch_tiles<1, 2, 2, 1, 4>(t, p.parts, stream);
    default: return launch_tiles<1, 4, 2, 1, 3>(t, p.parts, stream);
    }
}

}  // namespace block
}  // namespace clear
