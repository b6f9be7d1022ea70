// The gated feed-forward projection H = act(X Wg^T) * (X Wu^T) and its gradients, on bf16 matrix instructions.
//
// Three products share one tile kernel: the fused forward product (both weights' tiles side by side, so that a lane ends up with
// gate and up of the same outputs and the activation is an epilogue on registers), dX = dG Wg + dU Wu (the contraction runs through both
// halves) and dWg = dG^T X, dWu = dU^T X.  Operand A is the one whose rows become the contiguous axis of the output, B gives its rows.
// An operand is stored along the contraction ("rows": X and the weights forward, dG and dU for dX) or across it ("columns": the weights
// for dX, everything for the weight gradients); the latter are read from LDS with the 16-bit transpose load.
//
// The largest tile is 256 x 256 for 8 waves of 64 x 128 (6 operand reads for 8 matrix instructions): at 16 717 x 2 432 x 9 728 forward 1.27 to 1.35 ms, 1.17 to 1.25 PFLOP/s, matrix pipe
// busy 60 % at 1.9 GHz - at the part's power limit, where a deeper pipeline (stages of 32, four in flight) saved 4 % of the cycles and no time.  Four waves of 128 x 128 read a third less
// from LDS, but a CU then has one wave a SIMD and the epilogue nothing beside it (+ 25 % time).  4 608 x 2 432 x 6 528: forward with the products kept 290 us, dX 270 (in 256 x 192), dWg and
// dWu 240.
#include <algorithm>

#include "block_tiles.h"

namespace clear {
namespace block {
namespace {

constexpr int kStep = 64;  // of the contraction: the measure of costs, and a stage of LDS of most shapes
typedef __attribute__((ext_vector_type(4))) short short4v;
typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8_ptr;
typedef __attribute__((address_space(3))) short4v* lds_short4_ptr;

enum Kind { kForward, kInputGrad, kWeightGrad };

// ---- a tile of ROWS rows (or columns) x STEP (32 or 64) of the contraction in LDS ----------------------------------------------
// Stored along the contraction: rows of 2 STEP bytes, 16-byte chunk c of row r in slot c ^ turn_of(r).  A load instruction fills 8 or 16 rows; the operand read
// takes 16 bytes of 32 rows a half wave, and 16 neighbouring rows (two or four of them to the 256 bytes that LDS is wide) lie in different banks.
// Stored across: STEP rows of 2 ROWS bytes; 32-byte granule g (16 columns) of contraction row k in slot g ^ spread(k & 3).  A load instruction
// fills 1 KB, 2 or 4 contraction rows.  The transpose read takes, for 16 lanes, 32 bytes of 4 contraction rows: with the spread of 0, 5, 2, 7 these lie in
// different banks, those of the neighbouring 16 lanes (the granule beside) too.
__device__ __forceinline__ int spread(int k) { return (k & 3) ^ ((k & 1) << 2); }

// A tile: WA x WB waves of NA x NB blocks of 32 x 32, RING stages of STEP of the contraction.
template <int KIND, int WA, int WB, int NA, int NB, int STEP, int RING>
struct Shape {
    static constexpr int TA = 32 * NA * WA, TB = 32 * NB * WB, WAVES = WA * WB, THREADS = 64 * WAVES;
    static constexpr bool A_COLUMNS = KIND != kForward, B_COLUMNS = KIND == kWeightGrad;
    static constexpr int A_BYTES = TA * 2 * STEP, B_BYTES = TB * 2 * STEP, STAGE = A_BYTES + B_BYTES, LDS = RING * STAGE;
    static constexpr int A_LOADS = A_BYTES / 1024 / WAVES, B_LOADS = B_BYTES / 1024 / WAVES, LOADS = A_LOADS + B_LOADS;  // instructions a wave, 1 KB each
    static_assert(A_BYTES / 1024 % WAVES == 0 && B_BYTES / 1024 % WAVES == 0, "the waves share the loads of a stage evenly");
    static_assert((!A_COLUMNS || 512 % TA == 0) && (!B_COLUMNS || 512 % TB == 0), "an instruction fills whole contraction rows");
    static_assert(A_COLUMNS || A_BYTES / 2048 % A_LOADS == 0, "a wave's share of A is of one weight");
    static_assert(STEP % 32 == 0 && NA % 2 == 0 && RING >= 2);
};

struct TileArgs {
    const __bf16 *a0, *a1, *b0, *b1;  // the operands, and the second of those that come in two
    long long ld_a0, ld_a1, ld_b0;
    int rows_a;          // extent of A's rows (the contiguous axis of the output)
    long long rows_b;    // of B's rows
    long long depth;     // the contraction (of each half)
    int tiles_a, tiles_b, act;
    __bf16 *out0, *out1;   // the output, and where its rows from rows_out0 on go (weight gradient)
    long long ld_out0, ld_out1, rows_out0;
    float* pre;            // forward: [2][rows_b] rows of ld_pre, or null
    long long ld_pre;
    float* parts;  // where the contraction is split: fp32 [gridDim.y][rows_b][rows_a], to be joined; else null
};

// 1 / (1 + 2^e).  The hardware's exponential and reciprocal, each good to an ulp or two, are far below the rounding of the result to bf16; an IEEE division
// made the epilogue of a 256 x 256 tile 4 us longer (of 70).
__device__ __forceinline__ float logistic2(float e) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(e)); }
constexpr float kLog2E = 1.4426950408889634f;
// tanh form: (1 + tanh z) / 2 = 1 / (1 + e^(-2 z)) with z = sqrt(2 / pi) (g + 0.044715 g^3); -2 z log2(e) = g (kTanh1 + kTanh3 g^2)
constexpr float kTanh1 = -2.f * 0.7978845608028654f * kLog2E, kTanh3 = kTanh1 * 0.044715f;

__device__ __forceinline__ float activation(float g, int act)
{
    if (act == CLEAR_ACT_SILU) return g * logistic2(-kLog2E * g);
    if (act == CLEAR_ACT_GELU_TANH) return g * logistic2(g * __builtin_fmaf(g * g, kTanh3, kTanh1));
    return 0.5f * g * (1.f + erff(g * 0.7071067811865476f));
}
// act(g) and act'(g).
__device__ __forceinline__ void activation_slope(float g, int act, float* value, float* slope)
{
    if (act == CLEAR_ACT_SILU) {
        const float s = logistic2(-kLog2E * g);
        *value = g * s;
        *slope = s + g * s * (1.f - s);
    } else if (act == CLEAR_ACT_GELU_TANH) {
        const float c = fabsf(g) > 30.f ? copysignf(30.f, g) : g;  // (s is 0 or 1 long before; a square that overflows would make 0 * inf of it)
        const float s = logistic2(c * __builtin_fmaf(c * c, kTanh3, kTanh1));
        *value = g * s;
        *slope = s + 2.f * c * s * (1.f - s) * 0.7978845608028654f * (1.f + 3.f * 0.044715f * c * c);
    } else {
        const float s = 0.5f * (1.f + erff(g * 0.7071067811865476f));
        *value = g * s;
        *slope = s + g * 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.5f * kLog2E * g * g);
    }
}

template <int KIND, int WA, int WB, int NA, int NB, int STEP, int RING>
__global__ void __launch_bounds__(64 * WA * WB) tile_kernel(const TileArgs t)
{
    typedef Shape<KIND, WA, WB, NA, NB, STEP, RING> S;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds_bytes[];
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)lds_bytes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wa = wave % WA, wb = wave / WA;
    int tile_a, tile_b;
    tile_of(blockIdx.x, gridDim.x, t.tiles_a, t.tiles_b, &tile_a, &tile_b);

    // origin of the tile; forward: the tile's A rows are TA / 2 rows of the gate weight and the same of the up weight
    const int a_first = tile_a * (KIND == kForward ? S::TA / 2 : S::TA);
    const long long b_first = (long long)tile_b * S::TB;
    const int steps_each = (int)((t.depth + STEP - 1) / STEP), steps_all = KIND == kInputGrad ? 2 * steps_each : steps_each;
    const int it_first = (int)((long long)steps_all * blockIdx.y / gridDim.y), it_end = (int)((long long)steps_all * (blockIdx.y + 1) / gridDim.y);
    const int steps = it_end - it_first;  // of this part of the contraction

    // ---- loads of a stage: instruction i of this wave is i-th of its share of A's, then of B's.  A lane's offsets stay as they are from stage to stage and the buffers
    // move on: a load costs the writing of M0 beside itself, a stage two scalar additions.
    const bool up = !S::A_COLUMNS && wave * S::A_LOADS >= S::A_BYTES / 2048;  // forward: this wave loads the up weight's rows
    // (The pointers and strides that the loop chooses between are pinned in registers: a choice between two arguments becomes a scalar load from the chosen
    // place otherwise, whose wait counts the LDS reads in flight too.)
    const __bf16 *a0 = up ? t.a1 : t.a0, *a1 = t.a1, *b0 = t.b0, *b1 = t.b1;
    long long ld_a0 = up ? t.ld_a1 : t.ld_a0, ld_a1 = t.ld_a1, ld_b = t.ld_b0;  // (the two halves of B are in one workspace and have one stride; those of A need not)
    asm("" : "+s"(a0), "+s"(a1), "+s"(b0), "+s"(b1), "+s"(ld_a0), "+s"(ld_a1), "+s"(ld_b));
    const long long rows_a = min((long long)t.rows_a - a_first, (long long)(KIND == kForward ? S::TA / 2 : S::TA)), rows_b = min(t.rows_b - b_first, (long long)S::TB);  // of the tile
    i32x4 buf_a, buf_b;
    unsigned voff[S::LOADS], lds_to = lds, move_a = 0, move_b = 0;
    int aimed = 0, plain_until = 0;  // the step that buffers and offsets are for; the first one behind it that takes more than moving the buffers on
    auto rows_offset = [&](int n, long long ld, int left) INLINED {
        constexpr int CHUNKS = STEP / 8, ROWS = 64 / CHUNKS;
        const int r = lane / CHUNKS, c = (lane % CHUNKS) ^ turn_of<STEP>(n * ROWS + r);
        return c * 8 < left ? (unsigned)((n * ROWS + r) * ld * 2 + c * 16) : kOutside;
    };
    auto columns_offset = [&](int n, int chunks, long long ld, long long width) INLINED {  // (chunks of 16 bytes a contraction row)
        const int k = n * (64 / chunks) + lane / chunks, slot = lane % chunks;
        const int c = ((slot >> 1) ^ spread(k)) << 1 | (slot & 1);
        return c * 8 < width ? (unsigned)(k * ld * 2 + c * 16) : kOutside;
    };
    // Buffers and offsets of step `aimed` of this part: the first one, one that is cut short by the contraction's end, the first of the second half, and those behind the
    // part's last, which read nothing.
    auto aim = [&]() INLINED {
        const int it = it_first + aimed;
        const bool upper = KIND == kInputGrad && it >= steps_each;
        const long long k0 = (long long)(upper ? it - steps_each : it) * STEP, left = it < it_end ? t.depth - k0 : 0, rows = min(left, (long long)STEP);
        const long long ld_a = upper ? ld_a1 : ld_a0;
        const __bf16 *const a = upper ? a1 : a0, *const b = upper ? b1 : b0;
        buf_a = S::A_COLUMNS ? buffer_of(a + k0 * ld_a + a_first, ((rows - 1) * ld_a + t.rows_a - a_first) * 2)
                             : buffer_of(a + a_first * ld_a + k0, left > 0 ? ((rows_a - 1) * ld_a + left) * 2 : 0);
        buf_b = S::B_COLUMNS ? buffer_of(b + k0 * ld_b + b_first, ((rows - 1) * ld_b + t.rows_b - b_first) * 2)
                             : buffer_of(b + b_first * ld_b + k0, left > 0 ? ((rows_b - 1) * ld_b + left) * 2 : 0);
        settled(buf_a, buf_b);
        // (A buffer that moves on along its rows keeps its length, which is still short of the row behind the last: what it lets through behind the last row's part of the
        // step, no lane's offset reaches.)
        move_a = left > 0 ? __builtin_amdgcn_readfirstlane((int)(S::A_COLUMNS ? STEP * ld_a * 2 : STEP * 2)) : 0;
        move_b = left > 0 ? __builtin_amdgcn_readfirstlane((int)(S::B_COLUMNS ? STEP * ld_b * 2 : STEP * 2)) : 0;
        plain_until = __builtin_amdgcn_readfirstlane(left > 0 ? min((upper ? steps_each : 0) + (int)(t.depth / STEP), it_end) - it_first : 0x7fffffff);
#pragma unroll
        for (int i = 0; i < S::A_LOADS; ++i) {
            const int n = wave * S::A_LOADS + i;
            voff[i] = S::A_COLUMNS ? columns_offset(n, S::TA / 8, ld_a, t.rows_a - a_first) : rows_offset(n - (up ? S::A_BYTES / 2048 : 0), ld_a, (int)rows);
        }
#pragma unroll
        for (int i = 0; i < S::B_LOADS; ++i) {
            const int n = wave * S::B_LOADS + i;
            voff[S::A_LOADS + i] = S::B_COLUMNS ? columns_offset(n, S::TB / 8, ld_b, t.rows_b - b_first) : rows_offset(n, ld_b, (int)rows);
        }
    };
    auto advance = [&](unsigned stage) INLINED {  // to the next step, whose place in LDS is `stage`
        lds_to = lds + stage;
        if (++aimed < plain_until) {
            move(buf_a, move_a);
            move(buf_b, move_b);
        } else
            aim();
    };
    auto load = [&](auto i) INLINED {
        if constexpr (i < S::A_LOADS)
            load_to_lds<i * 1024>(buf_a, voff[i], lds_to + wave * (S::A_LOADS * 1024));
        else
            load_to_lds<S::A_BYTES + (i - S::A_LOADS) * 1024>(buf_b, voff[i], lds_to + wave * (S::B_LOADS * 1024));
    };

    // ---- operand reads: 32 rows (columns), 16 s .. 16 s + 15 of the stage's contraction; lane l has row l % 32 and elements 8 (l / 32) .. + 7 of them.  Addresses:
    // along the contraction one for each s, the blocks at constant distances; across it one for each block, the s at constant distances.
    constexpr int SLOTS = STEP / 16, A_ADDR = S::A_COLUMNS ? NA : SLOTS, B_ADDR = S::B_COLUMNS ? NB : SLOTS;
    auto rows_address = [&](int first, int s) INLINED { return (unsigned)((first + (lane & 31)) * (2 * STEP) + (((2 * s + (lane >> 5)) ^ turn_of<STEP>(lane)) << 4)); };
    auto columns_address = [&](int first, int row_bytes) INLINED {
        const int j = lane & 15, k = 8 * (lane >> 5) + (j >> 2);
        return (unsigned)(k * row_bytes + ((((first >> 4) + ((lane >> 4) & 1)) ^ spread(j >> 2)) << 5) + 8 * (j & 3));
    };
    unsigned a_zero[A_ADDR], b_zero[B_ADDR], a_at[A_ADDR], b_at[B_ADDR];  // in stage 0, and in the present one
#pragma unroll
    for (int i = 0; i < A_ADDR; ++i)
        a_zero[i] = lds + (S::A_COLUMNS ? columns_address(32 * (NA * wa + i), 2 * S::TA) : rows_address((KIND == kForward ? 16 : 32) * NA * wa, i));
#pragma unroll
    for (int i = 0; i < B_ADDR; ++i) b_zero[i] = lds + S::A_BYTES + (S::B_COLUMNS ? columns_address(32 * (NB * wb + i), 2 * S::TB) : rows_address(32 * NB * wb, i));
    auto enter = [&](unsigned stage) INLINED {
#pragma unroll
        for (int i = 0; i < A_ADDR; ++i) a_at[i] = a_zero[i] + stage;
#pragma unroll
        for (int i = 0; i < B_ADDR; ++i) b_at[i] = b_zero[i] + stage;
    };
    auto read_columns = [&](unsigned base, int s, int row_bytes) INLINED {
        union {
            struct {
                short4v lo, hi;
            } h;
            bf16x8 v;
        } u;
        u.h.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(size_t)(base + (unsigned)(16 * s * row_bytes)));
        u.h.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_ptr)(size_t)(base + (unsigned)((16 * s + 4) * row_bytes)));
        return u.v;
    };
    bf16x8 a[2][NA], b[2][NB];
    // Read n of slot s, in the order of first use: a[0], b[0], the rest of a, the rest of b.
    auto read = [&](auto into, auto s, auto n) INLINED {
        if constexpr (n == 0 || (n >= 2 && n <= NA)) {
            constexpr int i = n == 0 ? 0 : n - 1;
            constexpr int away = KIND == kForward ? i / 2 * 64 * STEP + i % 2 * (S::A_BYTES / 2) : i * 64 * STEP;  // (forward: gate and up blocks in turn)
            if constexpr (S::A_COLUMNS)
                a[into][i] = read_columns(a_at[i], s, 2 * S::TA);
            else
                a[into][i] = *(lds_bf16x8_ptr)(size_t)(a_at[s] + away);
        } else {
            constexpr int j = n == 1 ? 0 : n - NA;
            if constexpr (S::B_COLUMNS)
                b[into][j] = read_columns(b_at[j], s, 2 * S::TB);
            else
                b[into][j] = *(lds_bf16x8_ptr)(size_t)(b_at[s] + j * 64 * STEP);
        }
    };

    f32x16 acc[NA][NB];
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // ---- the loop.  A stage is STEP / 16 slots; in each the operands of the next slot are read beside the products of this one, across the barrier too: its last
    // slot's operands are in registers when the stage is given up, and the next stage's first are read beside its products.  The order is written out, each read and
    // load behind a product of its own, as a wave's issue waits while the address unit is busy: loads take half of a stage's last slot and half of the next one's first.
    constexpr int PRODUCTS = NA * NB, READS = NA + NB, READ_IN = PRODUCTS * 3 / 4, EARLY = S::LOADS / 2;
    // Products of operands `from`; beside them the reads of slot s of the stage entered (not where s is SLOTS), and loads first .. last - 1.
    auto slot = [&](auto from, auto s, auto first, auto last) INLINED {
        auto one = [&](auto n) INLINED {
            if constexpr (s < SLOTS && n < READ_IN) {
                auto next = [&](auto r) INLINED { read(Int<1 - from>{}, s, r); };
                each_of<n * READS / READ_IN, (n + 1) * READS / READ_IN>(next);
            }
            __builtin_amdgcn_sched_barrier(0);
            acc[n % NA][n / NA] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[from][n % NA], b[from][n / NA], acc[n % NA][n / NA], 0, 0, 0);
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
    // All slots but the last, beside the first of them the rest of the loads begun before.
    auto slots = [&](auto loads) INLINED {
        auto one = [&](auto s) INLINED { slot(Int<s % 2>{}, Int<s + 1>{}, Int<EARLY>{}, Int<(s == 0 && loads ? S::LOADS : EARLY)>{}); };
        each_of<0, SLOTS - 1>(one);
    };
    // The loads of the stages after the last fall outside their buffers, all of them: nothing is read, and the loop has no branch for them.
    if (steps > 0) {
        aim();
        each_of<0, S::LOADS>(load);
#pragma unroll
        for (int i = 1; i < RING; ++i) {
            advance(i * S::STAGE);
            if (i + 1 < RING)
                each_of<0, S::LOADS>(load);
            else
                each_of<0, EARLY>(load);
        }
        settle(Int<(RING - 2) * S::LOADS + EARLY>{});
        enter(0);
        auto next = [&](auto r) INLINED { read(Int<0>{}, Int<0>{}, r); };
        each_of<0, READS>(next);
        unsigned stage = 0;
        for (int it = 0; it + 1 < steps; ++it) {
            const unsigned next_stage = stage + S::STAGE == S::LDS ? 0 : stage + S::STAGE;
            slots(std::true_type{});
            settle(Int<(RING - 2) * S::LOADS>{});
            advance(stage);
            enter(next_stage);
            __builtin_amdgcn_sched_barrier(0);
            slot(Int<1>{}, Int<0>{}, Int<0>{}, Int<EARLY>{});
            stage = next_stage;
        }
        slots(std::false_type{});
        slot(Int<1>{}, Int<SLOTS>{}, Int<0>{}, Int<0>{});
        settle(Int<0>{});  // (nothing may still be on its way to this workgroup's LDS, which is used again, and is given up in the end)
    }

    // ---- epilogue: register r of acc[i][j] is A row 8 (r / 4) + 4 (lane / 32) + r % 4 and B row lane % 32 of the two blocks.  Outputs go through a part of LDS of
    // the wave's own, so that neighbouring lanes store neighbouring 16 bytes of a row: 64 to 256 bytes together, where the registers hold 16 or 32 (4 608 x 2 432 x 6 528
    // with the products kept 320 -> 286 us).
    constexpr int OWN = S::LDS / S::WAVES;
    const unsigned own = lds + wave * OWN;
    // Of blocks j = from .. until - 1, `width` outputs of type T from `first` on.  value(j, g): this lane's outputs 8 g + 4 (lane / 32) .. + 3 of row lane % 32 of block j;
    // to(row): where a row is.  As many blocks at once as LDS has room for.
    auto store = [&](auto type, auto width, auto from, auto until, int first, auto value, auto to) INLINED {
        typedef decltype(type) T;
        typedef T four __attribute__((ext_vector_type(4)));
        constexpr int BLOCKS = until - from, BYTES = width * sizeof(T), PITCH = BYTES + 16, LANES = BYTES / 16, ROWS = 64 / LANES;
        constexpr int FIT = OWN / (32 * PITCH), TOGETHER = FIT >= BLOCKS ? BLOCKS : FIT >= 2 && BLOCKS % 2 == 0 ? 2 : 1;
        static_assert(FIT >= 1, "a block fits");
        const int c = first + lane % LANES * (int)(16 / sizeof(T));
        auto some = [&](auto k) INLINED {
            constexpr int j0 = from + k * TOGETHER;
            auto put_block = [&](auto n) INLINED {
                auto put = [&](auto g) INLINED {
                    *(__attribute__((address_space(3))) four*)(size_t)(own + (unsigned)((32 * n + (lane & 31)) * PITCH + (8 * g + 4 * (lane >> 5)) * (int)sizeof(T))) =
                        __builtin_convertvector(value(Int<j0 + n>{}, g), four);
                };
                each_of<0, width / 8>(put);
            };
            each_of<0, TOGETHER>(put_block);
            asm volatile("" ::: "memory");  // (a wave's LDS instructions are executed in order)
#pragma unroll
            for (int i = 0; i < TOGETHER * 32 / ROWS; ++i) {
                const int at = i * ROWS + lane / LANES;
                const i32x4 x = *(__attribute__((address_space(3))) i32x4*)(size_t)(own + (unsigned)(at * PITCH + lane % LANES * 16));
                const long long row = b_first + 32 * (NB * wb + j0) + at;
                if (row < t.rows_b && c < t.rows_a) *(i32x4*)(to(row) + c) = x;
            }
            asm volatile("" ::: "memory");
        };
        each_of<0, BLOCKS / TOGETHER>(some);
    };
    auto four_of = [&](auto i, auto j, auto g) INLINED {  // of block i of A and j of B
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = acc[i][j][4 * g + r];
        return x;
    };
    if constexpr (KIND == kForward) {
        const int first = a_first + 16 * NA * wa;
        const Int<16 * NA> width{};
        auto gate = [&](auto j, auto g) INLINED { return four_of(Int<g / 4 * 2>{}, j, Int<g % 4>{}); };
        auto up_of = [&](auto j, auto g) INLINED { return four_of(Int<g / 4 * 2 + 1>{}, j, Int<g % 4>{}); };
        auto hidden = [&](auto j, auto g) INLINED {
            const f32x4 x = gate(j, g), y = up_of(j, g);
            f32x4 h;
#pragma unroll
            for (int r = 0; r < 4; ++r) h[r] = activation(x[r], t.act) * y[r];
            return h;
        };
        auto block = [&](auto j) INLINED {
            const Int<j + 1> next{};
            store((__bf16)0.f, width, j, next, first, hidden, [&](long long row) INLINED { return t.out0 + row * t.ld_out0; });
            if (!t.pre) return;
            store(0.f, width, j, next, first, gate, [&](long long row) INLINED { return t.pre + row * t.ld_pre; });
            store(0.f, width, j, next, first, up_of, [&](long long row) INLINED { return t.pre + (t.rows_b + row) * t.ld_pre; });
        };
        each_of<0, NB>(block);
    } else {
        const int first = a_first + 32 * NA * wa;
        const Int<32 * NA> width{};
        auto sums = [&](auto j, auto g) INLINED { return four_of(Int<g / 4>{}, j, Int<g % 4>{}); };
        if (t.parts)
            store(0.f, width, Int<0>{}, Int<NB>{}, first, sums, [&](long long row) INLINED { return t.parts + (blockIdx.y * t.rows_b + row) * t.rows_a; });
        else
            store((__bf16)0.f, width, Int<0>{}, Int<NB>{}, first, sums, [&](long long row) INLINED {
                return KIND == kWeightGrad && row >= t.rows_out0 ? t.out1 + (row - t.rows_out0) * t.ld_out1 : t.out0 + row * t.ld_out0;
            });
    }
}

// ---- few tokens -----------------------------------------------------------------------------------------------------------
// Up to 16 MT tokens: bound by the one reading of the weights.  A workgroup takes 16 hidden channels (gate and up) and all of the contraction,
// its 8 waves every eighth 32 of it: weights go straight from memory to the operand registers (no other wave needs them), X comes from the caches.  The
// waves' sums are added in order in LDS.  One token, 4 096 x 11 264: 38 us, 4.9 TB/s (pieces of 64, more of them in flight
// or loads past the caches: 0 to 10 % slower).
constexpr int kFewWaves = 8;
template <int MT>
__global__ void __launch_bounds__(64 * kFewWaves) few_tokens_kernel(const GatedArgs g)
{
    __shared__ f32x4 part[kFewWaves][2 * MT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, C = g.channels;
    const int f0 = blockIdx.x * 16;
    const int f = min(f0 + (lane & 15), g.hidden - 1), sub = 8 * (lane >> 4);
    const __bf16* const wg = (const __bf16*)g.wg + f * g.ld_g + sub;
    const __bf16* const wu = (const __bf16*)g.wu + f * g.ld_u + sub;
    const __bf16* x[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = (const __bf16*)g.x + min((long long)(16 * m + (lane & 15)), g.tokens - 1) * g.ld_x + sub;
    f32x4 acc[2][MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[0][m] = acc[1][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 zero = {};
    constexpr int AHEAD = MT > 2 ? 2 : 4;  // pieces whose loads are in flight together
    for (int k0 = 32 * wave; k0 < C; k0 += 32 * kFewWaves * AHEAD) {
        bf16x8 a[AHEAD], b[AHEAD], v[AHEAD][MT];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int k = k0 + 32 * kFewWaves * i;
            const bool in = k + sub < C;  // (channels come in eights)
            a[i] = in ? *(const bf16x8*)(wg + k) : zero;
            b[i] = in ? *(const bf16x8*)(wu + k) : zero;
#pragma unroll
            for (int m = 0; m < MT; ++m) v[i][m] = in ? *(const bf16x8*)(x[m] + k) : zero;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                acc[0][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], v[i][m], acc[0][m], 0, 0, 0);
                acc[1][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[i], v[i][m], acc[1][m], 0, 0, 0);
            }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        part[wave][m][lane] = acc[0][m];
        part[wave][MT + m][lane] = acc[1][m];
    }
    __syncthreads();
    // register r of lane l: hidden channel 4 (l / 16) + r, token l % 16
    for (int at = threadIdx.x; at < MT * 64; at += 64 * kFewWaves) {
        const int m = at >> 6, l = at & 63;
        f32x4 a = part[0][m][l], u = part[0][MT + m][l];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) {
            a += part[w][m][l];
            u += part[w][MT + m][l];
        }
        const long long token = 16 * m + (l & 15);
        const int c = f0 + 4 * (l >> 4);
        if (token < g.tokens && c < g.hidden) {
            bf16x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = (__bf16)(activation(a[r], g.act) * u[r]);
            *(bf16x4*)((__bf16*)g.h + token * g.ld_h + c) = o;
            if (g.pre) {
                *(f32x4*)(g.pre + token * g.hidden + c) = a;
                *(f32x4*)(g.pre + (g.tokens + token) * g.hidden + c) = u;
            }
        }
    }
}

// dG = dH u act'(g) and dU = dH act(g) in bf16 [tokens][2 hidden], gate first, 8 channels a thread.  Memory-bound: 4 608 x 6 528 84 us, 5 TB/s
// (4 channels a thread, side by side, or 32-bit division: the same).  The rounding to bf16 is what the matrix instructions take: it adds 0.0017 of their norm to the error of dX, dWg
// and dWu, whose own rounding is as much, independently (0.0023 together); two terms each would take it out and double both products.
__global__ void __launch_bounds__(256) gated_gradient_kernel(const GatedArgs g, long long n)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= n) return;
    const int each = g.hidden / 8;
    const long long row = id / each;
    const int c = (int)(id - row * each) * 8;
    const bf16x8 dh = *(const bf16x8*)((const __bf16*)g.dh + row * g.ld_dh + c);
    const long long at = row * g.hidden + c, plane = g.tokens * g.hidden;
    f32x4 gate[2], up[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        gate[i] = *(const f32x4*)(g.pre + at + 4 * i);
        up[i] = *(const f32x4*)(g.pre + plane + at + 4 * i);
    }
    bf16x8 dg, du;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float value, slope;
        activation_slope(gate[j >> 2][j & 3], g.act, &value, &slope);
        dg[j] = (__bf16)((float)dh[j] * up[j >> 2][j & 3] * slope);
        du[j] = (__bf16)((float)dh[j] * value);
    }
    __bf16* const ws = (__bf16*)g.ws;
    *(bf16x8*)(ws + row * 2 * g.hidden + c) = dg;
    *(bf16x8*)(ws + row * 2 * g.hidden + g.hidden + c) = du;
}

// The sum of the parts of a split contraction, in order, to the output; 8 outputs a thread.
__global__ void __launch_bounds__(256) join_kernel(const TileArgs t, int parts, long long n)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= n) return;
    const int each = t.rows_a / 8;
    const long long row = id / each, plane = t.rows_b * t.rows_a;
    const int c = (int)(id - row * each) * 8;
    const float* const from = t.parts + row * t.rows_a + c;
    f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + 4);
#pragma unroll 4
    for (int p = 1; p < parts; ++p) {
        lo += *(const f32x4*)(from + p * plane);
        hi += *(const f32x4*)(from + p * plane + 4);
    }
    bf16x8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (__bf16)(j < 4 ? lo[j & 3] : hi[j & 3]);
    const bool second = t.out1 && row >= t.rows_out0;
    *(bf16x8*)((second ? t.out1 + (row - t.rows_out0) * t.ld_out1 : t.out0 + row * t.ld_out0) + c) = o;
}

template <int KIND, int WA, int WB, int NA, int NB, int STEP, int RING>
hipError_t launch_tiles(TileArgs t, int parts, hipStream_t stream)
{
    typedef Shape<KIND, WA, WB, NA, NB, STEP, RING> S;
    const int a_rows = KIND == kForward ? S::TA / 2 : S::TA;
    t.tiles_a = (t.rows_a + a_rows - 1) / a_rows;
    const long long tiles_b = (t.rows_b + S::TB - 1) / S::TB;
    if (tiles_b > 0x7fffffffLL || tiles_b * t.tiles_a > 0xffffffffLL / S::THREADS) return hipErrorInvalidValue;
    t.tiles_b = (int)tiles_b;
    if (parts == 1) t.parts = nullptr;
    static LdsLimit limit;
    const hipError_t allowed = limit.ensure((const void*)tile_kernel<KIND, WA, WB, NA, NB, STEP, RING>, S::LDS);
    if (allowed != hipSuccess) return allowed;
    tile_kernel<KIND, WA, WB, NA, NB, STEP, RING><<<dim3((unsigned)(tiles_b * t.tiles_a), parts), dim3(S::THREADS), S::LDS, stream>>>(t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    const long long n = t.rows_b * (t.rows_a / 8), blocks = (n + 255) / 256;
    if (blocks > 0xffffffffLL / 256) return hipErrorInvalidValue;
    join_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(t, parts, n);
    return hipGetLastError();
}

// Tile shape and number of parts that the contraction is split into, by the time they are expected to take: rounds of workgroups over the 256 CUs, each of a
// part's steps (64 of the contraction) and of what a tile costs beside (first loads, epilogue).  The constants, in us, were fitted to 1100 timings of the three products
// in all shapes and 1 to 16 parts, at 100 to 8192 tokens and widths of 512 x 1024 to 4096 x 11264: the chosen form takes 0.3 % longer than the best of them on average, at most
// 4 % (dW of the smallest width 11 %).  (At 2432 x 6528 dG, dU and dX of 100 tokens take 241 us in 256 x 256 tiles, 85 in deep ones, 26 in those with the
// contraction in 8 parts; of 4608 tokens 362 in 256 x 256 tiles, which leave 76 CUs without one, 336 in 256 x 192 and 378 in small ones.)
enum TileShape { kLarge, kMedium, kPair, kDeep, kNarrow };  // 256 x 256; 256 x 192; 128 x 128, two workgroups a CU; 128 x 128, one a CU with four stages in flight; 64 x 128, one with six
struct Plan {
    TileShape shape;
    int parts;
    double us;  // expected
};
Plan plan_of(int kind, long long rows_a, long long rows_b, long long depth)
{
    const long long a = kind == kForward ? 2 * rows_a : rows_a, steps = (depth + kStep - 1) / kStep * (kind == kInputGrad ? 2 : 1);
    const auto up = [](long long x, long long by) { return (x + by - 1) / by; };
    const long long large = up(a, 256) * up(rows_b, 256), medium = up(a, 256) * up(rows_b, 192), small = up(a, 128) * up(rows_b, 128);
    // Forward, where a CU each is enough for them, tiles of 32 hidden channels x 128 tokens: what few tokens wait for is the weights, and more CUs ask for them (33 and 128 tokens
    // with weights from memory: 1536 x 4096 13 and 17 us, in 128 x 128 tiles 17 and 21; 2432 x 6528 19 and 24, 24 and 30; 4096 x 8192 31 and 37, 37 and 46; with tiles for two
    // rounds 2048 x 8640 31 and 36, 23 and 27).
    if (kind == kForward && up(a, 64) * up(rows_b, 128) <= 256) return {kNarrow, 1, steps * 0.37 + 5.5};
    Plan best = {kLarge, 1, 0};
    for (int parts = 1; parts <= (kind == kForward ? 1 : 16); ++parts) {
        if (parts > 1 && steps < 8 * parts) break;
        const double each = (double)up(steps, parts);
        // (the parts are written and read once more)
        const double join = parts == 1 ? 0 : 2.01 + (1.8 * parts + 0.5) * rows_a * rows_b * 4 / 4e6;
        const double us[4] = {up(large * parts, 256) * (each * 1.3 + 8.58) + join, up(medium * parts, 256) * (each * 1.07 + 8.22) + join,
                              (small * parts <= 256 ? each * 0.625 + 7.29 : up(small * parts, 512) * (each * 0.89 + 7.29)) + join,  // (a CU to itself where there are enough)
                              up(small * parts, 256) * (each * 0.468 + 7.71) + join};
        for (int s = 0; s < 4; ++s)
            if ((best.us == 0 || us[s] < best.us) && !(s == kMedium && kind == kWeightGrad))  // (stored across, 192 columns are no whole part of a load instruction)
                best = {(TileShape)s, parts, us[s]};
    }
    return best;
}
Plan input_plan(long long tokens, int channels, int hidden) { return plan_of(kInputGrad, channels, tokens, hidden); }
Plan weight_plan(long long tokens, int channels, int hidden) { return plan_of(kWeightGrad, channels, 2LL * hidden, tokens); }

template <int KIND>
hipError_t launch_plan(const TileArgs& t, const Plan& p, hipStream_t stream)
{
    // Stages of 32, four in flight, instead of 64 and two: dX and dW at 4 608 x 2 432 x 6 528 8 and 4 % faster; forward, where then both operands would be read in
    // halves of cache lines, 4 to 10 % slower.  256 x 192 has four waves there, as eight would not share its loads evenly.
    constexpr int STEP = KIND == kForward ? 64 : 32, RING = 128 / STEP;
    if (p.shape == kLarge) return launch_tiles<KIND, 4, 2, 2, 4, STEP, RING>(t, p.parts, stream);
    if constexpr (KIND == kForward) {
        if (p.shape == kNarrow) return launch_tiles<KIND, 1, 4, 2, 1, STEP, 6>(t, p.parts, stream);
        if (p.shape == kMedium) return launch_tiles<KIND, 4, 2, 2, 3, STEP, RING>(t, p.parts, stream);
    }
    if constexpr (KIND == kInputGrad)
        if (p.shape == kMedium) return launch_tiles<KIND, 2, 2, 4, 3, STEP, RING>(t, p.parts, stream);
    return p.shape == kPair ? launch_tiles<KIND, 2, 2, 2, 2, 64, 2>(t, p.parts, stream) : launch_tiles<KIND, 2, 2, 2, 2, 64, 4>(t, p.parts, stream);
}

// Hidden channels of the first of two launches forward, or all of them.  Where 256 x 256 tiles fill some rounds and a small part of another one, the channels of the full
// rounds, or of one less, go first and the rest in the tiles that suit it, if that is expected to save 5 % with 4 us for the second launch (1500 tokens at 2432 x 6528 98 -> 91 us,
// 1000 at 4096 x 11264 182 -> 161, 3000 there 486 -> 448; where less was expected it did not: 4608 at 2432 x 6528 245 -> 251).
int first_launch(const GatedArgs& a)
{
    const long long bands = (a.tokens + 255) / 256, columns = (a.hidden + 127) / 128, rounds = (bands * columns + 255) / 256;
    double best = 0.95 * plan_of(kForward, a.hidden, a.tokens, a.channels).us;
    int first = a.hidden;
    for (long long full = std::max(1LL, rounds - 2); full < rounds; ++full) {
        const long long some = full * 256 / bands;
        if (some < 1 || some >= columns) continue;
        const double us = plan_of(kForward, some * 128, a.tokens, a.channels).us + plan_of(kForward, a.hidden - some * 128, a.tokens, a.channels).us + 4;
        if (us < best) best = us, first = (int)(some * 128);
    }
    return first;
}

// Whether the form for few tokens is the faster one, by the times, in us, that both are expected to take with weights from memory.  It reads X again for every 16 hidden
// channels and is not faster for a CU that has less of them than others; the tiles take nearly the same time up to 64 tokens.  Measured, 1, 16 and 32 tokens here, 16 in
// tiles: 1 536 x 4 096 11, 11, 11 and 13; 2 432 x 6 528 16, 19, 23 and 19; 3 200 x 8 640 28, 35, 40 and 31; 4 096 x 11 264 38, 46, 55 and 44; 5 120 x 13 824 63, 79, 97 and 52.
bool few_tokens(const GatedArgs& a)
{
    if (a.tokens > 64) return false;
    const double here = 3.1e-3 * a.channels * ((a.hidden + 4095) / 4096) * (1 + a.tokens / 64.);
    const double tiles = a.hidden <= 8192 ? 6.7e-3 * a.channels + 2.3 : (9.4e-3 * a.channels + 2) * ((a.hidden + 16383) / 16384);
    return here <= tiles;
}

}  // namespace

hipError_t launch_gated_forward(const GatedArgs& a, hipStream_t stream)
{
    if (few_tokens(a)) {
        const dim3 grid((a.hidden + 15) / 16), block(64 * kFewWaves);
        if (a.tokens <= 16) few_tokens_kernel<1><<<grid, block, 0, stream>>>(a);
        else if (a.tokens <= 32) few_tokens_kernel<2><<<grid, block, 0, stream>>>(a);
        else few_tokens_kernel<4><<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    }
    TileArgs t = {};
    t.a0 = (const __bf16*)a.wg, t.a1 = (const __bf16*)a.wu, t.b0 = (const __bf16*)a.x;
    t.ld_a0 = a.ld_g, t.ld_a1 = a.ld_u, t.ld_b0 = a.ld_x;
    t.rows_a = a.hidden, t.rows_b = a.tokens, t.depth = a.channels;
    t.act = a.act;
    t.out0 = (__bf16*)a.h, t.ld_out0 = a.ld_h;
    t.pre = a.pre, t.ld_pre = a.hidden;
    const int first = first_launch(a);
    t.rows_a = first;
    const hipError_t e = launch_plan<kForward>(t, plan_of(kForward, t.rows_a, t.rows_b, t.depth), stream);
    if (e != hipSuccess || first == a.hidden) return e;
    t.a0 += first * t.ld_a0, t.a1 += first * t.ld_a1;
    t.out0 += first;
    if (t.pre) t.pre += first;
    t.rows_a = a.hidden - first;
    return launch_plan<kForward>(t, plan_of(kForward, t.rows_a, t.rows_b, t.depth), stream);
}

// dG and dU at the head of the workspace.
static size_t gradient_bytes(long long tokens, int hidden) { return (size_t)tokens * hidden * 4; }

size_t gated_workspace_bytes(long long tokens, int channels, int hidden)
{
    if (tokens == 0) return 0;
    const int in = input_plan(tokens, channels, hidden).parts, w = weight_plan(tokens, channels, hidden).parts;
    const size_t in_bytes = in > 1 ? (size_t)in * tokens * channels * 4 : 0, w_bytes = w > 1 ? (size_t)w * 2 * hidden * channels * 4 : 0;
    return gradient_bytes(tokens, hidden) + std::max(in_bytes, w_bytes);  // dG and dU, then the parts of one of the products at a time
}

hipError_t launch_gated_backward(const GatedArgs& a, hipStream_t stream)
{
    const __bf16* const dg = (const __bf16*)a.ws;
    const __bf16* const du = dg + a.hidden;
    float* const parts = (float*)((unsigned char*)a.ws + gradient_bytes(a.tokens, a.hidden));  // (16-byte aligned: hidden is a multiple of 8)
    hipError_t e = hipSuccess;
    if (a.tokens > 0) {
        const long long n = a.tokens * (a.hidden / 8), blocks = (n + 255) / 256;
        if (blocks > 0xffffffffLL / 256) return hipErrorInvalidValue;
        gated_gradient_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(a, n);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.dx && a.tokens > 0) {
        TileArgs t = {};
        t.a0 = (const __bf16*)a.wg, t.a1 = (const __bf16*)a.wu, t.b0 = dg, t.b1 = du;
        t.ld_a0 = a.ld_g, t.ld_a1 = a.ld_u, t.ld_b0 = 2LL * a.hidden;
        t.rows_a = a.channels, t.rows_b = a.tokens, t.depth = a.hidden;
        t.out0 = (__bf16*)a.dx, t.ld_out0 = a.ld_dx;
        t.parts = parts;
        e = launch_plan<kInputGrad>(t, input_plan(a.tokens, a.channels, a.hidden), stream);
    }
    if (e == hipSuccess && a.dwg) {
        TileArgs t = {};
        t.a0 = (const __bf16*)a.x, t.b0 = dg;
        t.ld_a0 = a.ld_x, t.ld_b0 = 2LL * a.hidden;
        t.rows_a = a.channels, t.rows_b = 2LL * a.hidden, t.depth = a.tokens;
        t.rows_out0 = a.hidden;
        t.out0 = (__bf16*)a.dwg, t.ld_out0 = a.ld_dwg;
        t.out1 = (__bf16*)a.dwu, t.ld_out1 = a.ld_dwu;
        t.parts = parts;
        e = launch_plan<kWeightGrad>(t, weight_plan(a.tokens, a.channels, a.hidden), stream);
    }
    return e;
}

}  // namespace block
}  // namespace clear
