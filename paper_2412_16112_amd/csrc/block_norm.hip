// Layer norm over the last axis and its backward pass.  Memory-bound: a row is read once and kept in registers between its
// mean, its variance (of the differences from the mean) and its result; the backward pass reads dy and x once for dX and both
// weight sums.
//
// A team of TEAM waves holds a row in chunks of 8 channels a lane: lane l of the team owns chunks l, l + 64 TEAM, ... (fp32: pairs of fours, so that neighbouring lanes load
// neighbouring 16 bytes: 16 717 x 1 111 forward 37 -> 34 us), any alignment.  Forward, a row takes as few waves as it fills well: one up to 1536 channels (sums by lane
// exchange, no barrier) and for bf16 from 2049 to 2560 (five chunks; two waves would leave a fifth of their lanes idle: 9 216 rows of 2 056, 2 304, 2 560 channels 17.7, 19.5,
// 18.6 us, in two waves 18.5, 19.8, 20.7; in fp32 28.2, 30.4, 32.1 and 26.7, 28.5, 31.3), else 2, 4 or 8; workgroups of 256, of which more fit beside each other than of 512
// (16 896 x 4 096 52 -> 48).  Backward, where a lane also holds two sums for each of its channels, a wave holds up to 1536
// channels and longer rows take 2, 4 or 8 (with 5 chunks a lane the registers no longer suffice).
// What bounds it is what is in flight: a branch that waits for a load where the next row is asked for cost a third (9 216 x 2 432 bf16 backward 42 -> 29), so ragged ends have none.
// 9 216 x 2 432 bf16: forward 20 us (4.5 TB/s), backward 29 (4.7), 3.4 for the join of the sums; 16 717 x 1 111 fp32 30 and 39 (4.9 and 5.7), 4.4; 16 896 x 4 096 bf16 47 (5.9 TB/s) and 79
// with the join (5.3).
#include <algorithm>
#include <type_traits>

#include "block_internal.h"

namespace clear {
namespace block {
namespace {

__host__ __device__ constexpr int forward_threads(int team) { return team == 8 ? 512 : 256; }
// With one chunk a lane 16 waves (or as many whole teams) have the registers, else 8: fp32 rows of 256 channels 47 -> 40 us a 60000, bf16 of 512 27 -> 24 a 32768.
__host__ __device__ constexpr int backward_threads(int team, int ch) { return ch == 1 ? 16 / team * team * 64 : 512; }
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

template <typename T, typename TW, int TEAM, int CH, bool WHOLE>
__global__ void __launch_bounds__(forward_threads(TEAM)) norm_forward_kernel(NormArgs a, long long row_first)
{
    constexpr int WAVES = forward_threads(TEAM) / 64, TEAMS = WAVES / TEAM;
    typedef Layout<T, TEAM, CH, WHOLE> L;
    __shared__ float slots[2][WAVES][1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x % (64 * TEAM);
    const long long total = (long long)a.groups * a.rows;
    const long long row = row_first + (long long)blockIdx.x * TEAMS + wave / TEAM;
    const bool live = row < total;
    const int at = live ? (int)row : 0;
    const int g = at / a.rows, r = at - g * a.rows;
    const T* const x = (const T*)a.x + g * a.st[0] + r * a.st[1];
    const int C = a.channels;
    Chunk8<T> v[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = L::first(lane, i);
        v[i].template load<L::GAP>(x + c, C - c, L::form(C, i));
    }
    const TW* const w = a.w ? (const TW*)a.w + (a.per_group ? (long long)g * C : 0) : nullptr;
    const TW* const b = a.b ? (const TW*)a.b + (a.per_group ? (long long)g * C : 0) : nullptr;
    Chunk8<TW> cw[CH], cb[CH];  // (asked for here: they arrive while the sums are formed)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = L::first(lane, i);
        if (w) cw[i].template load<L::GAP>(w + c, C - c, L::form(C, i));
        if (b) cb[i].template load<L::GAP>(b + c, C - c, L::form(C, i));
    }
    const int last = C - L::first(lane, CH - 1);
    const RowForm form = L::form(C, CH - 1);  // of the last chunks; the others are whole
    v[CH - 1].template clear_others<L::GAP>(last, form);
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += v[i].get(j);
    team_sum<TEAM>(s, slots[0], wave);
    const float mean = s[0] / (float)C;
    float q[1] = {0.f};
    auto add_squares = [&](int i, auto all) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = v[i].get(j) - mean;
            q[0] += all || L::P::own(j, last, form) ? d * d : 0.f;
        }
    };
#pragma unroll
    for (int i = 0; i + 1 < CH; ++i) add_squares(i, std::true_type{});
    add_squares(CH - 1, std::bool_constant<WHOLE>{});
    team_sum<TEAM>(q, slots[1], wave);
    const float rstd = 1.0f / sqrtf(q[0] / (float)C + a.eps);
    if (!live) return;
    if (a.stats && lane == 0) {
        a.stats[row] = mean;
        a.stats[total + row] = rstd;
    }
    T* const y = (T*)a.y + g * a.st[2] + r * a.st[3];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = L::first(lane, i);
        if (c >= C) break;
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            o[j] = (v[i].get(j) - mean) * rstd;
            if (w) o[j] *= a.offset + cw[i].get(j);
            if (b) o[j] += cb[i].get(j);
        }
        Chunk8<T>::template store<L::GAP>(y + c, C - c, L::form(C, i), o);
    }
}

// Workgroup (p, set) of the grid takes rows p TEAMS + team, then every gridDim.x TEAMS further ones, of the set (a group, or everything when the weight
// is shared), writes their dX and adds up dy xhat and dy in registers; the teams' sums are added in order and become partial p of the set.
template <typename T, typename TW, int TEAM, int CH, bool WHOLE>
__global__ void __launch_bounds__(backward_threads(TEAM, CH)) norm_backward_kernel(NormArgs a)
{
    constexpr int WAVES = backward_threads(TEAM, CH) / 64, TEAMS = WAVES / TEAM;
    typedef Layout<T, TEAM, CH, WHOLE> L;
    extern __shared__ __attribute__((aligned(16))) float lds[];  // [2][padded channels] where a workgroup has several teams
    __shared__ float slots[2][WAVES][2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x % (64 * TEAM), team = wave / TEAM;
    const int C = a.channels, set = blockIdx.y;
    const long long in_set = a.per_group ? a.rows : (long long)a.groups * a.rows;
    const long long first = a.per_group ? (long long)set * a.rows : 0;
    const long long total = (long long)a.groups * a.rows;
    const bool sums = a.dw || a.db;
    const TW* const w = a.w ? (const TW*)a.w + (a.per_group ? (long long)set * C : 0) : nullptr;
    Chunk8<TW> cw[CH];
    if (w) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = L::first(lane, i);
            cw[i].template load<L::GAP>(w + c, C - c, L::form(C, i));
        }
    }
    float dw[CH][8], db[CH][8];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.f;
    const long long step = (long long)gridDim.x * TEAMS;
    struct Row {
        Chunk8<T> x[CH], dy[CH];
        float mean, rstd;
        int g, r;
        bool live;
    };
    auto fetch = [&](long long base, Row* to) {  // (a row that is not there: the set's first, with a dy of 0)
        to->live = base + team < in_set;
        const long long row = first + (to->live ? base + team : 0);
        to->g = (int)row / a.rows;
        to->r = (int)row - to->g * a.rows;
        const T* const x = (const T*)a.x + to->g * a.st[2] + to->r * a.st[3];
        const T* const dy = (const T*)a.dy + to->g * a.st[0] + to->r * a.st[1];
        to->mean = a.stats[row];
        to->rstd = a.stats[total + row];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = L::first(lane, i);
            to->x[i].template load<L::GAP>(x + c, C - c, L::form(C, i));
            to->dy[i].template load<L::GAP>(dy + c, to->live ? C - c : 0, to->live ? L::form(C, i) : RowForm{false, false});
        }
    };
    constexpr bool AHEAD = CH < 4;  // the next row's loads are under way while a row is worked on; with 4 chunks a lane there are no registers for it
    Row now, next;
    if (AHEAD) fetch((long long)blockIdx.x * TEAMS, &next);
    int turn = 0;
    for (long long base = (long long)blockIdx.x * TEAMS; base < in_set; base += step, turn ^= 1) {  // (the same number of turns for every wave)
        if (AHEAD) {
            __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);  // vmcnt 0, here and not behind the next row's loads, where the compiler would put it for the first turn's sake
            now = next;
            if (base + step < in_set) fetch(base + step, &next);
        } else {
            fetch(base, &now);
        }
        now.dy[CH - 1].template clear_others<L::GAP>(C - L::first(lane, CH - 1), L::form(C, CH - 1));
        const Chunk8<T>(&vx)[CH] = now.x, (&vd)[CH] = now.dy;
        const float mean = now.mean, rstd = now.rstd;
        const bool live = now.live;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = vd[i].get(j), h = (vx[i].get(j) - mean) * rstd;
                const float dyw = w ? d * (a.offset + cw[i].get(j)) : d;
                s[0] += dyw;
                s[1] += dyw * h;
                if (sums && live) {
                    dw[i][j] += d * h;
                    db[i][j] += d;
                }
            }
        if (a.dx) {
            team_sum<TEAM>(s, slots[turn], wave);
            const float s1 = s[0] / (float)C, s2 = s[1] / (float)C;
            if (live) {
                T* const dx = (T*)a.dx + now.g * a.st[4] + now.r * a.st[5];
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const int c = L::first(lane, i);
                    if (c >= C) break;
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float d = vd[i].get(j), h = (vx[i].get(j) - mean) * rstd;
                        o[j] = rstd * ((w ? d * (a.offset + cw[i].get(j)) : d) - s1 - h * s2);
                    }
                    Chunk8<T>::template store<L::GAP>(dx + c, C - c, L::form(C, i), o);
                }
            }
        }
    }
    if (!sums) return;
    const int wide = padded(C);
    float* const out = a.ws + ((long long)set * gridDim.x + blockIdx.x) * 2 * wide;
    // (LDS by pointers of its own address space: with one pointer to either, the stores become flat ones, whose base, taken in front of the first channel and led back by
    // the instruction's offset, can lie outside LDS and is then an address in memory.)
    const shared_float sum = (shared_float)lds;
    auto give = [&](auto to, bool more) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const int n = C - L::first(lane, i), c = C - n + L::P::first(h) + L::P::in(h);
                const RowForm form = L::form(C, i);
                if (form.whole || L::P::back(h, n) == 0) {
                    f32x4 sw = {dw[i][h], dw[i][h + 1], dw[i][h + 2], dw[i][h + 3]}, sb = {db[i][h], db[i][h + 1], db[i][h + 2], db[i][h + 3]};
                    if (more) {
                        sw += *(shared_f32x4)(sum + c);
                        sb += *(shared_f32x4)(sum + wide + c);
                    }
                    put_four(to + c, sw);
                    put_four(to + wide + c, sb);
                } else {
#pragma unroll
                    for (int j = h; j < h + 4; ++j) {
                        if (!L::P::own(j, n, form)) continue;
                        const int at = C - n + L::P::at(j, n, form);
                        to[at] = more ? dw[i][j] + sum[at] : dw[i][j];
                        to[wide + at] = more ? db[i][j] + sum[wide + at] : db[i][j];
                    }
                }
            }
        }
    };
    for (int t = 0; t < TEAMS; ++t) {
        if (team == t) {
            if (t + 1 < TEAMS)
                give(sum, t > 0);
            else
                give(out, t > 0);
        }
        __syncthreads();
    }
}

// d_weight and d_bias of a set from its partials: a workgroup takes 64 of their columns, wave w the partials w, w + 16, ...
template <typename TW>
__global__ void __launch_bounds__(1024) norm_join_kernel(NormArgs a, int partials)
{
    __shared__ float part[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wide = padded(a.channels), set = blockIdx.y;
    const int col = blockIdx.x * 64 + lane;
    const float* const from = a.ws + (long long)set * partials * 2 * wide + col;
    float s = 0.f;
    if (col < 2 * wide) {
        int p = wave;
        for (; p + 48 < partials; p += 64) {  // (four loads in flight)
            const float x0 = from[(long long)p * 2 * wide], x1 = from[(long long)(p + 16) * 2 * wide];
            const float x2 = from[(long long)(p + 32) * 2 * wide], x3 = from[(long long)(p + 48) * 2 * wide];
            s += (x0 + x1) + (x2 + x3);
        }
        for (; p < partials; p += 16) s += from[(long long)p * 2 * wide];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += part[i][lane];
        const int c = col < wide ? col : col - wide;
        TW* const to = (TW*)(col < wide ? a.dw : a.db);
        if (to && c < a.channels) to[(long long)set * a.channels + c] = (TW)s;
    }
}

// `whole`: rows fill their last chunks too; they have instances of their own, without masks.
struct Form {
    int team, ch;
    bool whole;
    Form(int team, int channels) : team(team), ch((channels + 512 * team - 1) / (512 * team)), whole(channels == 512 * team * ch) {}
};
Form forward_form(int channels, bool fp32)
{
    const int team = channels <= 1536 || (!fp32 && channels > 2048 && channels <= 2560) ? 1 : channels <= 4096 ? 2 : channels <= 8192 ? 4 : 8;
    return Form(team, channels);
}
Form backward_form(int channels, bool fp32)
{
    // (fp32 rows of 1025 to 1536 channels: three waves of one chunk, 15 waves a CU, instead of one of three, 8 a CU: 16717 rows of 1032, 1111, 1280, 1536 channels 40.5, 42.9, 46.9,
    // 58.4 us with the join, in one wave 43.8, 47.4, 50.7, 61.5)
    const int team = channels <= 1536 ? (fp32 && channels > 1024 ? 3 : 1) : channels <= 2 * 1536 ? 2 : channels <= 4 * 1536 ? 4 : 8;
    return Form(team, channels);
}

// call(team, ch, whole) with all three as integral constants, if (TEAM, CH) is the form.
template <int TEAM, int CH, typename F>
bool try_form(const Form& f, F& call)
{
    if (f.team != TEAM || f.ch != CH) return false;
    if (f.whole)
        call(std::integral_constant<int, TEAM>{}, std::integral_constant<int, CH>{}, std::true_type{});
    else
        call(std::integral_constant<int, TEAM>{}, std::integral_constant<int, CH>{}, std::false_type{});
    return true;
}

template <typename T, typename TW>
hipError_t forward(const NormArgs& a, hipStream_t stream)
{
    const Form f = forward_form(a.channels, sizeof(T) == 4);
    hipError_t e = hipSuccess;
    auto call = [&](auto team, auto ch, auto whole) {
        constexpr int TEAM = team, CH = ch, threads = forward_threads(TEAM), teams = threads / 64 / TEAM;
        constexpr long long most = 0xffffffffLL / threads;  // workgroups a launch can have
        const long long rows = (long long)a.groups * a.rows;
        for (long long first = 0; first < rows && e == hipSuccess; first += most * teams) {  // (one launch up to 2^23 rows and more)
            const long long blocks = std::min(most, (rows - first + teams - 1) / teams);
            norm_forward_kernel<T, TW, TEAM, CH, whole><<<dim3((unsigned)blocks), dim3(threads), 0, stream>>>(a, first);
            e = hipGetLastError();
        }
    };
    bool ok = try_form<1, 1>(f, call) || try_form<1, 2>(f, call) || try_form<1, 3>(f, call) || try_form<2, 2>(f, call) || try_form<2, 3>(f, call) ||
              try_form<2, 4>(f, call) || try_form<4, 3>(f, call) || try_form<4, 4>(f, call) || try_form<8, 3>(f, call) || try_form<8, 4>(f, call);
    if constexpr (sizeof(T) == 2) ok = ok || try_form<1, 5>(f, call);
    return ok ? e : hipErrorInvalidValue;
}

template <typename T, typename TW>
hipError_t backward(const NormArgs& a, hipStream_t stream)
{
    const Form f = backward_form(a.channels, sizeof(T) == 4);
    const int sets = a.per_group ? a.groups : 1;
    const int partials = norm_partials(a.groups, a.rows, a.channels, a.per_group);
    hipError_t e = hipSuccess;
    if (partials > 0) {
        auto call = [&](auto team, auto ch, auto whole) {
            constexpr int TEAM = team, CH = ch, threads = backward_threads(TEAM, CH), teams = threads / 64 / TEAM;
            const size_t lds = teams > 1 && (a.dw || a.db) ? (size_t)padded(a.channels) * 8 : 0;  // (at most 48 KB)
            norm_backward_kernel<T, TW, TEAM, CH, whole><<<dim3(partials, sets), dim3(threads), lds, stream>>>(a);
        };
        bool ok = try_form<1, 1>(f, call) || try_form<1, 2>(f, call) || try_form<2, 2>(f, call) || try_form<2, 3>(f, call) || try_form<4, 2>(f, call) ||
                  try_form<4, 3>(f, call) || try_form<8, 2>(f, call) || try_form<8, 3>(f, call) || try_form<8, 4>(f, call);
        if constexpr (sizeof(T) == 4)
            ok = ok || try_form<3, 1>(f, call);
        else
            ok = ok || try_form<1, 3>(f, call);
        e = ok ? hipGetLastError() : hipErrorInvalidValue;
    }
    if (e == hipSuccess && (a.dw || a.db)) {
        norm_join_kernel<TW><<<dim3((2 * padded(a.channels) + 63) / 64, sets), dim3(1024), 0, stream>>>(a, partials);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int norm_partials(long long groups, long long rows, int channels, int per_group)
{
    // 256 workgroups, one for each CU, or as many as there are rows for; the sets share them.  (With two or four a CU at narrow widths the sums written and read back
    // cost more than the rows gained: 16896 x 1024 36 -> 47 us.)
    const Form f = backward_form(channels, true);  // (at most as many teams a workgroup as for bf16)
    const long long teams = backward_threads(f.team, f.ch) / 64 / f.team, in_set = per_group ? rows : groups * rows, sets = per_group ? groups : 1;
    if (in_set == 0 || sets == 0) return 0;
    return (int)std::min<long long>((in_set + teams - 1) / teams, std::max<long long>(1, 256 / sets));
}

hipError_t launch_norm_forward(const NormArgs& a, int dtype, int weight_dtype, hipStream_t stream)
{
    if (dtype == CLEAR_BF16) return weight_dtype == CLEAR_BF16 ? forward<__bf16, __bf16>(a, stream) : forward<__bf16, float>(a, stream);
    return weight_dtype == CLEAR_BF16 ? forward<float, __bf16>(a, stream) : forward<float, float>(a, stream);
}

hipError_t launch_norm_backward(const NormArgs& a, int dtype, int weight_dtype, hipStream_t stream)
{
    if (dtype == CLEAR_BF16) return weight_dtype == CLEAR_BF16 ? backward<__bf16, __bf16>(a, stream) : backward<__bf16, float>(a, stream);
    return weight_dtype == CLEAR_BF16 ? backward<float, __bf16>(a, stream) : backward<float, float>(a, stream);
}

}  // namespace block
}  // namespace clear
