// What lies between two sublayers of a block: r = a x + gate * post(y), h = norm(r) * (offset + w) + b, where post and norm take the size (and for a layer norm the mean) off
// each row; and the backward pass.  Memory-bound: forward x and y are read and r and h written once; backward x, y, dr and dh are read and dx and dy written once, with all sums
// over rows beside.
//
// A team of TEAM waves holds a row, 8 channels a lane, in registers between its statistics and its results; r goes into its norm as it is, in fp32, before it is rounded for
// memory, and the backward pass forms it again from x and y, which it reads in the place of r: as many bytes, and no rounding between the two.
//
// 2 x 4 608 x 2 432 bf16: forward 39 us (4.6 TB/s), backward 52 (5.2), 4.6 for the join of the sums; 16 896 x 4 096 bf16 with an fp32 stream and both norms 162 forward (5.1); 16 717 x 1 111 fp32 with both norms 62 and 91 (4.8 and
// 4.9).  bf16 with an fp32 stream: 2 x 4 608 x 2 432 forward 49 us (5.4), backward with its sums 82 (4.9).  4 096 rows of 8 192: bf16 forward 56 (4.8), backward 92 (4.4), with a norm before too 83 (3.2) and 104 (3.9); with an
// fp32 stream backward 127 (4.7), fp32 166 (4.8).  The widest rows have one team a workgroup, whose loads, barriers and stores follow each other: bf16 of 7 000 channels with both norms, the slowest, 79 forward (2.9) and
// 96 backward (3.6).  Beside the bytes, what counts is instructions: a choice for each element by what is absent (no gate, no post norm), and masks where a row is whole, cost the backward pass 10 to 18 %.
#include <algorithm>
#include <type_traits>

#include "block_rows.h"
#include "block_tiles.h"

namespace clear {
namespace block {
namespace {

constexpr int kSums = 4;  // of the gate, weight, bias, post weight

__host__ __device__ constexpr int forward_waves(int team) { return team >= 3 ? team : 4; }
// As many waves as have the registers: for bf16 128 each, with fp32 among the rows 256 where a team is not wider.
__host__ __device__ constexpr int backward_waves(int team, bool wide) { return wide && team <= 8 ? 8 / team * team : 16 / team * team; }
// Where a wave has 128 registers the sums over rows are in LDS, each lane's own in a place of its own, else in registers.  (12 waves of 168 registers instead: 2 x 4 608 x 2 432 bf16 67 -> 76 us.)
__host__ __device__ constexpr bool sums_in_lds(int team, bool wide) { return backward_waves(team, wide) > 8; }

// Both rows of a type lie in eights a lane, but fp32 alone in fours, so that neighbouring lanes load neighbouring 16 bytes.
template <typename T, typename TS, int TEAM>
using RowLayout = Layout<std::conditional_t<sizeof(T) == 4 && sizeof(TS) == 4, float, __bf16>, TEAM, 1, false>;

// A lane's part of a vector, or 1 where there is none (the formulas need no branches then).
template <int GAP, typename TW>
__device__ __forceinline__ void load_or_ones(Chunk8<TW>& to, const TW* p, int n, RowForm form)
{
    if (p) to.template load<GAP>(p, n, form);
    else to.fill(1.f);
}
// Whether every lane of this wave has 8 channels (a branch that the whole wave takes).
template <typename L>
__device__ __forceinline__ bool whole_wave(int lane, int channels)
{
    const int last = lane | 63, n = channels - L::first(last, 0);
    return __builtin_amdgcn_readfirstlane(n >= L::P::first(4) + (L::GAP == 4 ? 8 : 4));
}
template <typename TW>
__device__ __forceinline__ const TW* vector_of(const void* p, int set, int channels) { return p ? (const TW*)p + (long long)set * channels : nullptr; }

template <typename T, typename TS, typename TW, bool POST, int TEAM>
__global__ void __launch_bounds__(64 * forward_waves(TEAM)) residual_forward_kernel(ResidualArgs a, long long row_first)
{
    constexpr int WAVES = forward_waves(TEAM), TEAMS = WAVES / TEAM;
    typedef RowLayout<T, TS, TEAM> L;
    __shared__ float slots[2][WAVES][1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x % (64 * TEAM);
    const long long total = (long long)a.groups * a.rows;
    const long long row = row_first + (long long)blockIdx.x * TEAMS + wave / TEAM;
    const bool live = row < total;
    const int at = live ? (int)row : 0;
    const int g = at / a.rows, r = at - g * a.rows;
    const int C = a.channels, c = L::first(lane, 0), n = C - c;
    const RowForm form = L::form(C, 0);
    Chunk8<TS> vx;
    Chunk8<T> vy;
    vy.template load<L::GAP>((const T*)a.y + g * a.st[2] + r * a.st[3] + c, n, form);
    vx.template load<L::GAP>((const TS*)a.x + g * a.st[0] + r * a.st[1] + c, n, form);
    Chunk8<TW> cg, cp, cw, cb;  // (asked for here: they arrive while the sums are formed)
    const TW* const w = vector_of<TW>(a.w, a.per_group ? g : 0, C);
    const TW* const b = vector_of<TW>(a.b, a.per_group ? g : 0, C);
    const TW* const gate = vector_of<TW>(a.gate, a.gate_per_group ? g : 0, C);
    const float offset = w ? a.offset : 0.f, post_offset = a.pw ? a.post_offset : 0.f;
    if (POST) load_or_ones<L::GAP>(cp, a.pw ? (const TW*)a.pw + c : nullptr, n, form);
    load_or_ones<L::GAP>(cg, gate ? gate + c : nullptr, n, form);
    load_or_ones<L::GAP>(cw, w ? w + c : nullptr, n, form);
    if (b) cb.template load<L::GAP>(b + c, n, form);
    else cb.fill(0.f);
    const bool all = whole_wave<L>(lane, C);
    int turn = 0;
    auto sum = [&](auto value) {  // of value(j) over the row's channels
        float s[1] = {0.f};
        if (all) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += value(j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += L::P::own(j, n, form) ? value(j) : 0.f;
        }
        team_sum<TEAM>(s, slots[turn], wave);
        turn ^= 1;
        return s[0];
    };
    // Mean (0 where it stays) and 1 / size of a row; the squares are those of the differences from the mean.
    auto size_of_row = [&](const float (&v)[8], int kind, float* mean, float* rstd) {
        *mean = kind == CLEAR_NORM_LAYER ? sum([&](int j) { return v[j]; }) / (float)C : 0.f;
        const float m = *mean;
        *rstd = 1.0f / sqrtf(sum([&](int j) { return (v[j] - m) * (v[j] - m); }) / (float)C + a.eps);
    };
    float v[8], mean_y = 0.f, rstd_y = 1.f, mean, rstd;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = vy.get(j);
    if (POST) {
        size_of_row(v, a.post, &mean_y, &rstd_y);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (v[j] - mean_y) * rstd_y * (post_offset + cp.get(j));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = a.scale * vx.get(j) + cg.get(j) * v[j];
    size_of_row(v, a.kind, &mean, &rstd);
    if (!live) return;
    if (a.stats && lane == 0) {
        a.stats[row] = mean;
        a.stats[total + row] = rstd;
        if (POST) {
            a.stats[2 * total + row] = mean_y;
            a.stats[3 * total + row] = rstd_y;
        }
    }
    if (c >= C) return;
    // (r and h may lie on x and y: what the team's waves read of these has arrived before the sum over r)
    Chunk8<TS>::template store<L::GAP>((TS*)a.r + g * a.st[4] + r * a.st[5] + c, n, form, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (v[j] - mean) * rstd * (offset + cw.get(j)) + cb.get(j);
    Chunk8<T>::template store<L::GAP>((T*)a.h + g * a.st[6] + r * a.st[7] + c, n, form, v);
}

// Workgroup (p, set) of the grid takes rows p TEAMS + team, then every gridDim.x TEAMS further ones, of the set (a group where anything is a group's own, else everything),
// writes their dx and dy and adds up in registers what the vectors' gradients are sums of; the teams' sums are added in order and become partial p of the set.
//     d = dr + norm'(dh (offset + w)),   dx = a d,   dz = gate d,   dy = post'(dz (post_offset + post weight))
template <typename T, typename TS, typename TW, bool POST, int TEAM>
__global__ void __launch_bounds__(64 * backward_waves(TEAM, sizeof(T) + sizeof(TS) > 4)) residual_backward_kernel(ResidualArgs a)
{
    constexpr bool WIDE = sizeof(T) + sizeof(TS) > 4;
    constexpr int WAVES = backward_waves(TEAM, WIDE), TEAMS = WAVES / TEAM;
    typedef RowLayout<T, TS, TEAM> L;
    constexpr bool IN_LDS = sums_in_lds(TEAM, WIDE);
    extern __shared__ __attribute__((aligned(16))) float lds[];  // the lanes' sums; in the end [padded channels] where a workgroup has several teams
    __shared__ float slots[2][WAVES][2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x % (64 * TEAM), team = wave / TEAM;
    const int C = a.channels, set = blockIdx.y, c = L::first(lane, 0), n = C - c;
    const RowForm form = L::form(C, 0);
    const bool sets = a.per_group || a.gate_per_group;
    const long long in_set = sets ? a.rows : (long long)a.groups * a.rows;
    const long long first = sets ? (long long)set * a.rows : 0;
    const long long total = (long long)a.groups * a.rows;
    const bool layer = a.kind == CLEAR_NORM_LAYER, post_layer = a.post == CLEAR_NORM_LAYER;
    const float inv_c = 1.f / (float)C;
    Chunk8<TW> cg, cp, cw;
    const TW* const w = vector_of<TW>(a.w, a.per_group ? set : 0, C);
    const TW* const gate = vector_of<TW>(a.gate, a.gate_per_group ? set : 0, C);
    const float offset = w ? a.offset : 0.f, post_offset = a.pw ? a.post_offset : 0.f;
    load_or_ones<L::GAP>(cw, w ? w + c : nullptr, n, form);
    load_or_ones<L::GAP>(cg, gate ? gate + c : nullptr, n, form);
    if (POST) load_or_ones<L::GAP>(cp, a.pw ? (const TW*)a.pw + c : nullptr, n, form);
    const shared_float sum = (shared_float)lds;  // (LDS by a pointer of its own address space: as in the layer norm's backward pass)
    float sums[IN_LDS ? 1 : kSums][8];
    // Sum k, which is wanted where `wanted` is not null, and v more.
    auto lane_sum = [&](int k, int h) { return (shared_f32x4)sum + (2 * k + h) * (64 * WAVES) + threadIdx.x; };
    auto add = [&](auto k, const void* wanted, const float (&v)[8]) {
        if (!wanted) return;
        if constexpr (IN_LDS) {
#pragma unroll
            for (int h = 0; h < 2; ++h) *lane_sum(k, h) += f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[k][j] += v[j];
        }
    };
    constexpr std::integral_constant<int, 0> SUM_GATE{};
    constexpr std::integral_constant<int, 1> SUM_WEIGHT{};
    constexpr std::integral_constant<int, 2> SUM_BIAS{};
    constexpr std::integral_constant<int, 3> SUM_POST{};
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if constexpr (IN_LDS) {
            *lane_sum(k, 0) = *lane_sum(k, 1) = f32x4{0.f, 0.f, 0.f, 0.f};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[k][j] = 0.f;
        }
    }
    const long long step = (long long)gridDim.x * TEAMS;
    struct Row {
        Chunk8<TS> x, dr;
        Chunk8<T> y, dh;
        float mean, rstd, mean_y, rstd_y;
        int g, r;
        bool live;
    };
    // (Where the tensors lie is read from the kernel's arguments again for every row: kept, it would take more scalar registers than there are.)
    typedef const __attribute__((address_space(4))) ResidualArgs* args_ptr;
    auto args_anew = [] {
        args_ptr p = (args_ptr)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(p));
        return p;
    };
    auto fetch = [&](long long base, Row* to) {  // (a row that is not there: the set's first, with gradients of 0)
        const args_ptr q = args_anew();
        to->live = base + team < in_set;
        const long long row = first + (to->live ? base + team : 0);
        const int g = (int)row / q->rows, r = (int)row - g * q->rows;
        to->g = g, to->r = r;
        to->mean = q->stats[row];
        to->rstd = q->stats[total + row];
        if (POST) {
            to->mean_y = q->stats[2 * total + row];
            to->rstd_y = q->stats[3 * total + row];
        }
        const int m = to->live ? n : 0;
        const RowForm f = to->live ? form : RowForm{false, false};
        to->x.template load<L::GAP>((const TS*)q->x + g * q->st[4] + r * q->st[5] + c, n, form);
        to->y.template load<L::GAP>((const T*)q->y + g * q->st[6] + r * q->st[7] + c, n, form);
        to->dh.template load<L::GAP>((const T*)q->dh + g * q->st[2] + r * q->st[3] + c, m, f);
        to->dr.template load<L::GAP>((const TS*)q->dr + g * q->st[0] + r * q->st[1] + c, q->dr ? m : 0, q->dr ? f : RowForm{false, false});
    };
    constexpr bool AHEAD = WIDE ? !IN_LDS : TEAM < 16;  // the next row's loads are under way while a row is worked on, where there are registers for it
    Row now, next;
    if (AHEAD) fetch((long long)blockIdx.x * TEAMS, &next);
    int turn = 0;
    for (long long base = (long long)blockIdx.x * TEAMS; base < in_set; base += step) {  // (the same number of turns for every wave)
        if (!AHEAD) fetch(base, &now);
        __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);  // vmcnt 0: here and not behind the next row's loads, and before anything is written: dx and dy may lie on dr and dh
        if (AHEAD) {
            now = next;
            if (base + step < in_set) fetch(base + step, &next);
        }
        now.dh.template clear_others<L::GAP>(n, form);
        const float mean = now.mean, rstd = now.rstd, mean_y = now.mean_y, rstd_y = now.rstd_y;
        const bool live = now.live;
        // of element j: the sublayer's output in its unit form, as it goes to the gate, and the sum in its unit form
        auto unit_y = [&](int j) { return (now.y.get(j) - mean_y) * rstd_y; };
        auto post_w = [&](int j) { return post_offset + cp.get(j); };
        auto out_y = [&](int j) { return POST ? unit_y(j) * post_w(j) : now.y.get(j); };
        auto unit = [&](int j) { return (a.scale * now.x.get(j) + cg.get(j) * out_y(j) - mean) * rstd; };
        auto grad = [&](int j) { return now.dh.get(j) * (offset + cw.get(j)); };
        float s[2] = {0.f, 0.f}, h[8], v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h[j] = unit(j);
            const float dyw = grad(j);
            s[0] += dyw;
            s[1] += dyw * h[j];
        }
        if (live) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = now.dh.get(j) * h[j];
            add(SUM_WEIGHT, a.dw, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = now.dh.get(j);
            add(SUM_BIAS, a.db, v);
        }
        if (!a.rows_out) continue;  // (weight and bias alone)
        team_sum<TEAM>(s, slots[turn], wave);
        turn ^= 1;
        const float s0 = layer ? s[0] * inv_c : 0.f, s1 = s[1] * inv_c;
        float d[8], t[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            d[j] = now.dr.get(j) + rstd * (grad(j) - s0 - h[j] * s1);
            v[j] = d[j] * out_y(j);
            h[j] = d[j] * cg.get(j);  // dz
            d[j] *= a.scale;
        }
        if (live) add(SUM_GATE, a.dgate, v);
        const args_ptr q = args_anew();
        if (live && c < C && q->dx) Chunk8<TS>::template store<L::GAP>((TS*)q->dx + now.g * q->st[8] + now.r * q->st[9] + c, n, form, d);
        if (POST) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float u = unit_y(j), dz = L::P::own(j, n, form) ? h[j] : 0.f;
                v[j] = dz * u;
                h[j] = dz * post_w(j);
                t[0] += h[j];
                t[1] += h[j] * u;
            }
            if (live) add(SUM_POST, a.dpw, v);
            team_sum<TEAM>(t, slots[turn], wave);
            turn ^= 1;
            const float t0 = post_layer ? t[0] * inv_c : 0.f, t1 = t[1] * inv_c;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = rstd_y * (h[j] - t0 - unit_y(j) * t1);
        }
        if (live && c < C && q->dy) Chunk8<T>::template store<L::GAP>((T*)q->dy + now.g * q->st[10] + now.r * q->st[11] + c, n, form, h);
    }
    const int wide = padded(C);
    float* out = a.ws + ((long long)set * gridDim.x + blockIdx.x) * a.sums * wide;
    auto give = [&](auto to, const float (&v)[8], bool more) {
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const int at = c + L::P::first(h) + L::P::in(h);
            if (L::P::back(h, n) == 0) {
                f32x4 x = {v[h], v[h + 1], v[h + 2], v[h + 3]};
                if (more) x += *(shared_f32x4)(sum + at);
                put_four(to + at, x);
            } else {
#pragma unroll
                for (int j = h; j < h + 4; ++j) {
                    if (!L::P::own(j, n, form)) continue;
                    const int k = c + L::P::at(j, n, form);
                    to[k] = more ? v[j] + sum[k] : v[j];
                }
            }
        }
    };
    float mine[kSums][8];
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if constexpr (IN_LDS) {
            const f32x4 lo = *lane_sum(k, 0), hi = *lane_sum(k, 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) mine[k][j] = lo[j], mine[k][4 + j] = hi[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[k][j] = sums[k][j];
        }
    }
    if (IN_LDS && TEAMS > 1) __syncthreads();  // (LDS is the teams' from here on)
    auto give_sum = [&](const void* wanted, const float (&v)[8]) {
        if (!wanted) return;
        for (int t = 0; t < TEAMS; ++t) {
            if (team == t) {
                if (t + 1 < TEAMS)
                    give(sum, v, t > 0);
                else
                    give(out, v, t > 0);
            }
            __syncthreads();
        }
        out += wide;
    };
    give_sum(a.dgate, mine[SUM_GATE]);
    give_sum(a.dw, mine[SUM_WEIGHT]);
    give_sum(a.db, mine[SUM_BIAS]);
    give_sum(a.dpw, mine[SUM_POST]);
}

struct Joined {
    void* to[kSums];
    int own[kSums];  // a set each; else one of all sets
};
// A vector's gradient from the partials: workgroup (i, set, k) takes 64 columns of sum k, its wave w the partials w, w + 16, ...
template <typename TW>
__global__ void __launch_bounds__(1024) residual_join_kernel(const float* ws, Joined out, int channels, int partials, int sets)
{
    __shared__ float part[16][64];
    const int k = blockIdx.z, set = blockIdx.y;
    if (!out.own[k] && set > 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wide = padded(channels), col = blockIdx.x * 64 + lane;
    const long long stride = (long long)gridDim.z * wide, count = out.own[k] ? partials : (long long)partials * sets;
    const float* const from = ws + (long long)set * partials * stride + (long long)k * wide + col;
    float s = 0.f;
    if (col < wide) {
        long long p = wave;
        for (; p + 48 < count; p += 64) {  // (four loads in flight)
            const float x0 = from[p * stride], x1 = from[(p + 16) * stride], x2 = from[(p + 32) * stride], x3 = from[(p + 48) * stride];
            s += (x0 + x1) + (x2 + x3);
        }
        for (; p < count; p += 16) s += from[p * stride];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += part[i][lane];
        if (col < channels) ((TW*)out.to[k])[(long long)set * channels + col] = (TW)s;
    }
}

int team_of(int channels)
{
    const int need = (channels + 511) / 512;
    for (int team : {1, 2, 3, 4, 5, 6, 8, 12})
        if (need <= team) return team;
    return 16;
}

// call(team) with the team as an integral constant.
template <typename F>
void with_team(int team, F&& call)
{
    switch (team) {
    case 1: return call(std::integral_constant<int, 1>{});
    case 2: return call(std::integral_constant<int, 2>{});
    case 3: return call(std::integral_constant<int, 3>{});
    case 4: return call(std::integral_constant<int, 4>{});
    case 5: return call(std::integral_constant<int, 5>{});
    case 6: return call(std::integral_constant<int, 6>{});
    case 8: return call(std::integral_constant<int, 8>{});
    case 12: return call(std::integral_constant<int, 12>{});
    default: return call(std::integral_constant<int, 16>{});
    }
}

template <typename T, typename TS, typename TW, bool POST>
hipError_t forward(const ResidualArgs& a, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    with_team(team_of(a.channels), [&](auto team) {
        constexpr int TEAM = team, threads = 64 * forward_waves(TEAM), teams = forward_waves(TEAM) / TEAM;
        constexpr long long most = 0xffffffffLL / threads;  // workgroups a launch can have
        const long long rows = (long long)a.groups * a.rows;
        for (long long first = 0; first < rows && e == hipSuccess; first += most * teams) {
            const long long blocks = std::min(most, (rows - first + teams - 1) / teams);
            residual_forward_kernel<T, TS, TW, POST, TEAM><<<dim3((unsigned)blocks), dim3(threads), 0, stream>>>(a, first);
            e = hipGetLastError();
        }
    });
    return e;
}

template <typename T, typename TS, typename TW, bool POST>
hipError_t backward(ResidualArgs a, hipStream_t stream)
{
    const int sets = a.per_group || a.gate_per_group ? a.groups : 1;
    const int partials = residual_partials(a.groups, a.rows, a.channels, sets);
    Joined out = {};
    a.sums = 0;
    auto add = [&](void* to, int own) {
        if (!to) return;
        out.to[a.sums] = to;
        out.own[a.sums++] = own && sets > 1;
    };
    add(a.dgate, a.gate_per_group);
    add(a.dw, a.per_group);
    add(a.db, a.per_group);
    add(a.dpw, 0);
    a.rows_out = a.dx || a.dy || a.dgate || a.dpw;
    hipError_t e = hipSuccess;
    if (partials > 0) {
        with_team(team_of(a.channels), [&](auto team) {
            constexpr bool WIDE = sizeof(T) + sizeof(TS) > 4;
            constexpr int TEAM = team, waves = backward_waves(TEAM, WIDE);
            size_t lds = waves / TEAM > 1 && a.sums ? (size_t)padded(a.channels) * 4 : 0;  // (at most 16 KB)
            if constexpr (sums_in_lds(TEAM, WIDE)) {
                constexpr size_t all = 64 * waves * kSums * 32;  // (at most 128 KB)
                static LdsLimit limit;
                e = limit.ensure((const void*)residual_backward_kernel<T, TS, TW, POST, TEAM>, all);
                if (e != hipSuccess) return;
                lds = all;
            }
            residual_backward_kernel<T, TS, TW, POST, TEAM><<<dim3(partials, sets), dim3(64 * waves), lds, stream>>>(a);
            e = hipGetLastError();
        });
    }
    if (e == hipSuccess && a.sums) {
        residual_join_kernel<TW><<<dim3((padded(a.channels) + 63) / 64, sets, a.sums), dim3(1024), 0, stream>>>(a.ws, out, a.channels, partials, sets);
        e = hipGetLastError();
    }
    return e;
}

// f(a value of T, of TS, of TW): of the output's, the stream's and the vectors' types.
template <typename F>
hipError_t with_types(int dtype, int stream_dtype, int weight_dtype, F&& f)
{
    const __bf16 h = (__bf16)0.f;
    if (dtype == CLEAR_BF16 && stream_dtype == CLEAR_BF16) return weight_dtype == CLEAR_BF16 ? f(h, h, h) : f(h, h, 0.f);
    if (dtype == CLEAR_BF16) return weight_dtype == CLEAR_BF16 ? f(h, 0.f, h) : f(h, 0.f, 0.f);
    return weight_dtype == CLEAR_BF16 ? f(0.f, 0.f, h) : f(0.f, 0.f, 0.f);
}

}  // namespace

int residual_partials(long long groups, long long rows, int channels, long long sets)
{
    // 256 workgroups, one for each CU, or as many as there are rows for in bf16; the sets share them, rounded down.  (The workspace is asked for without a type.  With fp32 among the rows a workgroup has fewer teams, which
    // take several rows one after the other where all would fit at once: 77 fp32 rows of 2 432 channels are 26 workgroups of three rows each.)
    const int team = team_of(channels);
    const long long teams = backward_waves(team, false) / team, in_set = sets > 1 || groups == 1 ? rows : groups * rows;
    if (in_set == 0 || sets == 0) return 0;
    return (int)std::min<long long>((in_set + teams - 1) / teams, std::max<long long>(1, 256 / sets));
}

hipError_t launch_residual_forward(const ResidualArgs& a, int dtype, int stream_dtype, int weight_dtype, hipStream_t stream)
{
    return with_types(dtype, stream_dtype, weight_dtype, [&](auto t, auto ts, auto tw) { return a.post ? forward<decltype(t), decltype(ts), decltype(tw), true>(a, stream) : forward<decltype(t), decltype(ts), decltype(tw), false>(a, stream); });
}

hipError_t launch_residual_backward(const ResidualArgs& a, int dtype, int stream_dtype, int weight_dtype, hipStream_t stream)
{
    return with_types(dtype, stream_dtype, weight_dtype, [&](auto t, auto ts, auto tw) { return a.post ? backward<decltype(t), decltype(ts), decltype(tw), true>(a, stream) : backward<decltype(t), decltype(ts), decltype(tw), false>(a, stream); });
}

}  // namespace block
}  // namespace clear
