// clear_block_rotary's rules on where tensors may lie, checked against the elements themselves: over small layouts of every kind, a call that is let through has no
// element that one thread writes and another reads or writes.  The launcher is a stand-in that records that it was reached.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <vector>

#include "../../paper_2412_16112_amd/csrc/block_internal.h"

static int launches = 0;

namespace clear {
namespace block {
hipError_t launch_rotary(const RotaryArgs&, bool, bool, int, hipStream_t)
{
    ++launches;
    return hipSuccess;
}
hipError_t launch_norm_forward(const NormArgs&, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_backward(const NormArgs&, int, int, hipStream_t) { return hipSuccess; }
int norm_partials(long long, long long, int, int) { return 0; }
hipError_t launch_gated_forward(const GatedArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_gated_backward(const GatedArgs&, hipStream_t) { return hipSuccess; }
size_t gated_workspace_bytes(long long, int, int) { return 0; }
hipError_t launch_adamw(int, const clear_block_adamw_tensor*, const AdamHyper&, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_adamw_decode(const void*, const float*, const void*, const float*, float*, float*, long long, hipStream_t) { return hipSuccess; }
}  // namespace block
}  // namespace clear

static unsigned long long state = 88172645463325252ULL;
static unsigned next(unsigned n)
{
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return (unsigned)(state % n);
}

constexpr int kRow = 4;  // channels
struct Tensor {
    long long at;  // first element
    long long st[3];
    int n[3];
};
// Rows of a tensor by number, as the elements they cover.
template <typename F>
static void each_element(const Tensor& t, F f)
{
    for (int b = 0; b < t.n[0]; ++b)
        for (int h = 0; h < t.n[1]; ++h)
            for (int i = 0; i < t.n[2]; ++i)
                for (int c = 0; c < kRow; ++c) f(t.at + b * t.st[0] + h * t.st[1] + i * t.st[2] + c, (b * t.n[1] + h) * t.n[2] + i);
}
// Whether some element of an output is that of another row too, of an input or of an output.  In place a row's element is its own input's.
static bool races(const Tensor& q, const Tensor& qo, const Tensor& k, const Tensor& ko)
{
    std::map<long long, std::vector<int>> written, read;
    const auto put = [](std::map<long long, std::vector<int>>& m, const Tensor& t, int base) { each_element(t, [&](long long at, int row) { m[at].push_back(base + row); }); };
    put(written, qo, 0), put(written, ko, 1000), put(read, q, 0), put(read, k, 1000);
    for (const auto& [at, rows] : written) {
        if (rows.size() > 1) return true;
        const auto r = read.find(at);
        if (r == read.end()) continue;
        for (int row : r->second)
            if (row != rows[0]) return true;
    }
    return false;
}

static int call(const Tensor& q, const Tensor& qo, const Tensor& k, const Tensor& ko)
{
    static const int positions[8] = {};
    static const double freqs[2] = {1, 1};
    const long long ps[3] = {0, 0, 1};
    long long st[12];
    const Tensor* const t[4] = {&q, &qo, &k, &ko};
    for (int i = 0; i < 4; ++i) std::copy(t[i]->st, t[i]->st + 3, st + 3 * i);
    const auto place = [](const Tensor& x) { return (void*)(0x100000000ULL + 2 * (unsigned long long)x.at); };
    const int before = launches;
    const int rc = clear_block_rotary(place(q), place(qo), q.n[1], place(k), place(ko), k.n[1], st, q.n[0], q.n[2], kRow, kRow, 1, positions, 32, ps, 1, freqs, 1.f, 0, CLEAR_BF16, nullptr);
    if ((rc == CLEAR_OK) != (launches > before)) abort();
    return rc;
}
static Tensor plain(long long at, int B, int H, int N) { return {at, {(long long)H * N * kRow, (long long)N * kRow, kRow}, {B, H, N}}; }

#define EXPECT(what)                                       \
    do {                                                   \
        if (!(what)) {                                     \
            printf("line %d: not so: %s\n", __LINE__, #what); \
            return 1;                                      \
        }                                                  \
    } while (0)

int main()
{
    const long long away = 1 << 20;
    // In place with the keys beside the queries in a projection's output [B, N, 3, H, d], [B, N, (Hq + 2 Hk) d], [B, H, N, 3, d], [3, B, H, N, d]; keys first; keys to a tensor of their own.
    const auto fine = [&](const Tensor& q, const Tensor& k) {
        return call(q, q, k, k) == CLEAR_OK && call(k, k, q, q) == CLEAR_OK && call(q, q, k, plain(away, k.n[0], k.n[1], k.n[2])) == CLEAR_OK &&
               call(q, plain(away, q.n[0], q.n[1], q.n[2]), k, k) == CLEAR_OK && !races(q, q, k, k);
    };
    const int B = 2, H = 3, N = 5;
    EXPECT(fine({0, {3 * N * H * kRow, kRow, 3 * H * kRow}, {B, H, N}}, {H * kRow, {3 * N * H * kRow, kRow, 3 * H * kRow}, {B, H, N}}));
    EXPECT(fine({0, {N * 7 * kRow, kRow, 7 * kRow}, {B, 4, N}}, {4 * kRow, {N * 7 * kRow, kRow, 7 * kRow}, {B, 2, N}}));
    EXPECT(fine({0, {3 * H * N * kRow, 3 * N * kRow, 3 * kRow}, {B, H, N}}, {kRow, {3 * H * N * kRow, 3 * N * kRow, 3 * kRow}, {B, H, N}}));
    EXPECT(fine(plain(0, B, H, N), plain(B * H * N * kRow, B, H, N)));
    EXPECT(fine({0, {7 * kRow, kRow, 7 * kRow}, {1, 4, 1}}, {4 * kRow, {99, kRow, 1}, {1, 2, 1}}));  // a single token
    EXPECT(fine({0, {N * 7 * kRow, kRow, 7 * kRow}, {1, 4, N}}, {-2 * kRow, {0, kRow, 7 * kRow}, {1, 2, N}}));
    // Read only, queries and keys may be one tensor.
    EXPECT(call(plain(0, B, H, N), plain(away, B, H, N), plain(0, B, H, N), plain(2 * away, B, H, N)) == CLEAR_OK);
    // One tensor as queries and keys with one of them in place, keys some heads or tokens on.
    const Tensor q = plain(0, B, H, N), other = plain(away, B, H, N), shifted = {N * kRow, {H * N * kRow, N * kRow, kRow}, {B, H - 1, N}};
    EXPECT(call(q, q, q, other) == CLEAR_ERR_INVALID_ARG && call(q, other, q, q) == CLEAR_ERR_INVALID_ARG && call(q, q, q, q) == CLEAR_ERR_INVALID_ARG);
    EXPECT(call(q, q, shifted, shifted) == CLEAR_ERR_INVALID_ARG && call(q, q, shifted, plain(away, B, H - 1, N)) == CLEAR_ERR_INVALID_ARG);
    EXPECT(call(q, other, shifted, shifted) == CLEAR_ERR_INVALID_ARG);
    // Rows of an output on one another.
    const Tensor close = {away, {H * N * kRow, N * kRow, kRow - 1}, {B, H, N}}, folded = {away, {kRow, N * kRow, kRow}, {B, H, N}};
    EXPECT(call(q, close, plain(2 * away, B, H, N), plain(3 * away, B, H, N)) == CLEAR_ERR_INVALID_ARG);
    EXPECT(call(q, folded, plain(2 * away, B, H, N), plain(3 * away, B, H, N)) == CLEAR_ERR_INVALID_ARG);
    EXPECT(call(close, close, q, plain(3 * away, B, H, N)) == CLEAR_ERR_INVALID_ARG);

    int accepted = 0, racing = 0;
    for (int turn = 0; turn < 300000; ++turn) {
        const int n0 = 1 + next(2), n2 = 1 + next(3), hq = 1 + next(3), hk = 1 + next(3);
        const auto stride = [] { return (long long)std::vector<int>{1, 3, 4, 4, 8, 8, 12, 12, 16, 20, 24, 24, 36, 48, 72, 96}[next(16)]; };
        Tensor t[4];
        const long long shared[3] = {stride(), stride(), stride()};
        for (int i = 0; i < 4; ++i) {
            t[i] = {(long long)next(100), {}, {n0, i < 2 ? hq : hk, n2}};
            const bool same = next(8) != 0;
            for (int a = 0; a < 3; ++a) t[i].st[a] = same ? shared[a] : stride();
            if (next(2)) t[i].at += 1000 * i;
        }
        if (next(2)) t[1] = t[0];
        if (next(2)) t[3] = t[2];
        const bool race = races(t[0], t[1], t[2], t[3]);
        racing += race;
        if (call(t[0], t[1], t[2], t[3]) != CLEAR_OK) continue;
        ++accepted;
        if (race) {
            printf("let through with a race: B %d, heads %d and %d, tokens %d\n", n0, hq, hk, n2);
            for (const Tensor& x : t) printf("  at %lld strides %lld %lld %lld\n", x.at, x.st[0], x.st[1], x.st[2]);
            return 1;
        }
    }
    printf("%d calls let through, %d layouts with a race: none of these among them\n", accepted, racing);
    return accepted > 20000 && racing > 20000 ? 0 : 1;
}
