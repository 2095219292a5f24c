// Sampling distinct hosts from a policy's logits with given random numbers (nbos_policy_sample).
//
// Weights are whole numbers, w = floor(2^31 * 2^((x - m) c)), c = log2(e) / T: every sum of them is exact, so the
// split of a row over lanes, warps and blocks cannot change which host a random number selects. top-k, top-p and
// min-p each keep a first part of the order (x descending, index ascending); the draw runs in index order over what
// is left, so nothing has to be sorted: top-k finds its last value by bisection on counts, top-p on exact sums.
// A team of warps shares a row: one warp up to 1,024 hosts, a block up to 32,768, a cluster of up to 8 blocks up to
// 262,144. Each lane holds 32 elements in registers, as logits until the top-k cut is known and as weights from
// then on, so the logits are read once. Longer rows keep their elements in the workspace instead.
// A warp's columns are one stretch of the row and a lane's 16 bytes of it are neighbours, so index order is
// warp, then 16-byte chunk, then lane.
#include <math.h>

#include "nbos_policy.cuh"

namespace nbos {
namespace {

using namespace policy;

constexpr int kElems = 32;
constexpr int kMaxCluster = 8;
constexpr int kBlockRow = 1024 * kElems;
typedef unsigned long long u64;

struct SampleArgs {
    const void *x;
    long long rows, stride;
    int n, draws, aligned;
    const float *u, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *hosts, *found;
    unsigned int *store;   // rows longer than the registers of a cluster: [clusters][n]
};

// floats in the order of unsigned integers
__device__ __forceinline__ unsigned int key_of(float x)
{
    const unsigned int b = __float_as_uint(x);
    return b ^ ((unsigned int)((int)b >> 31) | 0x80000000u);
}

__device__ __forceinline__ float float_of(unsigned int key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// +inf counts as the largest finite float
constexpr float kMaxFinite = 3.402823466e38f;

// floor(2^31 * 2^((x - m) scale)): difference and product are rounded one by one (no contraction). The power is at
// most 1, so its significand shifted by its exponent is the whole number; below 2^-31 nothing is left.
__device__ __forceinline__ unsigned int weight_of(float x, float m, float scale)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(__fsub_rn(x, m), scale)));
    const unsigned int b = __float_as_uint(e), shift = 127u - (b >> 23);
    const unsigned int w = (b << 8) | 0x80000000u;
    return shift < 32u ? w >> shift : 0u;
}

// sum += w + 2^44 if w > t: a sum of weights with their number above it, in three instructions
__device__ __forceinline__ void add_above(unsigned int &lo, unsigned int &hi, unsigned int w, unsigned int t)
{
    asm("{\n\t.reg .pred p;\n\t"
        "setp.gt.u32 p, %2, %3;\n\t"
        "@p add.cc.u32 %0, %0, %2;\n\t"
        "@p addc.u32 %1, %1, 4096;\n\t}"
        : "+r"(lo), "+r"(hi)
        : "r"(w), "r"(t));
}

// sum over the warp of values below 2^52, by two 26-bit halves
__device__ __forceinline__ u64 warp_sum(u64 v)
{
    const unsigned int lo = __reduce_add_sync(kFull, (unsigned int)v & 0x3FFFFFFu);
    const unsigned int hi = __reduce_add_sync(kFull, (unsigned int)(v >> 26));
    return ((u64)hi << 26) + lo;
}
__device__ __forceinline__ u64 warp_scan(u64 v, int lane)   // inclusive
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const u64 other = __shfl_up_sync(kFull, v, off);
        if (lane >= off) v += other;
    }
    return v;
}

__device__ __forceinline__ unsigned int warp_scan32(unsigned int v, int lane)
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const unsigned int other = __shfl_up_sync(kFull, v, off);
        if (lane >= off) v += other;
    }
    return v;
}

// floor(total * steps / 2^24); total below 2^52, steps at most 2^24
__device__ __forceinline__ u64 share_of(u64 total, unsigned int steps)
{
    return (u64)steps * (total >> 24) + (((u64)steps * (total & 0xFFFFFFu)) >> 24);
}

// The warps that share a row. MULTI = false: one warp, no shared memory.
template <bool MULTI>
struct Team {
    ulonglong2 (*slots)[kMaxCluster * 32];   // two sets, taken in turn
    int warps, cs, me, lane, turn;           // me: this warp's place among all of the row

    // every warp's (a, b), which the lanes of a warp agree on, to every warp, in slots[result]
    __device__ __forceinline__ int exchange(u64 a, u64 b)
    {
        const int now = turn;
        if (lane < cs) cluster_peer(slots[now], lane, cs)[me] = make_ulonglong2(a, b);
        cluster_sync(cs);
        turn ^= 1;
        return now;
    }
    __device__ __forceinline__ void sum2(u64 &a, u64 &b)
    {
        a = warp_sum(a), b = warp_sum(b);
        if (!MULTI) return;
        const int now = exchange(a, b);
        a = 0, b = 0;
        for (int i = lane; i < warps; i += 32) a += slots[now][i].x, b += slots[now][i].y;
        a = warp_sum(a), b = warp_sum(b);
    }
    // a lane's sum of at most 32 weights with their number above bit 44, as one value: mass and number over the row
    __device__ __forceinline__ void sum_packed(u64 v, u64 &mass, u64 &number)
    {
        const unsigned int lo = __reduce_add_sync(kFull, (unsigned int)v & 0x3FFFFFFu);
        const unsigned int hi = __reduce_add_sync(kFull, (unsigned int)(v >> 26) & 0x3FFFFu);
        mass = ((u64)hi << 26) + lo;
        number = __reduce_add_sync(kFull, (unsigned int)(v >> 44));
        if (!MULTI) return;
        const int now = exchange(mass, number);
        u64 a = 0;
        unsigned int b = 0;
        for (int i = lane; i < warps; i += 32) a += slots[now][i].x, b += (unsigned int)slots[now][i].y;
        mass = warp_sum(a), number = __reduce_add_sync(kFull, b);
    }
    __device__ __forceinline__ unsigned int count(unsigned int v)
    {
        v = __reduce_add_sync(kFull, v);
        if (!MULTI) return v;
        const int now = exchange(v, 0);
        v = 0;
        for (int i = lane; i < warps; i += 32) v += (unsigned int)slots[now][i].x;
        return __reduce_add_sync(kFull, v);
    }
    __device__ __forceinline__ float max(float v)
    {
        v = lanes_max(v, 32);
        if (!MULTI) return v;
        const int now = exchange(__float_as_uint(v), 0);
        v = neg_inf();
        for (int i = lane; i < warps; i += 32) v = fmaxf(v, __uint_as_float((unsigned int)slots[now][i].x));
        return lanes_max(v, 32);
    }
    __device__ __forceinline__ unsigned int max_key(unsigned int v)
    {
        v = __reduce_max_sync(kFull, v);
        if (!MULTI) return v;
        const int now = exchange(v, 0);
        v = 0;
        for (int i = lane; i < warps; i += 32) v = ::max(v, (unsigned int)slots[now][i].x);
        return __reduce_max_sync(kFull, v);
    }
    // sums of `mine`, which the lanes of a warp agree on: over the warps before this one, and over all
    __device__ __forceinline__ void prefix(u64 mine, u64 &before, u64 &all)
    {
        before = 0, all = mine;
        if (!MULTI) return;
        const int now = exchange(mine, 0);
        u64 b = 0, a = 0;
        for (int i = lane; i < warps; i += 32) {
            const u64 v = slots[now][i].x;
            a += v;
            if (i < me) b += v;
        }
        before = warp_sum(b), all = warp_sum(a);
    }
    // the warp that has something (has: agreed in the warp) tells all
    __device__ __forceinline__ void tell(bool has, u64 &a, u64 &b)
    {
        if (!MULTI) return;
        const int now = turn;
        if (has && lane < cs) cluster_peer(slots[now], lane, cs)[0] = make_ulonglong2(a, b);
        cluster_sync(cs);
        turn ^= 1;
        a = slots[now][0].x, b = slots[now][0].y;
    }
};

// A lane's elements: registers (REGS), or the workspace for rows that do not fit. Chunk c of the lane covers the
// columns base + c * 32 * VEC + 0 .. VEC - 1.
template <int VEC_, int CH_, bool REGS_>
struct Elems {
    static constexpr int VEC = VEC_, CH = CH_;
    static constexpr bool REGS = REGS_;
    unsigned int r[REGS ? CH * VEC : 1];
    unsigned int *store;
    int chunks;
    int base, n;   // first column of the lane's chunk 0; columns of the row
    template <typename F>
    __device__ __forceinline__ void each(F f)   // f(value &, column)
    {
        if constexpr (REGS) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) f(r[c * VEC + i], base + c * 32 * VEC + i);
        } else {
            for (int c = 0; c < chunks; ++c)
                for (int i = 0; i < VEC; ++i) {
                    const int col = base + c * 32 * VEC + i;
                    if (col >= n) return;
                    unsigned int v = store[col];
                    f(v, col);
                    store[col] = v;
                }
        }
    }
    // the sum of value(element, column) over the lane's part of chunk c
    template <typename F>
    __device__ __forceinline__ u64 chunk_sum(int c, F value)
    {
        u64 s = 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int col = base + c * 32 * VEC + i;
            if constexpr (REGS)
                s += value(r[c * VEC + i], col);
            else
                s += col < n ? value(store[col], col) : 0;
        }
        return s;
    }
    // The first column, in index order over the warp, at which the running sum of value(element, column) from `from`
    // exceeds t, and the value there; the warp must hold it. sum_of(c): the lane's sum over chunk c.
    template <typename S, typename F>
    __device__ __forceinline__ void find(u64 t, u64 from, int lane, S sum_of, F value, int &col_out, u64 &val_out)
    {
        u64 run = from, s_found = 0, run_found = 0;
        int c_found = -1;
        auto step = [&](int c) {
            if (c_found >= 0) return;
            const u64 s = sum_of(c), total = warp_sum(s);
            if (t < run + total) c_found = c, s_found = s, run_found = run;
            run += total;
        };
        if constexpr (REGS) {
#pragma unroll
            for (int c = 0; c < CH; ++c) step(c);
        } else {
            for (int c = 0; c < chunks; ++c) step(c);
        }
        const u64 upto = run_found + warp_scan(s_found, lane);
        const int owner = __ffs(__ballot_sync(kFull, t < upto)) - 1;
        u64 acc = upto - s_found, val = 0;
        int col = -1;
        const int first = base + c_found * 32 * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            u64 v = 0;
            if constexpr (REGS) {
                unsigned int raw = r[i];
#pragma unroll
                for (int c = 1; c < CH; ++c) raw = c == c_found ? r[c * VEC + i] : raw;
                v = value(raw, first + i);
            } else if (c_found >= 0 && first + i < n) {
                v = value(store[first + i], first + i);
            }
            acc += v;
            if (col < 0 && t < acc) col = first + i, val = v;
        }
        col_out = __shfl_sync(kFull, col, owner);
        val_out = __shfl_sync(kFull, val, owner);
    }
};

// The column of the m-th (from 0) element, in index order over the row, that `pick` accepts.
template <bool MULTI, typename E, typename F>
__device__ __forceinline__ int nth_column(Team<MULTI> &team, E &e, u64 m, F pick)
{
    auto one = [&](unsigned int v, int col) -> u64 { return pick(v, col) ? 1 : 0; };
    unsigned int here = 0;
    e.each([&](unsigned int &v, int col) { here += pick(v, col) ? 1u : 0u; });
    const u64 mine = __reduce_add_sync(kFull, here);
    u64 before, all;
    team.prefix(mine, before, all);
    int col = -1;
    u64 val = 0;
    const bool has = m >= before && m < before + mine;
    if (has) e.find(m, before, team.lane, [&](int c) { return e.chunk_sum(c, one); }, one, col, val);
    u64 where = (u64)(unsigned int)col;
    team.tell(has, where, val);
    return (int)(unsigned int)where;
}

struct Row {
    float m, scale, top_p, min_p;
    int k;          // 0: off
    bool greedy, none;
};

constexpr int kSort = 64;   // weights that one warp sorts, two a lane

// descending over (a of lane 0 .. 31, b of lane 0 .. 31), a bitonic network
__device__ __forceinline__ void sort64(unsigned int &a, unsigned int &b, int lane)
{
#pragma unroll
    for (int k = 2; k <= 64; k *= 2)
#pragma unroll
        for (int j = k / 2; j > 0; j /= 2) {
            if (j == 32) {
                const unsigned int hi = max(a, b), lo = min(a, b);
                a = hi, b = lo;
            } else {
                const unsigned int oa = __shfl_xor_sync(kFull, a, j), ob = __shfl_xor_sync(kFull, b, j);
                const bool first = (lane & j) == 0;
                const bool max_a = ((lane & k) == 0) == first;                 // elements lane and lane + 32
                const bool max_b = (((lane + 32) & k) == 0) == first;
                a = max_a ? max(a, oa) : min(a, oa);
                b = max_b ? max(b, ob) : min(b, ob);
            }
        }
}

// The weight at which the running sum of weights, in descending order, reaches `limit`; the sum of those above it and
// how many have just it. Bisection (on the logarithm at first, with the bounds moved onto weights that
// occur every few steps) until at most 64 weights are left between the bounds, which one warp then sorts.
template <bool MULTI, typename E>
__device__ __forceinline__ void nucleus(Team<MULTI> &team, E &e, u64 limit, u64 total, u64 count, unsigned int *sort_list,
                                        unsigned int &cut, u64 &mass_above, u64 &ties)
{
    // invariant: mass(w > hi) < limit <= mass(w > lo)
    unsigned int lo = 0, hi = 0x80000000u;
    u64 mass_hi = 0, count_hi = 0, count_lo = count;
    // Weights below (total - limit) / n together hold less than what may be left out: the cut lies above them.
    const u64 least = (total - limit) / (unsigned int)e.n;
    for (int it = 0; hi - lo > 1 && count_lo - count_hi > kSort; ++it) {
        if ((it & 3) == 3) {
            unsigned int most = 0, least_in = 0xFFFFFFFFu;
            e.each([&](unsigned int &v, int) {
                if (v <= hi) most = max(most, v);
                if (v > lo) least_in = min(least_in, v);
            });
            hi = team.max_key(most), lo = ~team.max_key(~least_in) - 1;
            if (hi - lo <= 1) break;
        }
        unsigned int mid = __float2uint_rd(__uint_as_float((__float_as_uint(__uint2float_rn(lo ? lo : 1)) + __float_as_uint(__uint2float_rn(hi))) / 2));
        if (it == 0 && least > 1) mid = (unsigned int)least - 1;
        if (mid <= lo || mid >= hi) mid = lo + (hi - lo) / 2;
        u64 mass = 0, c = 0;
        if constexpr (E::REGS) {
            unsigned int sum_lo = 0, sum_hi = 0;
            e.each([&](unsigned int &v, int) { add_above(sum_lo, sum_hi, v, mid); });
            team.sum_packed(((u64)sum_hi << 32) | sum_lo, mass, c);
        } else {
            e.each([&](unsigned int &v, int) {
                if (v > mid) mass += v, ++c;
            });
            team.sum2(mass, c);
        }
        if (mass < limit)
            hi = mid, mass_hi = mass, count_hi = c;
        else
            lo = mid, count_lo = c;
    }
    cut = hi, mass_above = mass_hi, ties = count_lo - count_hi;
    if (hi - lo <= 1) return;
    unsigned int here = 0;
    e.each([&](unsigned int &v, int) { here += v - lo - 1 < hi - lo ? 1u : 0u; });
    const unsigned int incl = warp_scan32(here, team.lane);
    u64 before, all;
    team.prefix(__shfl_sync(kFull, incl, 31), before, all);
    unsigned int *to = MULTI ? cluster_peer(sort_list, 0, team.cs) : sort_list;
    unsigned int at = (unsigned int)before + incl - here;
    e.each([&](unsigned int &v, int) {
        if (v - lo - 1 < hi - lo) to[at++] = v;
    });
    if (MULTI)
        cluster_sync(team.cs);
    else
        __syncwarp();
    u64 packed = 0;
    if (team.me == 0) {
        unsigned int a = team.lane < (int)all ? sort_list[team.lane] : 0u, b = team.lane + 32 < (int)all ? sort_list[team.lane + 32] : 0u;
        sort64(a, b, team.lane);
        const u64 run_a = mass_hi + warp_scan(a, team.lane);
        const u64 run_b = __shfl_sync(kFull, run_a, 31) + warp_scan(b, team.lane);
        const unsigned int in_a = __ballot_sync(kFull, run_a >= limit), in_b = __ballot_sync(kFull, run_b >= limit);
        cut = in_a ? __shfl_sync(kFull, a, __ffs(in_a) - 1) : __shfl_sync(kFull, b, __ffs(in_b) - 1);
        mass_above = mass_hi + warp_sum((u64)(a > cut ? a : 0u) + (b > cut ? b : 0u));
        packed = ((u64)__reduce_add_sync(kFull, (a == cut ? 1u : 0u) + (b == cut ? 1u : 0u)) << 32) | cut;
    }
    team.tell(team.me == 0, mass_above, packed);
    cut = (unsigned int)packed, ties = packed >> 32;
    if (!MULTI) __syncwarp();   // the list may be written again
}

// Filters and draws. e holds logits (as bits); logit(col) reads one again, host(col) names the column's host.
template <bool MULTI, typename E, typename X, typename H>
__device__ __forceinline__ void decide(const SampleArgs &a, long long row, const Row &p, Team<MULTI> &team, E &e,
                                       unsigned int *sort_list, X logit, H host)
{
    const int lane = team.lane;
    // top-k: cut_x = the k-th largest logit; of its ties the first in index order stay. Hosts below m - 32 / c have
    // weight 0: if at most k are above that, top-k changes nothing.
    float cut_x = neg_inf();    // logits above it stay
    int tie_col = -1;           // and of those equal to it the columns up to this one
    if (!p.none && p.k > 0 && p.k < e.n) {
        const unsigned int k = (unsigned int)p.k;
        auto above = [&](float x) -> unsigned int {
            unsigned int c = 0;
            e.each([&](unsigned int &v, int) { c += __uint_as_float(v) > x ? 1u : 0u; });
            return team.count(c);
        };
        float lo_f = __fsub_rn(p.m, __fdiv_rn(32.0f, p.scale)), hi_f = p.m;
        if (!(lo_f < hi_f)) lo_f = neg_inf();   // m so large that the distance vanishes
        unsigned int lo = key_of(lo_f), hi = key_of(hi_f);
        unsigned int above_hi = 0;
        bool exact = above(lo_f) <= k;
        // invariant: above(hi) < k <= above(lo)
        for (int it = 1; !exact && hi - lo > 1; ++it) {
            if ((it & 3) == 0) {   // the bounds onto logits that occur
                float most = neg_inf();
                unsigned int least = 0xFFFFFFFFu;
                e.each([&](unsigned int &v, int) {
                    const float x = __uint_as_float(v);
                    if (x <= hi_f) most = fmaxf(most, x);
                    if (x > lo_f) least = min(least, key_of(x + 0.0f));   // + 0: one zero
                });
                hi_f = team.max(most), hi = key_of(hi_f + 0.0f);
                lo = ~team.max_key(~least) - 1, lo_f = float_of(lo);
                if (hi - lo <= 1) break;
            }
            unsigned int mid = lo + (hi - lo) / 2;
            if (it < 24) {   // halving the values converges faster than halving the keys at first
                const unsigned int g = key_of(0.5f * lo_f + 0.5f * hi_f);
                if (g > lo && g < hi) mid = g;
            }
            const float mid_f = float_of(mid);
            const unsigned int c = above(mid_f);
            if (c >= k) {
                lo = mid, lo_f = mid_f;
                exact = c == k;
            } else {
                hi = mid, hi_f = mid_f, above_hi = c;
            }
        }
        if (exact) {
            cut_x = lo_f;
        } else {
            cut_x = hi_f;
            tie_col = nth_column(team, e, k - above_hi - 1, [&](unsigned int v, int) { return __uint_as_float(v) == cut_x; });
        }
    }
    // weights from here on
    u64 total = 0, count = 0;
    if constexpr (E::REGS) {
        unsigned int sum_lo = 0, sum_hi = 0;
        e.each([&](unsigned int &v, int col) {
            const float f = __uint_as_float(v);
            v = f > cut_x || (f == cut_x && col <= tie_col) ? weight_of(f, p.m, p.scale) : 0u;
            add_above(sum_lo, sum_hi, v, 0u);
        });
        total = ((u64)sum_hi << 32) | sum_lo;
        if (p.top_p < 1.0f) team.sum_packed(total, total, count);
    } else {
        e.each([&](unsigned int &v, int col) {
            const float f = __uint_as_float(v);
            v = f > cut_x || (f == cut_x && col <= tie_col) ? weight_of(f, p.m, p.scale) : 0u;
            total += v;
            count += v != 0;
        });
        if (p.top_p < 1.0f) team.sum2(total, count);
    }

    unsigned int least = 0;   // weights below it go
    if (p.min_p > 0.0f) least = (unsigned int)(fminf(p.min_p, 1.0f) * 0x1p31f);
    if (p.top_p < 1.0f && !p.greedy && total > 0) {
        u64 limit = share_of(total, (unsigned int)(fmaxf(p.top_p, 0.0f) * 0x1p24f));
        if (limit == 0) limit = 1;
        unsigned int cut;
        u64 mass_above, ties;
        nucleus(team, e, limit, total, count, sort_list, cut, mass_above, ties);
        least = max(least, cut);
        // the first ceil((limit - mass_above) / cut) of the ties in (x descending, index ascending) stay
        const u64 keep = (limit - mass_above + cut - 1) / cut;
        if (keep < ties && least == cut) {
            // the ties' logits may still differ: bisection on their keys
            auto key_at = [&](int col) { return key_of(fminf(logit(col), kMaxFinite) + 0.0f); };
            unsigned int least_key = 0xFFFFFFFFu, most_key = 0;
            e.each([&](unsigned int &v, int col) {
                if (v == cut) {
                    const unsigned int key = key_at(col);
                    least_key = min(least_key, key), most_key = max(most_key, key);
                }
            });
            // above(khi) < keep <= above(klo) among the ties
            unsigned int klo = ~team.max_key(~least_key) - 1, khi = team.max_key(most_key);
            u64 above_khi = 0, above_klo = ties;
            while (khi - klo > 1 && above_klo > keep) {
                const unsigned int mid = klo + (khi - klo) / 2;
                unsigned int c = 0;
                e.each([&](unsigned int &v, int col) {
                    if (v == cut) c += key_at(col) > mid ? 1u : 0u;
                });
                c = team.count(c);
                if (c >= keep)
                    klo = mid, above_klo = c;
                else
                    khi = mid, above_khi = c;
            }
            unsigned int kcut = klo;
            int kcol = -1;
            if (above_klo > keep) {
                kcut = khi;
                kcol = nth_column(team, e, keep - above_khi - 1, [&](unsigned int v, int col) { return v == cut && key_at(col) == kcut; });
            }
            e.each([&](unsigned int &v, int col) {
                if (v != cut) return;
                const unsigned int key = key_at(col);
                if (!(key > kcut || (key == kcut && col <= kcol))) v = 0;
            });
        }
    }
    if (least > 0)
        e.each([&](unsigned int &v, int) {
            if (v < least) v = 0;
        });

    auto as_is = [](unsigned int v, int) -> u64 { return v; };
    u64 sums[E::REGS ? E::CH : 1], mine = 0;   // the lane's weight in each chunk; the warp's
    if constexpr (E::REGS) {
#pragma unroll
        for (int c = 0; c < E::CH; ++c) sums[c] = e.chunk_sum(c, as_is), mine += sums[c];
    } else {
        e.each([&](unsigned int &v, int) { mine += v; });
    }
    mine = warp_sum(mine);
    int found = 0;
    for (int d = 0; d < a.draws; ++d) {
        u64 before, left;
        team.prefix(mine, before, left);
        int col = -1;
        if (left > 0) {
            unsigned int steps = (unsigned int)(fminf(fmaxf(a.u[row * a.draws + d], 0.0f), 1.0f) * 0x1p24f);
            if (steps > 0xFFFFFFu) steps = 0xFFFFFFu;
            const u64 t = share_of(left, steps);
            const bool has = t >= before && t < before + mine;
            u64 val = 0;
            if (has) {
                if constexpr (E::REGS)
                    e.find(t, before, lane, [&](int c) { return sums[c]; }, as_is, col, val);
                else
                    e.find(t, before, lane, [&](int c) { return e.chunk_sum(c, as_is); }, as_is, col, val);
                mine -= val;
                if (d + 1 < a.draws) {   // out of what is left
                    e.each([&](unsigned int &v, int at) {
                        if (at == col) v = 0;
                    });
                    if constexpr (E::REGS) {
#pragma unroll
                        for (int c = 0; c < E::CH; ++c) {
                            const int off = col - e.base - c * 32 * E::VEC;
                            if (off >= 0 && off < E::VEC) sums[c] -= val;
                        }
                    }
                }
            }
            u64 where = (u64)(unsigned int)col;
            team.tell(has, where, val);
            col = host((int)(unsigned int)where);
            ++found;
        }
        if (team.me == 0 && lane == 0) a.hosts[row * a.draws + d] = col;
    }
    if (a.found && team.me == 0 && lane == 0) a.found[row] = found;
}

constexpr int kList = 256;      // hosts a short list holds: 8 a lane of one warp
constexpr int kListK = 128;     // largest top-k that tries for one
struct ShortList {
    unsigned int sort[kSort];
    float x[kList];
    int col[kList];
};

// top-k of a long row leaves few hosts. A threshold that at least k of the lanes' chunk maxima exceed is exceeded by all
// of the k best, and by not many others: those go, in index order, to a list that one warp finishes alone. Returns
// the list's length, or -1 if it would be too long (many equal logits).
template <bool MULTI, typename E>
__device__ __forceinline__ int short_list(const Row &p, Team<MULTI> &team, E &e, ShortList *list)
{
    constexpr int VEC = E::VEC, CH = E::CH;
    float top[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        top[c] = neg_inf();
#pragma unroll
        for (int i = 0; i < VEC; ++i) top[c] = fmaxf(top[c], __uint_as_float(e.r[c * VEC + i]));
    }
    auto above = [&](float x) -> unsigned int {
        unsigned int n = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) n += top[c] > x ? 1u : 0u;
        return team.count(n);
    };
    const unsigned int k = (unsigned int)p.k;
    float lo = __fsub_rn(p.m, __fdiv_rn(32.0f, p.scale)), hi = p.m;   // weights at and below lo are 0
    if (!(lo < hi)) lo = neg_inf();
    unsigned int n = above(lo);
    for (int it = 0; it < 10 && n > k + k / 4 + 4; ++it) {
        const float mid = 0.5f * lo + 0.5f * hi;
        const unsigned int c = above(mid);
        if (c >= k)
            lo = mid, n = c;
        else
            hi = mid;
    }
    // where each chunk's hosts go: a field per chunk, wide enough for a warp's count in it (32 * VEC)
    constexpr int F = VEC > 4 ? 16 : 8;
    static_assert(CH * F <= 64, "a field per chunk");
    u64 mine = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        unsigned int here = 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) here += __uint_as_float(e.r[c * VEC + i]) > lo ? 1u : 0u;
        mine += (u64)here << (c * F);
    }
    const u64 incl = warp_scan(mine, team.lane), all = __shfl_sync(kFull, incl, 31), excl = incl - mine;
    unsigned int total = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) total += (unsigned int)(all >> (c * F)) & ((1u << F) - 1u);
    u64 before, length;
    team.prefix(total, before, length);
    if (length > kList) return -1;
    ShortList *to = MULTI ? cluster_peer(list, 0, team.cs) : list;
    unsigned int base = (unsigned int)before;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        unsigned int at = base + ((unsigned int)(excl >> (c * F)) & ((1u << F) - 1u));
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float x = __uint_as_float(e.r[c * VEC + i]);
            if (x > lo) {
                to->x[at] = x;
                to->col[at] = e.base + c * 32 * VEC + i;
                ++at;
            }
        }
        base += (unsigned int)(all >> (c * F)) & ((1u << F) - 1u);
    }
    return (int)length;
}

template <typename T, int CH, bool MULTI, bool REGS>
__device__ __forceinline__ void sample_row(const SampleArgs &a, long long row, Team<MULTI> team, ShortList *list, unsigned int *store, int chunks)
{
    constexpr int VEC = kPer16<T>;
    const T *x = static_cast<const T *>(a.x) + row * a.stride;
    const int lane = team.lane;
    Elems<VEC, CH, REGS> e;
    e.store = store, e.chunks = chunks, e.n = a.n;
    e.base = team.me * (REGS ? CH : chunks) * 32 * VEC + lane * VEC;
    Row p;
    const float temperature = a.temperature ? a.temperature[row] : 1.0f;
    p.greedy = !(temperature > 0x1p-20f);
    p.scale = __fdiv_rn(kLog2e, p.greedy ? 1.0f : temperature);
    p.k = p.greedy ? 1 : (a.top_k ? a.top_k[row] : 0);
    p.top_p = a.top_p ? a.top_p[row] : 1.0f;
    p.min_p = a.min_p ? a.min_p[row] : 0.0f;

    float m = neg_inf();
    if constexpr (REGS) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = e.base + c * 32 * VEC;
            float v[VEC];
            if (a.aligned) {
                load_cols<T, VEC>(x, col, a.n, neg_inf(), v);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = col + i < a.n ? to_float(x[col + i]) : neg_inf();
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                m = fmaxf(m, v[i]);   // a NaN is never the larger, nor above any bound, and has weight 0
                e.r[c * VEC + i] = __float_as_uint(v[i]);
            }
        }
    } else {
        e.each([&](unsigned int &v, int col) {
            const float f = to_float(x[col]);
            m = fmaxf(m, f);
            v = __float_as_uint(f);
        });
    }
    p.m = team.max(m);
    if (p.m > kMaxFinite) {
        p.m = kMaxFinite;
        e.each([&](unsigned int &v, int) {
            if (v == 0x7F800000u) v = __float_as_uint(kMaxFinite);
        });
    }
    p.none = p.m == neg_inf();
    if constexpr (REGS && CH > 1) {
        if (!p.none && p.k > 0 && p.k <= kListK && p.k < a.n) {
            const int length = short_list(p, team, e, list);
            if (length >= 0) {
                if (MULTI)
                    cluster_sync(team.cs);
                else
                    __syncwarp();
                if (team.me != 0) return;
                Team<false> one{nullptr, 1, 1, 0, lane, 0};
                Elems<8, kList / 256, true> f;
                f.store = nullptr, f.chunks = kList / 256, f.n = length, f.base = lane * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    f.r[i] = __float_as_uint(lane * 8 + i < length ? list->x[lane * 8 + i] : neg_inf());
                decide(a, row, p, one, f, list->sort, [&](int col) { return list->x[col]; }, [&](int col) { return list->col[col]; });
                return;
            }
        }
    }
    decide(a, row, p, team, e, list->sort, [&](int col) { return to_float(x[col]); }, [](int col) { return col; });
}

template <typename T, int CH>
__global__ void __launch_bounds__(128) sample_warp_kernel(SampleArgs a)
{
    __shared__ ShortList s_list[4];
    const int warp = threadIdx.x >> 5;
    const long long row = (long long)blockIdx.x * 4 + warp;
    if (row >= a.rows) return;
    Team<false> team{nullptr, 1, 1, 0, (int)(threadIdx.x & 31), 0};
    sample_row<T, CH, false, true>(a, row, team, &s_list[warp], nullptr, CH);
}

// grid: REGS one block / cluster per row; else `clusters` of them take the rows in turn
// THREADS: most threads of a block; blocks of up to 256 get more registers than 1,024 threads leave
template <typename T, bool REGS, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : 3) sample_block_kernel(SampleArgs a, int cs, int chunks)
{
    __shared__ ulonglong2 s_slots[2][kMaxCluster * 32];
    __shared__ ShortList s_list;
    const int rank = cluster_rank(cs), warps = blockDim.x >> 5;
    Team<true> team{s_slots, warps * cs, cs, rank * warps + (int)(threadIdx.x >> 5), (int)(threadIdx.x & 31), 0};
    cluster_sync(cs);   // all blocks of the cluster run
    const long long first = blockIdx.x / cs, step = gridDim.x / cs;
    for (long long row = first; row < a.rows; row += step) {
        sample_row<T, kElems / kPer16<T>, true, REGS>(a, row, team, &s_list, REGS ? nullptr : a.store + first * a.n, chunks);
        cluster_sync(cs);   // slots and list are free again
    }
}

template <typename T>
cudaError_t launch(SampleArgs a, int sms, int device, cudaStream_t stream)
{
    constexpr int VEC = kPer16<T>;
    if (a.n <= 32 * kElems) {
        const unsigned int blocks = (unsigned int)((a.rows + 3) / 4);
        if (a.n <= 32 * VEC)
            sample_warp_kernel<T, 1><<<blocks, 128, 0, stream>>>(a);
        else
            sample_warp_kernel<T, kElems / VEC><<<blocks, 128, 0, stream>>>(a);
        return cudaGetLastError();
    }
    const bool regs = a.n <= kMaxCluster * kBlockRow;
    auto threads_for = [&](int c) { return ((a.n + c * kElems - 1) / (c * kElems) + 31) / 32 * 32; };
    int cs = 1;
    while (cs < kMaxCluster && (threads_for(cs) > 1024 || (a.rows * cs < sms && threads_for(cs) > 256))) cs *= 2;
    const int threads = regs ? threads_for(cs) : 1024;
    const int warps = threads / 32 * cs;
    const int chunks = regs ? kElems / VEC : (a.n + warps * 32 * VEC - 1) / (warps * 32 * VEC);
    long long clusters = a.rows < (1ll << 27) ? a.rows : (1ll << 27);
    void *store = nullptr;
    if (!regs) {
        if (clusters > sms / cs) clusters = sms / cs;
        cudaMemPool_t pool = nullptr;
        if (library_pool(device, &pool)) return cudaErrorMemoryAllocation;
        const cudaError_t e = cudaMallocFromPoolAsync(&store, (size_t)clusters * a.n * sizeof(unsigned int), pool, stream);
        if (e != cudaSuccess) return e;
        a.store = static_cast<unsigned int *>(store);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned int)(clusters * cs));
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = !regs           ? cudaLaunchKernelEx(&cfg, sample_block_kernel<T, false, 1024>, a, cs, chunks)
                          : threads > 256 ? cudaLaunchKernelEx(&cfg, sample_block_kernel<T, true, 1024>, a, cs, chunks)
                                          : cudaLaunchKernelEx(&cfg, sample_block_kernel<T, true, 256>, a, cs, chunks);
    if (store) cudaFreeAsync(store, stream);
    return e;
}

}  // namespace
}  // namespace nbos

using namespace nbos;

extern "C" int nbos_policy_sample(const nbos_logits *logits, const float *uniforms, const float *temperature,
                                  const int32_t *top_k, const float *top_p, const float *min_p, int32_t draws,
                                  int32_t *out_hosts, int32_t *out_found, void *cuda_stream)
{
    int rc = check_logits(logits);
    if (rc) return rc;
    if (draws < 1 || draws > NBOS_POLICY_MAX_DRAWS)
        return fail(NBOS_ERR_INVALID_ARG, "draws must be in 1..%d (got %d)", NBOS_POLICY_MAX_DRAWS, draws);
    if (logits->rows == 0) return NBOS_OK;
    if (!uniforms || !out_hosts) return fail(NBOS_ERR_INVALID_ARG, "uniforms / out_hosts is NULL");
    if (!aligned_to(uniforms, 4) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) ||
        !aligned_to(min_p, 4) || !aligned_to(out_hosts, 4) || !aligned_to(out_found, 4))
        return fail(NBOS_ERR_INVALID_ARG, "an int32 / float array is not 4-byte aligned");
    int sms = 0, device = 0;
    if ((rc = check_sm100(&sms, &device))) return rc;
    SampleArgs a{logits->data, logits->rows, logits->row_stride, logits->n_hosts, draws, 0, uniforms, temperature, top_k,
                 top_p, min_p, out_hosts, out_found, nullptr};
    if (a.rows == 1) a.stride = a.n;
    a.aligned = rows_aligned16(a.x, a.rows, a.stride, dtype_bytes(logits->dtype));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = logits->dtype == NBOS_F32    ? launch<float>(a, sms, device, stream)
                          : logits->dtype == NBOS_BF16 ? launch<__nv_bfloat16>(a, sms, device, stream)
                                                       : launch<__half>(a, sms, device, stream);
    if (e == cudaErrorMemoryAllocation) {
        cudaGetLastError();
        return fail(NBOS_ERR_NO_MEMORY, "device allocation failed: %s", cudaGetErrorString(e));
    }
    if (e != cudaSuccess) return cuda_fail(e, "sampling launch");
    return NBOS_OK;
}
