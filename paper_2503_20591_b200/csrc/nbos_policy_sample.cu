// Sampling distinct hosts from a policy's logits with given random numbers (nbos_policy_sample).
//
// Weights are whole numbers, w = floor(2^31 * 2^((x - m) c)), c = log2(e) / T: every sum of them is exact, so the
// split of a row over lanes, warps and blocks cannot change which host a random number selects. top-k, top-p and
// min-p each keep a first part of the order (x descending, index ascending); the draw runs in index order over what
// is left, so nothing long has to be sorted: cuts are found by bisection on counts (top-k) and exact sums (top-p)
// until a short list is left that one warp finishes.
// A team of warps shares a row, 1,024 hosts each: one warp, a block (up to 32,768 hosts), a cluster of up to 8 blocks
// (262,144). The logits are read once and stay in shared memory, as logits until the top-k cut is known and as
// weights from then on. The work is some 20 passes of a few integer instructions over them, which is what bounds
// it; loops over shared memory keep the code short (unrolled over registers it did not fit the instruction
// cache) and the registers few, so that many rows are in flight. Longer rows keep their elements in the
// workspace instead.
// A warp's columns are one stretch of the row, a lane's four of each 128 are neighbours: index order is warp, then
// chunk of 128, then lane.
// Measured (B200): 16,384 x 4,096 bf16 with all filters and three draws 179 us = 755 GB/s; 262,144 x 1,024 bf16 nucleus, one draw,
// 978 us = 556 GB/s (some 3,400 warp instructions a row, the integer pipe 77 % busy), without filters 330 us.
#include <math.h>

#include "nbos_policy.cuh"

namespace nbos {
namespace {

using namespace policy;

constexpr int kChunk = 128;            // columns a warp takes at once, four a lane
constexpr int kWarpChunks = 8;         // chunks of a warp, except of rows in the workspace
constexpr int kWarpRow = kChunk * kWarpChunks;
// Longest row of one warp. bf16, us by one warp / by a block of a warp for each 1,024 hosts: 24,000 x 1,040 plain 55 / 176, nucleus 124 / 430,
// all filters 85 / 300; 24,000 x 3,000 142 / 194, 419 / 566, 193 / 314; 24,000 x 4,096 213 / 216, 580 / 662, 265 / 335.
constexpr int kLoneRow = 4096;
constexpr int kMaxCluster = 8;
constexpr int kBlockRow = 32 * kWarpRow;
constexpr int kSort = 64;              // weights that one warp sorts, two a lane
constexpr int kList = 128;             // hosts of a list that one warp holds in registers, four a lane
constexpr int kListK = 112;            // largest top-k that tries for one: below 128, so that a threshold is found in few steps
typedef unsigned long long u64;

struct SampleArgs {
    const void *x;
    long long rows, stride;
    int n, draws, aligned;
    const float *u, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *hosts, *found;
    unsigned int *store;   // rows longer than the shared memory of a cluster: [clusters][n padded]
};

// floats in the order of unsigned integers; both zeros are 0x80000000, so that key - 1 is the next smaller value
__device__ __forceinline__ unsigned int key_of(float x)
{
    const unsigned int b = __float_as_uint(x);
    return (int)b < 0 ? 0u - b : b + 0x80000000u;
}
__device__ __forceinline__ float float_of(unsigned int key)
{
    return __uint_as_float(key & 0x80000000u ? key - 0x80000000u : 0u - key);
}

// +inf counts as the largest finite float
constexpr float kMaxFinite = 3.402823466e38f;

// floor(2^31 * 2^((x - m) scale)): difference and product are rounded one by one (no contraction). The power is at
// most 1, so its significand shifted by its exponent is the whole number; below 2^-31, and for NaN, it is 0.
__device__ __forceinline__ unsigned int weight_of(float x, float m, float scale)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(__fsub_rn(x, m), scale)));
    const unsigned int b = __float_as_uint(e);
    unsigned int w;
    asm("shr.u32 %0, %1, %2;" : "=r"(w) : "r"((b << 8) | 0x80000000u), "r"(127u - (b >> 23)));   // shifts above 31 give 0
    return w;
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
template <typename V>
__device__ __forceinline__ V warp_scan(V v, int lane)   // inclusive
{
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const V other = __shfl_up_sync(kFull, v, off);
        if (lane >= off) v += other;
    }
    return v;
}

// floor(total * steps / 2^24); total below 2^52, steps at most 2^24
__device__ __forceinline__ u64 share_of(u64 total, unsigned int steps)
{
    return (u64)steps * (total >> 24) + (((u64)steps * (total & 0xFFFFFFu)) >> 24);
}

// The warps that share a row (one warp: nothing is exchanged).
struct Team {
    ulonglong2 (*slots)[kMaxCluster * 32];   // two sets, taken in turn
    int warps, cs, me, lane, turn;           // me: this warp's place among all of the row

    __device__ __forceinline__ bool alone() const { return warps == 1; }
    __device__ __forceinline__ void sync() const
    {
        if (alone())
            __syncwarp();
        else
            cluster_sync(cs);
    }
    // every warp's (a, b), which the lanes of a warp agree on, to every warp, in slots[result]
    __device__ __forceinline__ int exchange(u64 a, u64 b)
    {
        const int now = turn;
        if (lane < cs) cluster_peer(slots[now], lane, cs)[me] = make_ulonglong2(a, b);
        cluster_sync(cs);
        turn ^= 1;
        return now;
    }
    // mass and number over the row, from a lane's own
    __device__ __forceinline__ void sum(u64 &mass, unsigned int &number)
    {
        mass = warp_sum(mass), number = __reduce_add_sync(kFull, number);
        if (alone()) return;
        const int now = exchange(mass, number);
        mass = 0, number = 0;
        for (int i = lane; i < warps; i += 32) mass += slots[now][i].x, number += (unsigned int)slots[now][i].y;
        mass = warp_sum(mass), number = __reduce_add_sync(kFull, number);
    }
    // the row's number and the warp's own
    __device__ __forceinline__ unsigned int count(unsigned int v, unsigned int &mine)
    {
        mine = v = __reduce_add_sync(kFull, v);
        if (alone()) return v;
        const int now = exchange(v, 0);
        v = 0;
        for (int i = lane; i < warps; i += 32) v += (unsigned int)slots[now][i].x;
        return __reduce_add_sync(kFull, v);
    }
    __device__ __forceinline__ unsigned int count(unsigned int v)
    {
        unsigned int mine;
        return count(v, mine);
    }
    // the largest a and the smallest b of the row
    __device__ __forceinline__ void bounds(unsigned int &a, unsigned int &b)
    {
        a = __reduce_max_sync(kFull, a), b = __reduce_min_sync(kFull, b);
        if (alone()) return;
        const int now = exchange(a, b);
        for (int i = lane; i < warps; i += 32) a = max(a, (unsigned int)slots[now][i].x), b = min(b, (unsigned int)slots[now][i].y);
        a = __reduce_max_sync(kFull, a), b = __reduce_min_sync(kFull, b);
    }
    __device__ __forceinline__ float max_of(float v)
    {
        v = lanes_max(v, 32);
        if (alone()) return v;
        const int now = exchange(__float_as_uint(v), 0);
        for (int i = lane; i < warps; i += 32) v = fmaxf(v, __uint_as_float((unsigned int)slots[now][i].x));
        return lanes_max(v, 32);
    }
    // sums of `mine`, which the lanes of a warp agree on: over the warps before this one, and over all
    __device__ __forceinline__ void prefix(u64 mine, u64 &before, u64 &all)
    {
        before = 0, all = mine;
        if (alone()) return;
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
        if (alone()) return;
        const int now = turn;
        if (has && lane < cs) cluster_peer(slots[now], lane, cs)[0] = make_ulonglong2(a, b);
        cluster_sync(cs);
        turn ^= 1;
        a = slots[now][0].x, b = slots[now][0].y;
    }
};

// A warp's elements, chunk after chunk: the lane's four of chunk c are at store[c * 128 + lane * 4] and belong to the
// columns first + c * 128 + lane * 4 ... Beyond the row they are logits of -inf, later weights of 0.
// U: chunks that a pass has under way at once, many where few warps share an SM.
template <int U>
struct Elems {
    unsigned int *store;
    int chunks;
    int first;   // column of store[0]
    int n;       // columns of the row
    unsigned int *block_store;   // of the block's first warp
    int block_columns;           // of all its warps

    __device__ __forceinline__ uint4 &at(int c, int lane) const { return reinterpret_cast<uint4 *>(store)[c * 32 + lane]; }
    template <typename F>
    __device__ __forceinline__ void each(int lane, F f) const   // f(value, column)
    {
#pragma unroll U
        for (int c = 0; c < chunks; ++c) {
            const uint4 v = at(c, lane);
            const int col = first + c * kChunk + lane * 4;
            f(v.x, col), f(v.y, col + 1), f(v.z, col + 2), f(v.w, col + 3);
        }
    }
    template <typename F>
    __device__ __forceinline__ void change(int lane, F f) const   // value = f(value, column)
    {
#pragma unroll(U / 2)
        for (int c = 0; c < chunks; ++c) {
            uint4 v = at(c, lane);
            const int col = first + c * kChunk + lane * 4;
            v.x = f(v.x, col), v.y = f(v.y, col + 1), v.z = f(v.z, col + 2), v.w = f(v.w, col + 3);
            at(c, lane) = v;
        }
    }
    // The first column, in index order over the warp, at which the running sum of value(element, column) from `run`
    // exceeds t, and the value there; the warp must hold it.
    template <typename F>
    __device__ __forceinline__ void find(u64 t, u64 run, int lane, F value, int &col_out, u64 &val_out) const
    {
        unsigned int v[4] = {0, 0, 0, 0};
        u64 mine = 0;
        int c = 0;
        for (; c < chunks; ++c) {
            const uint4 raw = at(c, lane);
            const int col = first + c * kChunk + lane * 4;
            v[0] = value(raw.x, col), v[1] = value(raw.y, col + 1), v[2] = value(raw.z, col + 2), v[3] = value(raw.w, col + 3);
            mine = (u64)v[0] + v[1] + v[2] + v[3];
            const u64 total = warp_sum(mine);
            if (t < run + total) break;
            run += total;
        }
        const u64 upto = run + warp_scan(mine, lane);
        const int owner = __ffs(__ballot_sync(kFull, t < upto)) - 1;
        u64 acc = upto - mine;
        int col = -1;
        unsigned int val = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc += v[i];
            if (col < 0 && t < acc) col = first + c * kChunk + lane * 4 + i, val = v[i];
        }
        col_out = __shfl_sync(kFull, col, owner);
        val_out = __shfl_sync(kFull, val, owner);
    }
};

// The column of the m-th (from 0) element, in index order over the row, that `pick` accepts.
template <int U, typename F>
__device__ __forceinline__ int nth_column(Team &team, const Elems<U> &e, u64 m, F pick)
{
    auto one = [&](unsigned int v, int col) -> unsigned int { return pick(v, col) ? 1u : 0u; };
    unsigned int here = 0;
    e.each(team.lane, [&](unsigned int v, int col) { here += one(v, col); });
    const u64 mine = __reduce_add_sync(kFull, here);
    u64 before, all, val = 0;
    team.prefix(mine, before, all);
    int col = -1;
    const bool has = m >= before && m < before + mine;
    if (has) e.find(m, before, team.lane, one, col, val);
    u64 where = (u64)(unsigned int)col;
    team.tell(has, where, val);
    return (int)(unsigned int)where;
}

struct Row {
    float m, scale, top_p, min_p;
    int k;          // 0: off
    bool greedy;   // T too small to divide by: the best host
};

// Weights at and below this logit are 0: 32 powers of two below the best one, and one more for the quotient's rounding. Rounded down: where
// neighbouring floats are as far apart as that, the nearest one may lie above and have a weight.
__device__ __forceinline__ float zero_below(const Row &p) { return __fsub_rd(p.m, __fdiv_rn(33.0f, p.scale)); }

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

struct SortList {
    unsigned int w[kSort];
    int col[kSort];
};
struct ShortList {   // hosts, in index order
    unsigned int x[kList];
    int col[kList];
};
union Lists {        // a row makes one or the other
    SortList sort;
    ShortList hosts;
};

// The nucleus: the first weights, in (x descending, index ascending) order, before which less than `limit` stands.
// Returns the weight of the last of them. Of the `ties` that have just this weight the first `keep` are to stay (0: all that
// are left in the row: the others have been taken out). Bisection (on the logarithm at first, with the bounds moved onto weights that
// occur every few steps) until at most 64 weights are left between the bounds, which one warp then sorts.
// key_at(column): the order of the logit there.
template <int U, typename K>
__device__ __forceinline__ unsigned int nucleus(Team &team, const Elems<U> &e, u64 limit, u64 total, unsigned int count,
                                                SortList *list, u64 &keep, u64 &ties, K key_at)
{
    const int lane = team.lane;
    // invariant: mass(w > hi) < limit <= mass(w > lo)
    unsigned int lo = 0, hi = 0x80000000u, count_hi = 0, count_lo = count;
    u64 mass_hi = 0;
    // Weights below (total - limit) / n together hold less than what may be left out: the cut lies above them.
    const u64 least = (total - limit) / (unsigned int)e.n;
    for (int it = 0; hi - lo > 1 && count_lo - count_hi > kSort; ++it) {
        if ((it & 3) == 2 && it > 4) {
            unsigned int most_in = 0, least_in = 0xFFFFFFFFu;
            e.each(lane, [&](unsigned int v, int) {
                if (v <= hi) most_in = max(most_in, v);
                if (v > lo) least_in = min(least_in, v);
            });
            team.bounds(most_in, least_in);
            hi = most_in, lo = least_in - 1;
            if (hi - lo <= 1) break;
        }
        unsigned int mid = __float2uint_rd(__uint_as_float((__float_as_uint(__uint2float_rn(lo ? lo : 1)) + __float_as_uint(__uint2float_rn(hi))) / 2));
        if (it == 0 && least > 1) mid = (unsigned int)least - 1;
        if (mid <= lo || mid >= hi) mid = lo + (hi - lo) / 2;
        u64 mass = 0;
        unsigned int c = 0;
        for (int at = 0; at < e.chunks; at += kWarpChunks) {   // 2^44 above 32 weights: a warp's usual chunks
            unsigned int sum_lo = 0, sum_hi = 0;
            const Elems<U> part{e.store + at * kChunk, min(kWarpChunks, e.chunks - at), 0, 0, nullptr, 0};
            part.each(lane, [&](unsigned int v, int) { add_above(sum_lo, sum_hi, v, mid); });
            mass += ((u64)(sum_hi & 0xFFFu) << 32) | sum_lo, c += sum_hi >> 12;
        }
        team.sum(mass, c);
        if (mass < limit)
            hi = mid, mass_hi = mass, count_hi = c;
        else
            lo = mid, count_lo = c;
    }
    if (hi - lo <= 1) {
        ties = count_lo - count_hi;
        keep = (limit - mass_hi + hi - 1) / hi;
        if (keep >= ties) keep = 0;
        return hi;
    }
    unsigned int here = 0;
    e.each(lane, [&](unsigned int v, int) { here += v - lo - 1 < hi - lo ? 1u : 0u; });
    const unsigned int incl = warp_scan(here, lane);
    u64 before, all;
    team.prefix(__shfl_sync(kFull, incl, 31), before, all);
    SortList *to = team.alone() ? list : cluster_peer(list, 0, team.cs);
    unsigned int pos = (unsigned int)before + incl - here;
    e.each(lane, [&](unsigned int v, int col) {
        if (v - lo - 1 < hi - lo) to->w[pos] = v, to->col[pos++] = col;
    });
    team.sync();
    u64 cut = 0, none = 0;
    if (team.me == 0) {
        const bool has_a = lane < (int)all, has_b = lane + 32 < (int)all;
        const unsigned int wa = has_a ? list->w[lane] : 0u, wb = has_b ? list->w[lane + 32] : 0u;
        unsigned int a = wa, b = wb;
        sort64(a, b, lane);
        const u64 run_a = mass_hi + warp_scan((u64)a, lane);
        const u64 run_b = __shfl_sync(kFull, run_a, 31) + warp_scan((u64)b, lane);
        const unsigned int in_a = __ballot_sync(kFull, run_a >= limit), in_b = __ballot_sync(kFull, run_b >= limit);
        cut = in_a ? __shfl_sync(kFull, a, __ffs(in_a) - 1) : __shfl_sync(kFull, b, __ffs(in_b) - 1);
        const u64 above = mass_hi + warp_sum((u64)(a > cut ? a : 0u) + (b > cut ? b : 0u));
        unsigned int tie_a = __ballot_sync(kFull, wa == cut), tie_b = __ballot_sync(kFull, wb == cut);
        const unsigned int stay = (unsigned int)min((limit - above + cut - 1) / cut, (u64)kSort);
        if (stay < (unsigned int)(__popc(tie_a) + __popc(tie_b))) {
            // each tie's place among them by logit, then index; those from `stay` on go
            const int col_a = wa == cut ? list->col[lane] : 0, col_b = wb == cut ? list->col[lane + 32] : 0;
            const unsigned int key_a = wa == cut ? key_at(col_a) : 0u, key_b = wb == cut ? key_at(col_b) : 0u;
            unsigned int place_a = 0, place_b = 0;
            while (tie_a | tie_b) {
                const bool from_a = tie_a != 0;
                const int src = __ffs(from_a ? tie_a : tie_b) - 1;
                if (from_a)
                    tie_a &= tie_a - 1;
                else
                    tie_b &= tie_b - 1;
                const unsigned int key = __shfl_sync(kFull, from_a ? key_a : key_b, src);
                const int col = __shfl_sync(kFull, from_a ? col_a : col_b, src);
                place_a += key > key_a || (key == key_a && col < col_a);
                place_b += key > key_b || (key == key_b && col < col_b);
            }
            auto out = [&](int col) {
                const int rank = team.cs > 1 ? col / e.block_columns : 0;
                unsigned int *at = team.cs > 1 && e.block_columns < (1 << 30) ? cluster_peer(e.block_store, rank, team.cs) : e.block_store;
                at[col - rank * e.block_columns] = 0;
            };
            if (wa == cut && place_a >= stay) out(col_a);
            if (wb == cut && place_b >= stay) out(col_b);
            __syncwarp();
        }
    }
    team.tell(team.me == 0, cut, none);
    keep = 0;
    return (unsigned int)cut;
}

// Filters and draws of a row whose logits (as bits) e holds.
template <typename T, int U>
__device__ __forceinline__ void decide(const SampleArgs &a, long long row, const T *x, const Row &p, Team &team,
                                       const Elems<U> &e, SortList *sort_list)
{
    const int lane = team.lane;
    // top-k: cut_x = the k-th largest logit; of its ties the first in index order stay. If at most k logits have a
    // weight above 0, top-k changes nothing.
    float cut_x = neg_inf();    // logits from it on stay
    if (p.k > 0 && p.k < e.n) {
        const unsigned int k = (unsigned int)p.k;
        float lo_f = zero_below(p), hi_f = p.m;
        unsigned int lo = key_of(lo_f), hi = key_of(hi_f), above_hi = 0;
        bool exact = false;
        // invariant: above(hi) < k <= above(lo); the first step looks at lo_f. Where that is the next value below hi, lo goes one further
        // down, so that the step is taken all the same.
        if (hi - lo == 1) --lo;
        for (int it = 0; !exact && hi - lo > 1; ++it) {
            if ((it & 3) == 3) {   // the bounds onto logits that occur
                unsigned int most_in = 0, least_in = 0xFFFFFFFFu;
                e.each(lane, [&](unsigned int v, int) {
                    const float f = __uint_as_float(v);
                    const unsigned int key = key_of(f);
                    if (f <= hi_f) most_in = max(most_in, key);
                    if (f > lo_f) least_in = min(least_in, key);
                });
                team.bounds(most_in, least_in);
                hi = most_in, hi_f = float_of(hi), lo = least_in - 1, lo_f = float_of(lo);
                if (hi - lo <= 1) break;
            }
            unsigned int mid = lo + (hi - lo) / 2;
            if (it < 24) {   // halving the values converges faster than halving the keys at first
                const unsigned int g = key_of(0.5f * lo_f + 0.5f * hi_f);
                if (g > lo && g < hi) mid = g;
            }
            const float mid_f = it == 0 ? lo_f : float_of(mid);
            unsigned int c = 0;
            e.each(lane, [&](unsigned int v, int) { c += __uint_as_float(v) > mid_f ? 1u : 0u; });
            c = team.count(c);
            if (it == 0) {
                exact = c <= k;
            } else if (c >= k) {
                lo = mid, lo_f = mid_f;
                exact = c == k;
            } else {
                hi = mid, hi_f = mid_f, above_hi = c;
            }
        }
        if (exact) {
            cut_x = float_of(lo + 1);
        } else {
            cut_x = hi_f;
            const int tie_col = nth_column(team, e, k - above_hi - 1, [&](unsigned int v, int) { return __uint_as_float(v) == cut_x; });
            e.change(lane, [&](unsigned int v, int col) { return __uint_as_float(v) == cut_x && col > tie_col ? 0xFF800000u : v; });
        }
    }
    // weights from here on
    u64 mine = 0;
    unsigned int count = 0;
    for (int at = 0; at < e.chunks; at += kWarpChunks) {
        unsigned int sum_lo = 0, sum_hi = 0;
        const Elems<U> part{e.store + at * kChunk, min(kWarpChunks, e.chunks - at), 0, 0, nullptr, 0};
        part.change(lane, [&](unsigned int v, int) {
            const float f = __uint_as_float(v);
            const unsigned int w = f >= cut_x ? weight_of(f, p.m, p.scale) : 0u;
            add_above(sum_lo, sum_hi, w, 0u);
            return w;
        });
        mine += ((u64)(sum_hi & 0xFFFu) << 32) | sum_lo, count += sum_hi >> 12;
    }

    unsigned int least = 0;   // weights below it go
    if (p.min_p > 0.0f) least = (unsigned int)(fminf(p.min_p, 1.0f) * 0x1p31f);
    if (p.top_p < 1.0f) {
        u64 total = mine;
        team.sum(total, count);
        u64 limit = share_of(total, (unsigned int)(fmaxf(p.top_p, 0.0f) * 0x1p24f));
        if (limit == 0) limit = 1;
        auto key_at = [&](int col) { return key_of(fminf(to_float(x[col]), kMaxFinite)); };
        u64 keep, ties;
        const unsigned int cut = nucleus(team, e, limit, total, count, sort_list, keep, ties, key_at);
        least = max(least, cut);
        if (keep > 0 && least == cut) {
            // many ties, whose logits may still differ: bisection on their keys
            unsigned int least_key = 0xFFFFFFFFu, most_key = 0;
            e.each(lane, [&](unsigned int v, int col) {
                if (v != cut) return;
                const unsigned int key = key_at(col);
                least_key = min(least_key, key), most_key = max(most_key, key);
            });
            team.bounds(most_key, least_key);
            // above(khi) < keep <= above(klo) among the ties
            unsigned int klo = least_key - 1, khi = most_key;
            u64 above_khi = 0, above_klo = ties;
            while (khi - klo > 1 && above_klo > keep) {
                const unsigned int mid = klo + (khi - klo) / 2;
                unsigned int c = 0;
                e.each(lane, [&](unsigned int v, int col) {
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
            e.change(lane, [&](unsigned int v, int col) {
                if (v != cut) return v;
                const unsigned int key = key_at(col);
                return key > kcut || (key == kcut && col <= kcol) ? v : 0u;
            });
        }
    }
    if (least > 0) {
        mine = 0;
        e.change(lane, [&](unsigned int v, int) {
            const unsigned int w = v < least ? 0u : v;
            mine += w;
            return w;
        });
    }
    mine = warp_sum(mine);

    auto as_is = [](unsigned int v, int) { return v; };
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
                e.find(t, before, lane, as_is, col, val);
                mine -= val;
                if (lane == 0) e.store[col - e.first] = 0;   // out of what is left
                __syncwarp();
            }
            u64 where = (u64)(unsigned int)col;
            team.tell(has, where, val);
            col = (int)(unsigned int)where;
            ++found;
        }
        if (team.me == 0 && lane == 0) a.hosts[row * a.draws + d] = col;
    }
    if (a.found && team.me == 0 && lane == 0) a.found[row] = found;
}

// descending over the positions lane + 32 j, j < R, a bitonic network
template <int R>
__device__ __forceinline__ void sort_places(unsigned int (&s)[4], int lane)
{
#pragma unroll
    for (int k = 2; k <= 32 * R; k *= 2)
#pragma unroll
        for (int d = k / 2; d > 0; d /= 2) {
            if (d >= 32) {
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const int o = j ^ (d / 32);
                    if (o < j) continue;
                    const unsigned int hi = max(s[j], s[o]), lo = min(s[j], s[o]);
                    const bool down = ((32 * j) & k) == 0;
                    s[j] = down ? hi : lo, s[o] = down ? lo : hi;
                }
            } else {
                const bool first = (lane & d) == 0;
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const unsigned int other = __shfl_xor_sync(kFull, s[j], d);
                    s[j] = (((lane + 32 * j) & k) == 0) == first ? max(s[j], other) : min(s[j], other);
                }
            }
        }
}

// Filters and draws of `places` (at most 128) hosts, in index order over the positions lane + 32 j: key[j] orders the logit there,
// 0 = no host. cols[position] names the host; NULL: the position does.
__device__ __forceinline__ void finish(const SampleArgs &a, long long row, const Row &p, unsigned int (&key)[4], int places, int lane, const int *cols)
{
    const unsigned int below = (1u << lane) - 1;
    unsigned int s[4], hosts = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s[j] = key[j];
        hosts += __popc(__ballot_sync(kFull, key[j] != 0));
    }
    const bool cut_k = p.k > 0 && p.k < (int)hosts;
    if (cut_k || p.top_p < 1.0f) {   // places above the last host hold 0 already
        if (places <= 32)
            sort_places<1>(s, lane);
        else
            sort_places<4>(s, lane);
    }
    auto at_place = [&](unsigned int i) {
        const unsigned int v = i < 64 ? (i < 32 ? s[0] : s[1]) : (i < 96 ? s[2] : s[3]);
        return __shfl_sync(kFull, v, i & 31);
    };
    // keep what has a key above v, and the first `stay` of those with v
    auto keep = [&](unsigned int v, unsigned int stay) {
        unsigned int before = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned int ties = __ballot_sync(kFull, key[j] == v);
            if (key[j] < v || (key[j] == v && before + __popc(ties & below) >= stay)) key[j] = 0;
            before += __popc(ties);
        }
    };
    if (cut_k) {
        const unsigned int v = at_place(p.k - 1);
        unsigned int above = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) above += __popc(__ballot_sync(kFull, key[j] > v));
        keep(v, (unsigned int)p.k - above);
        hosts = p.k;
    }
    auto weight = [&](unsigned int k) { return k ? weight_of(float_of(k), p.m, p.scale) : 0u; };
    unsigned int w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = weight(key[j]);
    if (p.top_p < 1.0f) {
        u64 limit = share_of(warp_sum((u64)w[0] + w[1] + w[2] + w[3]), (unsigned int)(fmaxf(p.top_p, 0.0f) * 0x1p24f));
        if (limit == 0) limit = 1;
        u64 run = 0;
        unsigned int v = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (v != 0) continue;
            const u64 upto = run + warp_scan((u64)(lane + 32 * j < (int)hosts ? weight(s[j]) : 0u), lane);
            const unsigned int in = __ballot_sync(kFull, upto >= limit);
            if (in) v = __shfl_sync(kFull, s[j], __ffs(in) - 1);
            run = __shfl_sync(kFull, upto, 31);
        }
        u64 above = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) above += key[j] > v ? w[j] : 0u;
        above = warp_sum(above);
        const unsigned int cut = weight(v);
        keep(v, (unsigned int)((limit - above + cut - 1) / cut));
    }
    unsigned int least = 0;
    if (p.min_p > 0.0f) least = (unsigned int)(fminf(p.min_p, 1.0f) * 0x1p31f);
    u64 upto[4], left = 0;   // running sums of the weights in index order
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (key[j] == 0 || w[j] < least) w[j] = 0;
        upto[j] = left;
        if (__any_sync(kFull, w[j])) {
            upto[j] = left + warp_scan((u64)w[j], lane);
            left = __shfl_sync(kFull, upto[j], 31);
        }
    }
    int found = 0;
    for (int d = 0; d < a.draws; ++d) {
        int host = -1;
        if (left > 0) {
            unsigned int steps = (unsigned int)(fminf(fmaxf(a.u[row * a.draws + d], 0.0f), 1.0f) * 0x1p24f);
            if (steps > 0xFFFFFFu) steps = 0xFFFFFFu;
            const u64 t = share_of(left, steps);
            int place = -1;
            unsigned int val = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned int over = __ballot_sync(kFull, upto[j] > t);
                if (place < 0 && over) {
                    place = 32 * j + __ffs(over) - 1;
                    val = __shfl_sync(kFull, w[j], place & 31);
                }
            }
            // out of what is left: its own running sum falls to the one before it
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (lane + 32 * j >= place) upto[j] -= val;
            left -= val;
            host = cols ? cols[place] : place;
            ++found;
        }
        if (lane == 0) a.hosts[row * a.draws + d] = host;
    }
    if (a.found && lane == 0) a.found[row] = found;
}

// top-k of a long row leaves few hosts: those above a threshold that at least k and at most 128 logits exceed go, in
// index order, to a list that one warp finishes alone. Returns the list's length, or -1 if no threshold was found
// (many equal logits).
template <int U>
__device__ __forceinline__ int short_list(const Row &p, Team &team, const Elems<U> &e, ShortList *list)
{
    const int lane = team.lane;
    const unsigned int k = (unsigned int)p.k;
    // bisection between the largest logit and where weights end, first at a quarter of the way
    float lo = zero_below(p), hi = p.m;
    unsigned int n = 0xFFFFFFFFu, mine = 0;
    for (int it = 0; it < 14; ++it) {
        float mid = it == 0 ? 0.25f * lo + 0.75f * hi : 0.5f * lo + 0.5f * hi;
        if (it == 6 && n == 0xFFFFFFFFu) mid = lo;   // perhaps there are no k with a weight
        unsigned int c = 0, own;
        e.each(lane, [&](unsigned int v, int) { c += __uint_as_float(v) > mid ? 1u : 0u; });
        c = team.count(c, own);
        if (c >= k || mid == lo)
            lo = mid, n = c, mine = own;
        else
            hi = mid;
        if (n <= kList) break;
    }
    if (n > kList) return -1;
    u64 before, all;
    team.prefix(mine, before, all);
    ShortList *to = team.alone() ? list : cluster_peer(list, 0, team.cs);
    unsigned int base = (unsigned int)before;
    for (int c = 0; c < e.chunks; ++c) {
        const uint4 v = e.at(c, lane);
        const unsigned int x[4] = {v.x, v.y, v.z, v.w};
        unsigned int here = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) here += __uint_as_float(x[i]) > lo ? 1u : 0u;
        if (!__any_sync(kFull, here)) continue;
        const unsigned int incl = warp_scan(here, lane);
        unsigned int pos = base + incl - here;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (__uint_as_float(x[i]) > lo) {
                to->x[pos] = x[i];
                to->col[pos] = e.first + c * kChunk + lane * 4 + i;
                ++pos;
            }
        base += __shfl_sync(kFull, incl, 31);
    }
    return (int)n;
}

__device__ __forceinline__ Row row_settings(const SampleArgs &a, long long row)
{
    Row p;
    p.m = neg_inf();
    const float temperature = a.temperature ? a.temperature[row] : 1.0f;
    p.greedy = !(temperature > 0x1p-20f);
    p.scale = __fdiv_rn(kLog2e, p.greedy ? 1.0f : temperature);
    p.k = a.top_k ? a.top_k[row] : 0;
    p.top_p = a.top_p ? a.top_p[row] : 1.0f;
    p.min_p = a.min_p ? a.min_p[row] : 0.0f;
    return p;
}
__device__ __forceinline__ void write_one(const SampleArgs &a, long long row, int host)   // host or none
{
    for (int d = 0; d < a.draws; ++d) a.hosts[row * a.draws + d] = d ? -1 : host;
    if (a.found) a.found[row] = host >= 0;
}

template <typename T, int U>
__device__ __forceinline__ void sample_row(const SampleArgs &a, long long row, Team team, const Elems<U> &e, Lists *lists)
{
    const T *x = static_cast<const T *>(a.x) + row * a.stride;
    const int lane = team.lane;
    Row p = row_settings(a, row);

    // all of a warp's loads in flight at once; a NaN is never the larger, nor above any bound, and has weight 0
    float m = neg_inf();
    constexpr int kLoads = U > 2 ? 2 * kWarpChunks : kWarpChunks;
    for (int c0 = 0; c0 < e.chunks; c0 += kLoads) {
        Raw4<T> raw[kLoads];
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            const int col = e.first + (c0 + c) * kChunk + lane * 4;
            if (c0 + c >= e.chunks) break;
            if (a.aligned && col + 4 <= a.n) {
                raw[c].load(x + col);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[c].set(i, col + i < a.n ? x[col + i] : from_float<T>(neg_inf()));
            }
        }
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
            if (c0 + c >= e.chunks) break;
            float v[4];
            raw[c].get(v);
            m = fmaxf(fmaxf(m, fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
            e.at(c0 + c, lane) = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
    }
    p.m = team.max_of(m);
    if (p.m == neg_inf()) {
        if (team.me == 0 && lane == 0) write_one(a, row, -1);
        return;
    }
    if (p.m > kMaxFinite) {
        p.m = kMaxFinite;
        e.change(lane, [&](unsigned int v, int) { return v == 0x7F800000u ? __float_as_uint(kMaxFinite) : v; });
    }
    if (p.greedy) {   // the first host with the largest logit
        unsigned int none = 0, col = 0xFFFFFFFFu;
        e.each(lane, [&](unsigned int v, int at) {
            if (__uint_as_float(v) == p.m) col = min(col, (unsigned int)at);
        });
        team.bounds(none, col);
        if (team.me == 0 && lane == 0) write_one(a, row, (int)col);
        return;
    }
    if (p.k > 0 && p.k <= kListK) {
        const int length = short_list(p, team, e, &lists->hosts);
        if (length >= 0) {
            team.sync();
            if (team.me != 0) return;
            unsigned int key[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                key[j] = lane + 32 * j < length ? key_of(__uint_as_float(lists->hosts.x[lane + 32 * j])) : 0u;
            finish(a, row, p, key, length, lane, lists->hosts.col);
            return;
        }
    }
    decide(a, row, x, p, team, e, &lists->sort);
}

// rows of at most 128 hosts: one warp per row, in registers
template <typename T>
__global__ void __launch_bounds__(128) sample_short_kernel(SampleArgs a)
{
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= a.rows) return;
    const T *x = static_cast<const T *>(a.x) + row * a.stride;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = lane + 32 * j < a.n ? to_float(x[lane + 32 * j]) : neg_inf();
    Row p = row_settings(a, row);
    unsigned int key[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = fminf(fmaxf(v[j], neg_inf()), kMaxFinite);   // NaN as -inf
        p.m = fmaxf(p.m, v[j]);
        key[j] = v[j] > neg_inf() ? key_of(v[j]) : 0u;
    }
    p.m = lanes_max(p.m, 32);
    if (p.greedy && p.m > neg_inf()) {
        int col = -1;
#pragma unroll
        for (int j = 3; j >= 0; --j) {
            const unsigned int here = __ballot_sync(kFull, v[j] == p.m);
            if (here) col = 32 * j + __ffs(here) - 1;
        }
        if (lane == 0) write_one(a, row, col);
        return;
    }
    finish(a, row, p, key, a.n, lane, nullptr);
}

// one warp per row; shared memory per warp: the row, the lists
template <typename T, int U>
__global__ void __launch_bounds__(128) sample_warp_kernel(SampleArgs a, int chunks, int warp_bytes)
{
    extern __shared__ __align__(16) char s_mem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * (blockDim.x >> 5) + warp;
    if (row >= a.rows) return;
    Lists *lists = reinterpret_cast<Lists *>(s_mem + warp * warp_bytes);
    unsigned int *store = reinterpret_cast<unsigned int *>(s_mem + (warp + 1) * warp_bytes) - chunks * kChunk;
    sample_row<T, U>(a, row, Team{nullptr, 1, 1, 0, lane, 0}, Elems<U>{store, chunks, 0, a.n, store, 0}, lists);
}

// grid: SHARED one block / cluster per row; else as many as the workspace has rows take them in turn
template <typename T, bool SHARED>
__global__ void __launch_bounds__(1024, 1) sample_block_kernel(SampleArgs a, int cs, int chunks)
{
    extern __shared__ __align__(16) char s_mem[];
    __shared__ ulonglong2 s_slots[2][kMaxCluster * 32];
    __shared__ Lists s_lists;
    const int rank = cluster_rank(cs), warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    const Team team{s_slots, warps * cs, cs, rank * warps + warp, (int)(threadIdx.x & 31), 0};
    const long long first = blockIdx.x / cs, step = gridDim.x / cs;
    const int span = chunks * kChunk;
    // the cluster's part of the workspace is one stretch: `cluster_peer` is not asked there
    unsigned int *block_store = SHARED ? reinterpret_cast<unsigned int *>(s_mem) : a.store + ((size_t)first * cs + rank) * span * warps;
    unsigned int *store = block_store + warp * span;
    cluster_sync(cs);   // all blocks of the cluster run
    for (long long row = first; row < a.rows; row += step) {
        sample_row<T, 2>(a, row, team, Elems<2>{store, chunks, team.me * span, a.n, SHARED ? block_store : block_store - (size_t)rank * span * warps, SHARED ? span * warps : 1 << 30}, &s_lists);
        cluster_sync(cs);   // slots and lists are free again
    }
}

template <typename T>
cudaError_t launch(SampleArgs a, int sms, int device, cudaStream_t stream)
{
    if (a.n <= kList) {
        sample_short_kernel<T><<<(unsigned int)((a.rows + 3) / 4), 128, 0, stream>>>(a);
        return cudaGetLastError();
    }
    // One warp alone exchanges nothing and waits for nobody: it takes rows of up to kLoneRow hosts as long as there are
    // enough of them to fill the SMs that way. Nucleus, us by one warp / by blocks: 600 x 4,096 34 / 29, 1,000 x 4,096 37 / 39,
    // 1,200 x 4,096 44 / 45, 2,400 x 4,096 72 / 79.
    if (a.n <= kWarpRow || (a.n <= kLoneRow && a.rows >= 8 * sms)) {
        const int chunks = (a.n + kChunk - 1) / kChunk, warps = chunks <= kWarpChunks ? 4 : 2;
        const int warp_bytes = (int)sizeof(Lists) + chunks * kChunk * 4;
        auto *kernel = chunks <= 2 * kWarpChunks ? sample_warp_kernel<T, 2> : sample_warp_kernel<T, 8>;
        kernel<<<(unsigned int)((a.rows + warps - 1) / warps), warps * 32, warps * warp_bytes, stream>>>(a, chunks, warp_bytes);
        return cudaGetLastError();
    }
    const bool shared = a.n <= kMaxCluster * kBlockRow;
    auto warps_for = [&](int c) { return (a.n + c * kWarpRow - 1) / (c * kWarpRow); };
    int cs = 1;
    while (cs < kMaxCluster && (warps_for(cs) > 32 || (a.rows * cs < sms && warps_for(cs) > 8))) cs *= 2;
    const int warps = shared ? warps_for(cs) : 32;
    const int chunks = shared ? kWarpChunks : (a.n + warps * cs * kChunk - 1) / (warps * cs * kChunk);
    long long clusters = a.rows < (1ll << 27) ? a.rows : (1ll << 27);
    void *store = nullptr;
    if (!shared) {
        if (clusters > sms / cs) clusters = sms / cs;
        cudaMemPool_t pool = nullptr;
        if (library_pool(device, &pool)) return cudaErrorMemoryAllocation;
        const cudaError_t e = cudaMallocFromPoolAsync(&store, (size_t)clusters * chunks * kChunk * warps * cs * 4, pool, stream);
        if (e != cudaSuccess) return e;
        a.store = static_cast<unsigned int *>(store);
    }
    auto *kernel = shared ? sample_block_kernel<T, true> : sample_block_kernel<T, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned int)(clusters * cs));
    cfg.blockDim = dim3(warps * 32);
    cfg.dynamicSmemBytes = shared ? (size_t)warps * kWarpRow * 4 : 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaSuccess;
    if (cfg.dynamicSmemBytes > 32 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlockRow * 4);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kernel, a, cs, chunks);
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
    // four elements at a time
    const size_t four = 4 * dtype_bytes(logits->dtype);
    a.aligned = aligned_to(a.x, four) && (a.rows == 1 || a.stride % 4 == 0);
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
