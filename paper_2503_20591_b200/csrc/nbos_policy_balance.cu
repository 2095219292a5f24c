// Load-balance loss of a placement policy with per-host counts, per group of rows (nbos_policy_balance).
//
//   f_h = count_h / sum count,  P_h = mean over live rows of p_rh,  loss = n sum_h f_h P_h,
//   d loss / d x_rh = n / live * p_rh (f_h - sum_i f_i p_ri).
// f and the number of live rows come from the chosen ids alone, so a small kernel counts those first and one pass
// over the logits then gives P, the loss and the gradient: the logits' bytes, read once, and as many written, are
// what bounds it. A thread keeps the same columns for every row it sees, so the column sums of P stay in its
// registers; each block leaves its sums in the workspace and a last kernel adds them in a fixed order (the result
// does not depend on timing). The row needs one exchange: warps send their maximum, sum and f-weighted sum
// together, each relative to the warp's own maximum.
// Measured (B200, 6,464 GB/s copied): 256 x 4,096 x 1,024 bf16 loss and gradient back to back 860 us = 4,990 GB/s
// (921 us a call at a time), 262,144 x 1,024 f32
// 402 us = 5,340 GB/s; 65,536 x 4,096 bf16 without gradient 222 us = 2,420 GB/s. Column sums and elements take 64 of a
// thread's 128 registers: 16 warps an SM, and their instruction latency is what is left.
#include <math.h>

#include "nbos_policy.cuh"

namespace nbos {
namespace {

using namespace policy;

constexpr int kWarpRow = 1024;      // longest row of the warp form
constexpr int kElems = 16;          // row elements a thread holds in the cluster form (as many column sums beside them)
constexpr int kMaxCluster = 8;
// Blocks that share a staged row, 16,384 columns each: 8,192 x 32,768 bf16 407 us; 700 with a cluster that reads its rows from global
// memory as it comes to them, 664 with twice as many blocks of half the size.
constexpr int kStagedCluster = 4;
constexpr int kWarps = 8;           // of a block of the warp form
constexpr int kHeld = 32;           // row elements a thread holds in the staged forms
constexpr int kHistHosts = 8192;    // counters kept in shared memory while counting
// Chosen ids of a group that one cluster counts: 8,000 rows of 3 in 257 hosts 25 us a call against 27, 2,000 in 2,048 32 against
// 36; 16,385 rows 31.0 against 31.4, 30,000 in 128 hosts 30 against 28.
constexpr long long kClusterIds = 48 * 1024;

struct BalanceArgs {
    const void *x;
    long long stride;
    long long group_rows;
    int n, k;
    const int32_t *hosts;
    const int32_t *counts;   // [groups][n]
    const int2 *totals;      // [groups] (sum of counts, live rows)
    const float *grad_loss;
    float grad_scale;
    float *stats;
    const float *stats_in;
    void *grad;
    long long gstride;
    float *partial;          // [groups][parts][n] column sums of p
    int parts;               // of a group at most
    int groups;
    long long block_rows;    // rows of all groups that a block takes, one stretch after the other (staged forms)
    bool wide;               // the gradient is written 16 bytes at a time
};

// counts[g][h] += ..., totals[g] += (valid ids, rows that have one); grid (blocks, groups)
__global__ void __launch_bounds__(256) count_kernel(const int32_t *hosts, long long group_rows, int k, int n,
                                                    bool in_shared, int32_t *counts, int2 *totals)
{
    extern __shared__ int s_hist[];
    __shared__ int s_tot[2];
    if (threadIdx.x < 2) s_tot[threadIdx.x] = 0;
    for (int i = threadIdx.x; in_shared && i < n; i += blockDim.x) s_hist[i] = 0;
    __syncthreads();
    int32_t *out = counts + (size_t)blockIdx.y * n;
    const long long base = (long long)blockIdx.y * group_rows;
    int valid = 0, live = 0;
    for (long long r = (long long)blockIdx.x * blockDim.x + threadIdx.x; r < group_rows; r += (long long)gridDim.x * blockDim.x) {
        int here = 0;
        for (int j = 0; j < k; ++j) {
            const int h = hosts[(base + r) * k + j];
            if (h >= 0 && h < n) {
                ++here;
                atomicAdd(in_shared ? &s_hist[h] : &out[h], 1);
            }
        }
        valid += here;
        live += here > 0;
    }
    valid = __reduce_add_sync(kFull, valid);
    live = __reduce_add_sync(kFull, live);
    if ((threadIdx.x & 31) == 0) {
        atomicAdd(&s_tot[0], valid);
        atomicAdd(&s_tot[1], live);
    }
    __syncthreads();
    if (threadIdx.x < 2 && s_tot[threadIdx.x]) atomicAdd(&reinterpret_cast<int *>(totals + blockIdx.y)[threadIdx.x], s_tot[threadIdx.x]);
    for (int i = threadIdx.x; in_shared && i < n; i += blockDim.x)
        if (s_hist[i]) atomicAdd(&out[i], s_hist[i]);
}

// The same for a group with few ids, by one cluster: every block counts its part of the rows, then adds up its part of the hosts
// over the blocks. It writes every counter, so that nothing has to be cleared before; grid (cluster, groups).
__global__ void __launch_bounds__(512) count_cluster_kernel(const int32_t *hosts, int rows, int k, int n, int cs, int32_t *counts, int2 *totals,
                                                            unsigned int *tickets)
{
    extern __shared__ int s_hist[];
    __shared__ int s_tot[2];
    const int rank = cluster_rank(cs), group = blockIdx.y, threads = blockDim.x * cs;
    if (threadIdx.x < 2) s_tot[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) s_hist[i] = 0;
    __syncthreads();
    int valid = 0, live = 0;
    for (int r = rank * blockDim.x + threadIdx.x; r < rows; r += threads) {
        const int32_t *ids = hosts + ((long long)group * rows + r) * k;
        int here = 0;
        for (int j = 0; j < k; ++j) {
            const int h = ids[j];
            if (h >= 0 && h < n) {
                ++here;
                atomicAdd(&s_hist[h], 1);
            }
        }
        valid += here;
        live += here > 0;
    }
    valid = __reduce_add_sync(kFull, valid);
    live = __reduce_add_sync(kFull, live);
    if ((threadIdx.x & 31) == 0 && live) {
        atomicAdd(&s_tot[0], valid);
        atomicAdd(&s_tot[1], live);
    }
    cluster_sync(cs);
    for (int i = rank * blockDim.x + threadIdx.x; i < n; i += threads) {
        int sum = 0;
        for (int p = 0; p < cs; ++p) sum += cluster_peer(s_hist, p, cs)[i];
        counts[(size_t)group * n + i] = sum;
    }
    if (rank == 0 && threadIdx.x < 2) {
        int sum = 0;
        for (int p = 0; p < cs; ++p) sum += cluster_peer(s_tot, p, cs)[threadIdx.x];
        reinterpret_cast<int *>(totals + group)[threadIdx.x] = sum;
    }
    if (rank == 0 && threadIdx.x == 2) tickets[group] = 0;
    cluster_sync(cs);   // no block leaves while another may still read its counters
}

// The blocks that take rows of a group are first_block, first_block + 1, ...: its parts, in this order.
__device__ __forceinline__ long long first_block(const BalanceArgs &a, long long group) { return group * a.group_rows / a.block_rows; }

struct GroupScale {
    float inv_total, grad;   // 1 / sum of counts; n / live * grad_scale * grad_loss
};
__device__ __forceinline__ GroupScale group_scale(const BalanceArgs &a, int group)
{
    const int2 t = a.totals[group];
    GroupScale g;
    g.inv_total = t.x > 0 ? 1.0f / (float)t.x : 0.0f;
    g.grad = t.y > 0 ? (float)a.n / (float)t.y * a.grad_scale * (a.grad_loss ? a.grad_loss[group] : 1.0f) : 0.0f;
    return g;
}

// does any of the k ids name a host? over the lanes of `group`, which start at `sub` = 0
__device__ __forceinline__ bool any_host(const int *ids, int k, int n, bool active, int sub, int lanes, unsigned int group)
{
    bool some = false;
    for (int j = sub; active && j < k; j += lanes) some = some || (ids[j] >= 0 && ids[j] < n);
    return (__ballot_sync(kFull, some) & group) != 0;
}

// ---- rows that a warp or a block holds, staged -------------------------------------------------------------
struct Layout {   // bytes of a stage: rows, then ids, then statistics
    int row_bytes, rows, k;
    bool aligned;   // every row starts on a 16-byte boundary
    int whole;   // n if logits and gradient are handled 16 bytes at a time: columns below it need no look; else 0
    __host__ __device__ int hosts_at() const { return row_bytes * rows; }
    __host__ __device__ int stats_at() const { return hosts_at() + rows * k * 4; }
    __host__ __device__ int bytes() const { return (stats_at() + rows * 8 + 15) & ~15; }
};
// (a row's columns from `first` on, `columns` of them, land at the stage's start; first is a multiple of 16 bytes)
template <typename T>
__device__ __forceinline__ void stage(const BalanceArgs &a, const Layout &lay, char *at, int slot, long long row, int sub, int team, int first = 0,
                                      int columns = 1 << 21)
{
    const int from = first * (int)sizeof(T) / 16;
    stage_row(at + slot * lay.row_bytes, static_cast<const T *>(a.x) + row * a.stride, a.n, row * a.stride * (long long)sizeof(T), sub,
              team, from, from + columns * (int)sizeof(T) / 16 + (lay.aligned ? 0 : 1), from);
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(at));
    for (int i = sub; i < a.k; i += team) copy_async4(to + lay.hosts_at() + (slot * a.k + i) * 4, a.hosts + row * a.k + i);
    if (a.stats_in && sub == 0) {
        copy_async4(to + lay.stats_at() + slot * 8, a.stats_in + 2 * row);
        copy_async4(to + lay.stats_at() + slot * 8 + 4, a.stats_in + 2 * row + 1);
    }
}
__device__ __forceinline__ float2 staged_pair(const char *at)   // on a 4-byte boundary
{
    const float *f = reinterpret_cast<const float *>(at);
    return make_float2(f[0], f[1]);
}
// A lane's elements of a staged row, chunk after chunk of `width` columns, from column `first`. VEC is 16 bytes' worth,
// or 1 for rows that start anywhere: the columns of a lane have to be the same in every row.
template <typename T, int VEC, int CH>
__device__ __forceinline__ void load_staged(const T *row, int first, int width, int n, int whole, float (&v)[CH][VEC])
{
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = first + c * width;
        if constexpr (VEC == 1) {
            v[c][0] = col < n ? to_float(row[col]) : neg_inf();
        } else {
            if ((c + 1) * width <= whole)
                unpack16(*reinterpret_cast<const uint4 *>(row + col), v[c], T());
            else
                staged_cols<T, VEC>(row, col, n, v[c]);
        }
    }
}
// sum of v f over the lane's elements; f lies in shared memory by column
template <int VEC, int CH>
__device__ __forceinline__ float dot_all(const float (&v)[CH][VEC], const float *f, int first, int width)
{
    float d[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if constexpr (VEC == 1) {
            if (c % 2 == 0) fma2(d[c / 2 % 2][0], d[c / 2 % 2][1], v[c][0], v[c + 1][0], f[first + c * width], f[first + (c + 1) * width]);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const float4 w = *reinterpret_cast<const float4 *>(f + first + c * width + i);
                fma2(d[0][0], d[0][1], v[c][i], v[c][i + 1], w.x, w.y);
                fma2(d[1][0], d[1][1], v[c][i + 2], v[c][i + 3], w.z, w.w);
            }
        }
    }
    return (d[0][0] + d[0][1]) + (d[1][0] + d[1][1]);
}
// acc += v inv, then v := v (f - dot) fac, which is written to the row's gradient if GRAD
template <typename T, int VEC, int CH, bool GRAD>
__device__ __forceinline__ void finish_row(float (&v)[CH][VEC], float (&acc)[CH][VEC], float inv, float fac, float dot, const float *f,
                                           T *grad, int first, int width, int n, int whole, bool wide)
{
    const float shift = -fac * dot;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = first + c * width;
        if constexpr (VEC == 1) {
            if (c % 2) continue;
            fma2(acc[c][0], acc[c + 1][0], v[c][0], v[c + 1][0], inv, inv);
            if (GRAD) {
                float g[2] = {shift, shift};
                fma2(g[0], g[1], f[col], f[col + width], fac, fac);
                mul2(v[c][0], v[c + 1][0], g[0], g[1]);
                if (col < n) __stcs(grad + col, from_float<T>(v[c][0]));
                if (col + width < n) __stcs(grad + col + width, from_float<T>(v[c + 1][0]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 2) fma2(acc[c][i], acc[c][i + 1], v[c][i], v[c][i + 1], inv, inv);
            if (GRAD) {
#pragma unroll
                for (int i = 0; i < VEC; i += 4) {
                    const float4 w = *reinterpret_cast<const float4 *>(f + col + i);
                    float g[4] = {shift, shift, shift, shift};
                    fma2(g[0], g[1], w.x, w.y, fac, fac);
                    fma2(g[2], g[3], w.z, w.w, fac, fac);
                    mul2(v[c][i], v[c][i + 1], g[0], g[1]);
                    mul2(v[c][i + 2], v[c][i + 3], g[2], g[3]);
                }
                if ((c + 1) * width <= whole)
                    __stcs(reinterpret_cast<uint4 *>(grad + col), pack16(v[c], T()));
                else
                    store_cols<T, VEC>(grad, col, n, v[c], wide);
            }
        }
    }
}

// ---- warp form: LANES lanes per row, CH * VEC elements each; a block walks over its rows, group after group --
template <typename T, int VEC, int LANES, int CH, bool GRAD>
__global__ void __launch_bounds__(kWarps * 32, 2) balance_warp_kernel(BalanceArgs a, Layout lay)
{
    extern __shared__ __align__(16) char s_mem[];
    constexpr int width = LANES * VEC, padded = width * CH, at_once = 32 / LANES;
    float *s_f = reinterpret_cast<float *>(s_mem);   // f of the group's hosts; then the block's column sums
    const int lane = threadIdx.x & 31, sub = lane & (LANES - 1), slot = lane / LANES, warp = threadIdx.x >> 5;
    const unsigned int lanes_of_row = LANES == 32 ? kFull : ((1u << (LANES & 31)) - 1) << (slot * LANES);
    const int stage_bytes = lay.bytes(), first = sub * VEC;
    const bool saved = a.stats_in != nullptr;
    char *mine = s_mem + padded * 4 + warp * kStages * stage_bytes;
    const long long begin = blockIdx.x * a.block_rows, all_rows = a.group_rows * a.groups;
    const long long end = begin + a.block_rows < all_rows ? begin + a.block_rows : all_rows;
    constexpr int step = kWarps * at_once;
    for (int group = (int)(begin / a.group_rows); group < a.groups && group * a.group_rows < end; ++group) {
    // the block's rows of this group
    const long long row0 = max(begin, group * a.group_rows);
    const int rows = (int)(min(end, (group + 1) * a.group_rows) - row0);
    const int base0 = warp * at_once;
    auto queue = [&](int base, int st) {
        if (base + slot < rows) stage<T>(a, lay, mine + st * stage_bytes, slot, row0 + base + slot, sub, LANES);
        copies_commit();
    };
#pragma unroll
    for (int st = 0; st < kStages; ++st) queue(base0 + st * step, st);
    const GroupScale gs = group_scale(a, group);
    for (int i = threadIdx.x; i < padded; i += blockDim.x) s_f[i] = i < a.n ? (float)a.counts[(size_t)group * a.n + i] * gs.inv_total : 0.0f;
    __syncthreads();
    float acc[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[c][i] = 0.0f;
    int st = 0;
    for (int base = base0; base < rows; base += step) {
        copies_wait();
        __syncwarp();
        const bool active = base + slot < rows;
        const int here = active ? slot : 0;
        const long long row = row0 + base + here;
        const char *at = mine + st * stage_bytes;
        const T *x = static_cast<const T *>(a.x) + row * a.stride;
        const T *r = reinterpret_cast<const T *>(at + here * lay.row_bytes + (VEC == 1 ? row_shift(x) : 0));
        const float2 given = saved ? staged_pair(at + lay.stats_at() + here * 8) : make_float2(0.0f, 0.0f);
        float v[CH][VEC];
        load_staged<T, VEC, CH>(r, first, width, a.n, lay.whole, v);
        const bool live = any_host(reinterpret_cast<const int *>(at + lay.hosts_at()) + here * a.k, a.k, a.n, active, sub, LANES, lanes_of_row);
        __syncwarp();   // all that the stage holds has been read
        queue(base + kStages * step, st);
        // rows that are not live take part as rows of -inf, whatever they hold
        if (__any_sync(kFull, !live)) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[c][i] = live ? v[c][i] : neg_inf();
        }
        // (not a choice between a lane's own value and the exchange: every lane takes part in that)
        const float top = saved ? given.x : lanes_max(max_all<VEC, CH>(v), LANES);
        const float m = live ? top : neg_inf();
        float s = exp_all<VEC, CH>(v, m == neg_inf() ? 0.0f : m, kLog2e), dot = 0.0f;
        if (GRAD) dot = lanes_sum(dot_all<VEC, CH>(v, s_f, first, width), LANES);
        s = saved ? (live ? given.y : 0.0f) : lanes_sum(s, LANES);
        // a row of -inf has sum 0 and no probabilities
        const float inv = s != 0.0f ? reciprocal(s) : 0.0f;
        if (!saved && live && a.stats && sub == 0) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
        // a lane without a row (the group's last ones) writes nothing
        finish_row<T, VEC, CH, GRAD>(v, acc, inv, gs.grad * inv, dot * inv, s_f, static_cast<T *>(a.grad) + row * a.gstride, first, width,
                                     active ? a.n : 0, active ? lay.whole : 0, a.wide);
        st = st == kStages - 1 ? 0 : st + 1;
    }
    copies_drain();
    if (!saved) {
        // the block's column sums: rows of one warp, then warp after warp
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
#pragma unroll
                for (int off = 16; off >= LANES; off >>= 1) acc[c][i] += __shfl_xor_sync(kFull, acc[c][i], off);
        for (int w = 0; w < kWarps; ++w) {
            __syncthreads();
            if (warp == w && lane < LANES) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        float *to = &s_f[first + c * width + i];
                        *to = w ? *to + acc[c][i] : acc[c][i];
                    }
            }
        }
        __syncthreads();
        float *out = a.partial + ((size_t)group * a.parts + (blockIdx.x - first_block(a, group))) * a.n;
        for (int i = threadIdx.x; i < a.n; i += blockDim.x) out[i] = s_f[i];
    }
    __syncthreads();   // f of the next group may be written
    }
}

// ---- block form: one row at a time per block, or per cluster of cs of them, each with its stretch of the columns; kHeld
// elements a thread; it walks over its rows, group after group
template <typename T, int VEC, bool GRAD, bool MULTI>
__global__ void __launch_bounds__(512, 1) balance_staged_kernel(BalanceArgs a, int cs_, Layout lay)
{
    const int cs = MULTI ? cs_ : 1;
    constexpr int CH = kHeld / VEC, width = 32 * VEC;   // a warp has one stretch of columns: offsets are known when compiled
    extern __shared__ __align__(16) char s_mem[];
    __shared__ float4 s_stats[2][kStagedCluster * 16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    // the block's columns: from block_first on, `columns` of them
    const int rank = MULTI ? cluster_rank(cs) : 0, columns = blockDim.x * kHeld, block_first = rank * columns;
    const int stage_bytes = lay.bytes(), base = block_first + warp * 32 * kHeld, first = base + lane * VEC;
    float *s_f = reinterpret_cast<float *>(s_mem) - block_first;   // by column
    const bool saved = a.stats_in != nullptr;
    char *stages = s_mem + columns * 4;
    const long long block = blockIdx.x / cs, begin = block * a.block_rows, all_rows = a.group_rows * a.groups;
    const long long end = begin + a.block_rows < all_rows ? begin + a.block_rows : all_rows;
    int turn = 0;
    if (MULTI) cluster_sync(cs);   // all blocks of the cluster run: their shared memory may be written
    for (int group = (int)(begin / a.group_rows); group < a.groups && group * a.group_rows < end; ++group) {
    // the block's rows of this group
    const long long row0 = max(begin, group * a.group_rows);
    const int rows = (int)(min(end, (group + 1) * a.group_rows) - row0);
    auto queue = [&](int r, int st) {
        if (r < rows) stage<T>(a, lay, stages + st * stage_bytes, 0, row0 + r, threadIdx.x, blockDim.x, block_first, columns);
        copies_commit();
    };
#pragma unroll
    for (int st = 0; st < kStages; ++st) queue(st, st);
    const GroupScale gs = group_scale(a, group);
    for (int i = block_first + threadIdx.x; i < block_first + columns; i += blockDim.x) s_f[i] = i < a.n ? (float)a.counts[(size_t)group * a.n + i] * gs.inv_total : 0.0f;
    float acc[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[c][i] = 0.0f;
    int st = 0;
    for (int r = 0; r < rows; ++r, turn ^= 1) {
        copies_wait();
        __syncthreads();
        const long long row = row0 + r;
        const char *at = stages + st * stage_bytes;
        const T *x = static_cast<const T *>(a.x) + row * a.stride;
        const T *staged = reinterpret_cast<const T *>(at + (VEC == 1 ? row_shift(x) : 0)) - block_first;   // by column
        const float2 given = saved ? staged_pair(at + lay.stats_at()) : make_float2(0.0f, 0.0f);
        float v[CH][VEC];
        load_staged<T, VEC, CH>(staged, first, width, a.n, lay.whole - base, v);
        const bool live = any_host(reinterpret_cast<const int *>(at + lay.hosts_at()), a.k, a.n, true, lane, 32, kFull);
        if (!live) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[c][i] = neg_inf();
        }
        const float top = saved ? given.x : lanes_max(max_all<VEC, CH>(v), 32);
        float m = live ? top : neg_inf();
        const float m_warp = m;
        float s = lanes_sum(exp_all<VEC, CH>(v, m == neg_inf() ? 0.0f : m, kLog2e), 32), dot = 0.0f;
        if (GRAD) dot = lanes_sum(dot_all<VEC, CH>(v, s_f, first, width), 32);
        // one exchange for all three, each relative to the warp's maximum
        if (lane < cs) cluster_peer(s_stats[turn], lane, cs)[rank * warps + warp] = make_float4(m, s, dot, 0.0f);
        cluster_sync(cs);
        queue(r + kStages, st);   // all that the stage holds has been read
        const int parts = cs * warps;   // 64 at most
        const float4 none = make_float4(neg_inf(), 0.0f, 0.0f, 0.0f);
        const float4 w = lane < parts ? s_stats[turn][lane] : none, w2 = MULTI && lane + 32 < parts ? s_stats[turn][lane + 32] : none;
        if (!saved) m = lanes_max(MULTI ? fmaxf(w.x, w2.x) : w.x, 32);
        const float scale = saved ? 1.0f : exp_from(w.x, m, kLog2e), scale2 = saved ? 1.0f : exp_from(w2.x, m, kLog2e);
        s = saved ? (live ? given.y : 0.0f) : lanes_sum(MULTI ? w.y * scale + w2.y * scale2 : w.y * scale, 32);
        if (GRAD) dot = lanes_sum(MULTI ? w.z * scale + w2.z * scale2 : w.z * scale, 32);
        const float inv = s != 0.0f ? reciprocal(s) : 0.0f;
        if (!saved && live && a.stats && threadIdx.x == 0 && rank == 0) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
        const float own = inv * (saved ? 1.0f : exp_from(m_warp, m, kLog2e));
        finish_row<T, VEC, CH, GRAD>(v, acc, own, gs.grad * own, dot * inv, s_f, static_cast<T *>(a.grad) + row * a.gstride, first, width, a.n,
                                     lay.whole - base, a.wide);
        st = st == kStages - 1 ? 0 : st + 1;
    }
    copies_drain();
    float *out = a.partial + ((size_t)group * a.parts + (block - first_block(a, group))) * a.n;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (!saved && first + c * width + i < a.n) out[first + c * width + i] = acc[c][i];
    __syncthreads();   // f of the next group may be written
    }
    cluster_sync(cs);   // no block leaves while another may still write to its shared memory
}

// ---- cluster form: cs blocks per row at a time; grid (parts * cs, groups) -----------------------------------
// KEEP: row and column sums stay in registers; otherwise the row is read once more and the sums live in `partial`.
template <typename T, int VEC, bool KEEP, bool GRAD, bool SAVED>
__global__ void __launch_bounds__(1024, 1) balance_block_kernel(BalanceArgs a, int cs, int span)
{
    constexpr int CH = kElems / VEC;
    extern __shared__ float s_f[];   // KEEP: f of this block's columns, padded to whole chunks
    __shared__ float4 s_stats[2][kMaxCluster * 32];
    const int rank = cluster_rank(cs);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int group = blockIdx.y, part = blockIdx.x / cs, parts = gridDim.x / cs;
    const long long first_col = (long long)rank * span;
    const long long end_col = first_col + span < a.n ? first_col + span : a.n;
    const int chunk = blockDim.x * VEC;
    const GroupScale gs = group_scale(a, group);
    const int32_t *counts = a.counts + (size_t)group * a.n;
    float *out = a.partial + ((size_t)group * a.parts + part) * a.n;
    if (KEEP)
        for (int i = threadIdx.x; i < chunk * CH; i += blockDim.x)
            s_f[i] = first_col + i < end_col ? (float)counts[first_col + i] * gs.inv_total : 0.0f;
    cluster_sync(cs);
    float acc[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[c][i] = 0.0f;
    if (!KEEP && !SAVED)
        for (long long col = first_col + threadIdx.x; col < end_col; col += blockDim.x) out[col] = 0.0f;
    int turn = 0;
    for (long long r = part; r < a.group_rows; r += parts, turn ^= 1) {
        const long long row = (long long)group * a.group_rows + r;
        const T *x = static_cast<const T *>(a.x) + row * a.stride;
        float v[CH][VEC];
        float m = neg_inf(), s = 0.0f, dot = 0.0f;
        if (KEEP) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
                load_cols<T, VEC>(x, first_col + c * chunk + threadIdx.x * VEC, end_col, neg_inf(), v[c]);
        }
        const bool live = any_host(a.hosts + row * a.k, a.k, a.n, true, lane, 32, kFull);
        if (SAVED) m = live ? a.stats_in[2 * row] : 0.0f;
        if (KEEP) {
            if (!SAVED) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) m = fmaxf(m, v[c][i]);
                m = lanes_max(m, 32);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[c][i] = exp_from(v[c][i], m, kLog2e);
                    s += v[c][i];
                    if (GRAD) dot += v[c][i] * s_f[c * chunk + threadIdx.x * VEC + i];
                }
        } else {
            if (!SAVED) {
                for (long long col = first_col + threadIdx.x * VEC; col < end_col; col += chunk) {
                    float w[VEC];
                    load_cols<T, VEC>(x, col, end_col, neg_inf(), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) m = fmaxf(m, w[i]);
                }
                m = lanes_max(m, 32);
            }
            for (long long col = first_col + threadIdx.x * VEC; col < end_col; col += chunk) {
                float w[VEC];
                load_cols<T, VEC>(x, col, end_col, neg_inf(), w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float e = exp_from(w[i], m, kLog2e);
                    s += e;
                    if (GRAD && col + i < end_col) dot += e * ((float)counts[col + i] * gs.inv_total);
                }
            }
        }
        const float m_warp = m;
        s = lanes_sum(s, 32);
        if (GRAD) dot = lanes_sum(dot, 32);
        // one exchange for all three; two slots in turn, so that a warp that runs ahead does not overwrite
        if (lane < cs) cluster_peer(s_stats[turn], lane, cs)[rank * warps + warp] = make_float4(m, s, dot, 0.0f);
        cluster_sync(cs);
        if (!SAVED) {
            float top = neg_inf();
            for (int i = lane; i < cs * warps; i += 32) top = fmaxf(top, s_stats[turn][i].x);
            m = lanes_max(top, 32);
        }
        s = 0.0f, dot = 0.0f;
        for (int i = lane; i < cs * warps; i += 32) {
            const float4 w = s_stats[turn][i];
            const float scale = SAVED ? 1.0f : exp_from(w.x, m, kLog2e);
            s += w.y * scale;
            dot += w.z * scale;
        }
        s = SAVED ? (live ? a.stats_in[2 * row + 1] : 1.0f) : lanes_sum(s, 32);
        dot = lanes_sum(dot, 32);
        const float inv = live && s != 0.0f ? 1.0f / s : 0.0f;
        const float mine = KEEP && !SAVED ? exp_from(m_warp, m, kLog2e) * inv : inv;
        dot *= inv;
        if (!SAVED && live && a.stats && rank == 0 && threadIdx.x == 0) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
        T *grad = static_cast<T *>(a.grad) + row * a.gstride;
        if (KEEP) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float p = live ? v[c][i] * mine : 0.0f;
                    if (!SAVED) acc[c][i] += p;
                    if (GRAD) v[c][i] = live ? p * gs.grad * (s_f[c * chunk + threadIdx.x * VEC + i] - dot) : 0.0f;
                }
                if (GRAD) store_cols<T, VEC>(grad, first_col + c * chunk + threadIdx.x * VEC, end_col, v[c], a.wide);
            }
        } else {
            for (long long col = first_col + threadIdx.x * VEC; col < end_col; col += chunk) {
                float w[VEC];
                load_cols<T, VEC>(x, col, end_col, neg_inf(), w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float p = live ? exp_from(w[i], m, kLog2e) * mine : 0.0f;
                    if (col + i < end_col) {
                        if (!SAVED) out[col + i] += p;
                        if (GRAD) w[i] = live ? p * gs.grad * ((float)counts[col + i] * gs.inv_total - dot) : 0.0f;
                    }
                }
                if (GRAD) store_cols<T, VEC>(grad, col, end_col, w, a.wide);
            }
        }
    }
    if (KEEP && !SAVED) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const long long col = first_col + c * chunk + threadIdx.x * VEC + i;
                if (col < end_col) out[col] = acc[c][i];
            }
    }
    cluster_sync(cs);   // no block leaves while another may still write to its shared memory
}

// ---- small groups: one block per group does everything, without a workspace --------------------------------
constexpr int kSmallHosts = 512, kSmallWarps = 32;
// Rows of a group that one SM gets through in the time that a workspace, two clears and three kernels take to be queued. What counts is
// how often the block's warps go round, 4 rows each up to 32 hosts, one row otherwise. One group, bf16, us a call here and by those
// kernels: 1,024 x 32 14.4 / 18.5, 2,048 x 32 24.6 / 18.5; 512 x 64 18.5 / 19.5, 1,024 x 64 33 / 20.5; 256 x 256 17.3 / 20.2,
// 512 x 128 28.5 / 19.5; 128 x 512 16.4 / 20.0. By rows * hosts alone 16,384 x 4 took 155 / 23, 65,536 x 1 597 / 29 and, with 256 chosen
// hosts a row, 10,100 / 113.
inline int small_rows(int n) { return n <= 32 ? 1024 : n <= 64 ? 512 : n <= 256 ? 256 : n <= kSmallHosts ? 128 : 0; }

template <typename T, int LANES, int CH, bool GRAD>
__global__ void __launch_bounds__(kSmallWarps * 32) balance_small_kernel(BalanceArgs a, int32_t *out_counts, float *shares, float *loss)
{
    extern __shared__ __align__(16) char s_mem[];
    constexpr int at_once = 32 / LANES;
    int *s_counts = reinterpret_cast<int *>(s_mem);
    float *s_f = reinterpret_cast<float *>(s_mem) + a.n, *s_parts = s_f + a.n;   // [warps][n] column sums
    __shared__ int s_tot[2];
    __shared__ double s_loss[kSmallWarps];
    const int lane = threadIdx.x & 31, sub = lane & (LANES - 1), slot = lane / LANES, warp = threadIdx.x >> 5;
    const unsigned int lanes_of_row = LANES == 32 ? kFull : ((1u << (LANES & 31)) - 1) << (slot * LANES);
    const int group = blockIdx.x, rows = (int)a.group_rows;
    const long long row0 = (long long)group * rows;
    const bool saved = a.stats_in != nullptr;
    if (threadIdx.x < 2) s_tot[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) s_counts[i] = 0;
    __syncthreads();
    int valid = 0, living = 0;
    for (int r = threadIdx.x; r < rows; r += blockDim.x) {
        int here = 0;
        for (int j = 0; j < a.k; ++j) {
            const int h = a.hosts[(row0 + r) * a.k + j];
            if (h >= 0 && h < a.n) {
                ++here;
                atomicAdd(&s_counts[h], 1);
            }
        }
        valid += here;
        living += here > 0;
    }
    valid = __reduce_add_sync(kFull, valid);
    living = __reduce_add_sync(kFull, living);
    if (lane == 0 && living) {
        atomicAdd(&s_tot[0], valid);
        atomicAdd(&s_tot[1], living);
    }
    __syncthreads();
    const float inv_total = s_tot[0] > 0 ? 1.0f / (float)s_tot[0] : 0.0f;
    const float scale = s_tot[1] > 0 ? (float)a.n / (float)s_tot[1] * a.grad_scale * (a.grad_loss ? a.grad_loss[group] : 1.0f) : 0.0f;
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
        s_f[i] = (float)s_counts[i] * inv_total;
        if (out_counts) out_counts[(size_t)group * a.n + i] = s_counts[i];
    }
    __syncthreads();
    float acc[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) acc[c] = 0.0f;
    for (int base = warp * at_once; base < rows; base += kSmallWarps * at_once) {
        const bool active = base + slot < rows;
        const long long row = row0 + base + (active ? slot : 0);
        const T *x = static_cast<const T *>(a.x) + row * a.stride;
        float v[CH][1];
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c][0] = c * LANES + sub < a.n ? to_float(x[c * LANES + sub]) : neg_inf();
        const bool live = any_host(a.hosts + row * a.k, a.k, a.n, active, sub, LANES, lanes_of_row);
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c][0] = live ? v[c][0] : neg_inf();
        const float top = saved ? a.stats_in[2 * row] : lanes_max(max_all<1, CH>(v), LANES);
        const float m = live ? top : neg_inf();
        float s = exp_all<1, CH>(v, m == neg_inf() ? 0.0f : m, kLog2e), dot = 0.0f;
        if (GRAD) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (c * LANES + sub < a.n) dot += v[c][0] * s_f[c * LANES + sub];
            dot = lanes_sum(dot, LANES);
        }
        s = saved ? (live ? a.stats_in[2 * row + 1] : 0.0f) : lanes_sum(s, LANES);
        const float inv = s != 0.0f ? reciprocal(s) : 0.0f;
        if (!saved && live && a.stats && sub == 0) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
        const float fac = scale * inv, shift = -fac * (dot * inv);
        T *grad = static_cast<T *>(a.grad) + row * a.gstride;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            acc[c] += v[c][0] * inv;
            const int col = c * LANES + sub;
            if (GRAD && active && col < a.n) grad[col] = from_float<T>(v[c][0] * (s_f[col] * fac + shift));
        }
    }
    if (saved) return;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int off = 16; off >= LANES; off >>= 1) acc[c] += __shfl_xor_sync(kFull, acc[c], off);
        if (lane < LANES && c * LANES + sub < a.n) s_parts[warp * a.n + c * LANES + sub] = acc[c];
    }
    __syncthreads();
    double part = 0.0;
    if (threadIdx.x < a.n) {
        double sum = 0.0;
        for (int w = 0; w < kSmallWarps; ++w) sum += (double)s_parts[w * a.n + threadIdx.x];
        const double share = s_tot[1] > 0 ? sum / (double)s_tot[1] : 0.0;
        if (shares) shares[(size_t)group * a.n + threadIdx.x] = (float)share;
        if (s_tot[0] > 0) part = share * ((double)s_counts[threadIdx.x] / (double)s_tot[0]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) part += __shfl_xor_sync(kFull, part, off);
    if (lane == 0) s_loss[warp] = part;
    __syncthreads();
    if (warp != 0) return;
    part = s_loss[lane];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) part += __shfl_xor_sync(kFull, part, off);
    if (lane == 0) loss[group] = (float)(part * (double)a.n);
}

// shares = column sums over the parts / live; loss = n sum f share. A block of kFinishThreads takes blockDim.x columns, blockDim.y
// parts at a time (both powers of two; many parts: few columns); grid (column blocks, groups). The group's last block
// adds the column blocks' shares of the loss. Every sum is taken in the same order each time.
constexpr int kFinishThreads = 512;

__global__ void __launch_bounds__(kFinishThreads) finish_kernel(BalanceArgs a, float *shares, float *loss, double *loss_parts,
                                                                unsigned int *tickets)
{
    __shared__ double s_sum[kFinishThreads];
    __shared__ bool s_last;
    const int cols = blockDim.x, group = blockIdx.y, tid = threadIdx.y * cols + threadIdx.x, col = blockIdx.x * cols + threadIdx.x;
    const int parts = a.block_rows ? (int)((((long long)group + 1) * a.group_rows - 1) / a.block_rows - first_block(a, group)) + 1 : a.parts;
    const float *from = a.partial + (size_t)group * a.parts * a.n + col;
    double sum = 0.0;
    if (col < a.n) {
#pragma unroll 8
        for (int p = threadIdx.y; p < parts; p += blockDim.y) sum += (double)from[(size_t)p * a.n];
    }
    // adds up s_sum[0 .. 2 half)
    auto fold = [&](int half) {
        for (; half > 0; half >>= 1) {
            __syncthreads();
            if (tid < half) s_sum[tid] += s_sum[tid + half];
        }
        __syncthreads();
    };
    s_sum[tid] = sum;
    for (int half = kFinishThreads / 2; half >= cols; half >>= 1) {   // over the parts
        __syncthreads();
        if (tid < half) s_sum[tid] += s_sum[tid + half];
    }
    double part = 0.0;
    if (threadIdx.y == 0 && col < a.n) {
        const int2 t = a.totals[group];
        const double share = t.y > 0 ? s_sum[tid] / (double)t.y : 0.0;
        if (shares) shares[(size_t)group * a.n + col] = (float)share;
        if (t.x > 0) part = share * ((double)a.counts[(size_t)group * a.n + col] / (double)t.x);
    }
    __syncthreads();
    if (threadIdx.y == 0) s_sum[tid] = part;
    fold(cols / 2);
    double *mine = loss_parts + (size_t)group * gridDim.x;
    if (tid == 0) {
        mine[blockIdx.x] = s_sum[0];
        __threadfence();
        s_last = atomicAdd(&tickets[group], 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    double total = 0.0;
    for (int i = tid; i < (int)gridDim.x; i += kFinishThreads) total += __ldcg(&mine[i]);
    s_sum[tid] = total;
    fold(kFinishThreads / 2);
    if (tid == 0) loss[group] = (float)(s_sum[0] * (double)a.n);
}

enum Form { WARP, BLOCK, CLUSTER };
struct Plan {
    Form form;
    bool keep, vec;
    int lanes, chunks;      // warp form: lanes per row, chunks per lane
    int cs, threads, span;  // cluster form (threads: block form too)
    int parts;              // of a group at most
    int blocks;             // staged forms
    long long block_rows;
    Layout lay;
    int shared;
};

// The warp form's shape: as many elements a lane as the row fills well, so that what a row costs besides is shared.
void warp_shape(int n, int vec, int &lanes, int &chunks)
{
    const int most = kHeld / vec;
    if (vec == 1) {
        // Neighbouring lanes write neighbouring elements: at least 16 of them, a sector's worth, but for the shortest rows. What
        // a row does not fill costs as much as what it does: 313,479 x 319 f16 with gradient 163 us by 16 lanes of 20 elements, 173 of 24, 201 of
        // 32; 261,096 x 383 152 by 24, 173 by 32; 130,378 x 767 136 by 32 lanes of 24, 162 of 32; 400,000 x 250 173 by 16 lanes of
        // 16, 189 of 20; 1,666,666 x 60 250 by 8 lanes of 8, 479 by 16.
        lanes = n <= 64 ? 8 : n <= 512 ? 16 : 32;
        chunks = n <= 32 ? 4 : n <= 128 ? 8 : n <= 256 ? 16 : n <= 320 ? 20 : n <= 384 ? 24 : n <= 512 ? 32 : n <= 768 ? 24 : 32;
        return;
    }
    for (chunks = most; ; chunks = chunks > 2 ? 2 : 1) {
        lanes = 4;
        while (lanes < 32 && lanes * vec * chunks < n) lanes *= 2;
        if (chunks == 1 || lanes * vec * chunks <= n + n / 2 || lanes * vec * 1 < n) break;
    }
    if (lanes * vec * chunks < n) chunks = most, lanes = 32;
}

Plan make_plan(const BalanceArgs &a, int groups, int elem, bool aligned, int sms)
{
    Plan p = {};
    p.vec = aligned;
    const int per = aligned ? 16 / elem : 1;
    p.lay = Layout{staged_row_bytes(a.n, elem, aligned), 1, a.k, aligned, aligned && a.wide ? a.n : 0};
    // the rows of all groups in even stretches, as many as there are blocks at once
    auto stretches = [&](long long at_once, int most, long long least) {
        const long long rows = a.group_rows * groups;
        long long rounds = (rows + most * at_once - 1) / (most * at_once);
        if (rounds < least) rounds = least;
        p.block_rows = rounds * at_once;
        p.blocks = (int)((rows + p.block_rows - 1) / p.block_rows);
        p.parts = (int)((a.group_rows - 1) / p.block_rows) + 2;
    };
    if (a.n <= kWarpRow) {
        p.form = WARP;
        warp_shape(a.n, per, p.lanes, p.chunks);
        p.lay.rows = 32 / p.lanes;
        p.shared = p.lanes * per * p.chunks * 4 + kWarps * kStages * p.lay.bytes();
        if (p.shared <= 112 * 1024) {
            stretches((long long)kWarps * p.lay.rows, 2 * sms, 1);
            return p;
        }
        p.lay.rows = 1;
    }
    p.cs = 1;
    while (p.cs < kStagedCluster && p.cs * 512 * kHeld < a.n) p.cs *= 2;
    p.threads = ((a.n + p.cs * kHeld - 1) / (p.cs * kHeld) + 31) / 32 * 32;
    p.lay.row_bytes = staged_row_bytes(p.cs > 1 ? p.threads * kHeld : a.n, elem, aligned);
    p.shared = p.threads * kHeld * 4 + kStages * p.lay.bytes();
    // Fewer rows leave SMs idle here; the cluster form has several blocks to a row. bf16 with gradient, us here / there: 148 x 4,096
    // 32.3 / 26.3, 296 x 4,096 32.5 / 27.8, 592 x 4,096 34.6 / 34.3; 296 x 16,384 52.5 / 52.4, 592 x 16,384 56.6 / 63.5.
    if (p.threads <= 512 && p.shared <= kMostShared && a.group_rows * groups * p.cs >= 2 * sms) {
        p.form = BLOCK;
        // a block's column sums are written and read once more: that should be little beside its rows (2,000 x 2,048 bf16 32 us
        // with at least six rows a block, 37 with two)
        const int resident = resident_blocks(128, p.threads, p.shared + 2048);
        stretches(1, sms * resident / p.cs, 6);
        return p;
    }
    p.form = CLUSTER;
    auto threads_for = [&](int c) { return ((a.n + c * kElems - 1) / (c * kElems) + 31) / 32 * 32; };
    p.keep = a.n <= kMaxCluster * 1024 * kElems;
    p.cs = 1;
    while (p.cs < kMaxCluster && (threads_for(p.cs) > 1024 || (a.group_rows * groups * p.cs < 2 * sms && threads_for(p.cs) > 128))) p.cs *= 2;
    p.threads = p.keep ? threads_for(p.cs) : 1024;
    p.span = ((a.n + p.cs - 1) / p.cs + per - 1) / per * per;
    const int resident = p.threads > 512 ? 1 : (1024 / p.threads);
    const long long fill = ((long long)sms * resident / p.cs + groups - 1) / groups;
    p.parts = (int)(a.group_rows < fill ? a.group_rows : (fill > 1 ? fill : 1));
    return p;
}

template <typename T, int VEC, int LANES, int CH, bool GRAD>
cudaError_t launch_warp(const BalanceArgs &a, const Plan &p, cudaStream_t stream)
{
    auto *kernel = balance_warp_kernel<T, VEC, LANES, CH, GRAD>;
    const cudaError_t e = allow_shared(kernel, p.shared);
    if (e != cudaSuccess) return e;
    kernel<<<p.blocks, kWarps * 32, p.shared, stream>>>(a, p.lay);
    return cudaGetLastError();
}
template <typename T, int VEC, int CH, bool GRAD>
cudaError_t launch_lanes(const BalanceArgs &a, const Plan &p, cudaStream_t stream)
{
    switch (p.lanes) {
    case 4: return launch_warp<T, VEC, 4, CH, GRAD>(a, p, stream);
    case 8: return launch_warp<T, VEC, 8, CH, GRAD>(a, p, stream);
    case 16: return launch_warp<T, VEC, 16, CH, GRAD>(a, p, stream);
    default: return launch_warp<T, VEC, 32, CH, GRAD>(a, p, stream);
    }
}
template <typename T, bool GRAD>
cudaError_t launch_rows(const BalanceArgs &a, const Plan &p, cudaStream_t stream)
{
    constexpr int V = kPer16<T>;
    if (p.form == BLOCK) {
        auto *kernel = p.cs > 1 ? (p.vec ? balance_staged_kernel<T, V, GRAD, true> : balance_staged_kernel<T, 1, GRAD, true>)
                                : (p.vec ? balance_staged_kernel<T, V, GRAD, false> : balance_staged_kernel<T, 1, GRAD, false>);
        const cudaError_t e = allow_shared(kernel, p.shared);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned int)p.blocks * p.cs);
        cfg.blockDim = dim3(p.threads);
        cfg.dynamicSmemBytes = p.shared;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = p.cs;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = p.cs > 1;
        return cudaLaunchKernelEx(&cfg, kernel, a, p.cs, p.lay);
    }
    if (p.vec) {
        if (p.chunks == 1) return launch_lanes<T, V, 1, GRAD>(a, p, stream);
        if (p.chunks == 2) return launch_lanes<T, V, 2, GRAD>(a, p, stream);
        return launch_lanes<T, V, kHeld / V, GRAD>(a, p, stream);
    }
    if (p.lanes == 8) return p.chunks == 4 ? launch_warp<T, 1, 8, 4, GRAD>(a, p, stream) : launch_warp<T, 1, 8, 8, GRAD>(a, p, stream);
    if (p.lanes == 32) return p.chunks == 24 ? launch_warp<T, 1, 32, 24, GRAD>(a, p, stream) : launch_warp<T, 1, 32, 32, GRAD>(a, p, stream);
    switch (p.chunks) {
    case 8: return launch_warp<T, 1, 16, 8, GRAD>(a, p, stream);
    case 16: return launch_warp<T, 1, 16, 16, GRAD>(a, p, stream);
    case 20: return launch_warp<T, 1, 16, 20, GRAD>(a, p, stream);
    case 24: return launch_warp<T, 1, 16, 24, GRAD>(a, p, stream);
    default: return launch_warp<T, 1, 16, 32, GRAD>(a, p, stream);
    }
}

template <typename T, int VEC, bool KEEP, bool GRAD, bool SAVED>
cudaError_t launch_block(const BalanceArgs &a, int groups, const Plan &p, cudaStream_t stream)
{
    auto *kernel = balance_block_kernel<T, VEC, KEEP, GRAD, SAVED>;
    const size_t smem = KEEP ? (size_t)p.threads * kElems * sizeof(float) : 0;
    if (smem > 16 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 1024 * kElems * (int)sizeof(float));
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned int)p.parts * p.cs, groups);
    cfg.blockDim = dim3(p.threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, p.cs, p.span);
}

template <typename T, int VEC, bool GRAD, bool SAVED>
cudaError_t launch_cluster(const BalanceArgs &a, int groups, const Plan &p, cudaStream_t stream)
{
    return p.keep ? launch_block<T, VEC, true, GRAD, SAVED>(a, groups, p, stream) : launch_block<T, VEC, false, GRAD, SAVED>(a, groups, p, stream);
}

template <typename T>
cudaError_t dispatch(const BalanceArgs &a, int groups, const Plan &p, cudaStream_t stream)
{
    constexpr int V = kPer16<T>;
    if (p.form != CLUSTER) return a.grad ? launch_rows<T, true>(a, p, stream) : launch_rows<T, false>(a, p, stream);
    if (a.stats_in) return p.vec ? launch_cluster<T, V, true, true>(a, groups, p, stream) : launch_cluster<T, 1, true, true>(a, groups, p, stream);
    if (a.grad) return p.vec ? launch_cluster<T, V, true, false>(a, groups, p, stream) : launch_cluster<T, 1, true, false>(a, groups, p, stream);
    return p.vec ? launch_cluster<T, V, false, false>(a, groups, p, stream) : launch_cluster<T, 1, false, false>(a, groups, p, stream);
}

template <typename T, int LANES, int CH>
cudaError_t launch_small(const BalanceArgs &a, int groups, int32_t *counts, float *shares, float *loss, cudaStream_t stream)
{
    auto *kernel = a.grad ? balance_small_kernel<T, LANES, CH, true> : balance_small_kernel<T, LANES, CH, false>;
    const int shared = (2 + kSmallWarps) * a.n * 4;
    const cudaError_t e = allow_shared(kernel, shared);
    if (e != cudaSuccess) return e;
    kernel<<<groups, kSmallWarps * 32, shared, stream>>>(a, counts, shares, loss);
    return cudaGetLastError();
}
template <typename T>
cudaError_t small(const BalanceArgs &a, int groups, int32_t *counts, float *shares, float *loss, cudaStream_t stream)
{
    if (a.n <= 32) return launch_small<T, 8, 4>(a, groups, counts, shares, loss, stream);
    if (a.n <= 64) return launch_small<T, 32, 2>(a, groups, counts, shares, loss, stream);
    if (a.n <= 256) return launch_small<T, 32, 8>(a, groups, counts, shares, loss, stream);
    return launch_small<T, 32, 16>(a, groups, counts, shares, loss, stream);
}

int balance(const nbos_logits *l, int32_t groups, const int32_t *hosts, int32_t k, const float *stats_in,
            const float *grad_loss, float grad_scale, float *out_loss, int32_t *out_counts, float *out_shares,
            float *out_stats, void *out_grad, int64_t gstride, cudaStream_t stream)
{
    int rc = check_logits(l);
    if (rc || (rc = check_k(k))) return rc;
    if (groups < 1 || groups > 65535) return fail(NBOS_ERR_INVALID_ARG, "n_groups must be in 1..65535 (got %d)", groups);
    if (l->rows % groups) return fail(NBOS_ERR_INVALID_ARG, "rows must be a multiple of n_groups");
    if (l->rows > NBOS_POLICY_MAX_ROWS / k) return fail(NBOS_ERR_INVALID_ARG, "rows * k must fit in 31 bits");
    if (l->rows > 0 && !hosts) return fail(NBOS_ERR_INVALID_ARG, "hosts is NULL");
    if (out_grad && (rc = check_grad(l, out_grad, gstride))) return rc;
    if (out_grad == l->data && out_grad && l->rows > 1 && gstride != l->row_stride)
        return fail(NBOS_ERR_INVALID_ARG, "a gradient written over the logits needs their row_stride");
    if (!aligned_to(hosts, 4) || !aligned_to(grad_loss, 4) || !aligned_to(out_loss, 4) || !aligned_to(out_counts, 4) ||
        !aligned_to(out_shares, 4) || !aligned_to(out_stats, 4) || !aligned_to(stats_in, 4))
        return fail(NBOS_ERR_INVALID_ARG, "an int32 / float array is not 4-byte aligned");
    int sms = 0, device = 0;
    if ((rc = check_sm100(&sms, &device))) return rc;
    const size_t n = l->n_hosts, cells = n * groups;
    if (l->rows == 0) {
        if (out_loss) NBOS_CUDA_TRY(cudaMemsetAsync(out_loss, 0, sizeof(float) * groups, stream));
        if (out_counts) NBOS_CUDA_TRY(cudaMemsetAsync(out_counts, 0, sizeof(int32_t) * cells, stream));
        if (out_shares) NBOS_CUDA_TRY(cudaMemsetAsync(out_shares, 0, sizeof(float) * cells, stream));
        return NBOS_OK;
    }
    BalanceArgs a = {};
    a.x = l->data, a.stride = l->row_stride, a.group_rows = l->rows / groups, a.n = l->n_hosts, a.k = k, a.hosts = hosts;
    a.grad_loss = grad_loss, a.grad_scale = grad_scale, a.stats = out_stats, a.stats_in = stats_in;
    a.grad = out_grad, a.gstride = gstride;
    if (l->rows == 1) a.stride = a.gstride = l->n_hosts;
    const size_t elem = dtype_bytes(l->dtype);
    // the path, and with it every rounding, goes by the logits alone: the loss is the same with a gradient or without
    const bool aligned = rows_aligned16(a.x, l->rows, a.stride, elem);
    a.wide = !a.grad || rows_aligned16(a.grad, l->rows, a.gstride, elem);
    if (a.group_rows <= small_rows(l->n_hosts)) {
        const cudaError_t e = l->dtype == NBOS_F32    ? small<float>(a, groups, out_counts, out_shares, out_loss, stream)
                              : l->dtype == NBOS_BF16 ? small<__nv_bfloat16>(a, groups, out_counts, out_shares, out_loss, stream)
                                                      : small<__half>(a, groups, out_counts, out_shares, out_loss, stream);
        if (e != cudaSuccess) return cuda_fail(e, "balance loss launch");
        return NBOS_OK;
    }
    const Plan p = make_plan(a, groups, (int)elem, aligned, sms);
    a.parts = p.parts, a.block_rows = p.block_rows, a.groups = groups;

    // workspace: totals and tickets (cleared), the counts if the caller takes none, the loss and column sums in parts
    auto round256 = [](size_t b) { return (b + 255) & ~(size_t)255; };
    int finish_rows = 1;
    while (finish_rows < 64 && finish_rows < p.parts) finish_rows *= 2;
    while (finish_rows > 1 && (long long)n * finish_rows / kFinishThreads > 8ll * sms) finish_rows /= 2;   // no more blocks than that
    const int finish_cols = kFinishThreads / finish_rows, col_blocks = (int)((n + finish_cols - 1) / finish_cols);
    const bool forward = stats_in == nullptr;
    const size_t b_clear = round256((size_t)groups * (sizeof(int2) + sizeof(unsigned int)));
    const size_t b_counts = out_counts ? 0 : round256(cells * sizeof(int32_t));
    const size_t b_loss = forward ? round256((size_t)groups * col_blocks * sizeof(double)) : 0;
    const size_t b_partial = forward ? cells * p.parts * sizeof(float) : 0;
    cudaMemPool_t pool = nullptr;
    if ((rc = library_pool(device, &pool))) return rc;
    char *ws = nullptr;
    cudaError_t e = cudaMallocFromPoolAsync(reinterpret_cast<void **>(&ws), b_clear + b_counts + b_loss + b_partial, pool, stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(NBOS_ERR_NO_MEMORY, "device allocation failed: %s", cudaGetErrorString(e));
    }
    int2 *totals = reinterpret_cast<int2 *>(ws);
    unsigned int *tickets = reinterpret_cast<unsigned int *>(ws + sizeof(int2) * groups);
    int32_t *counts = out_counts ? out_counts : reinterpret_cast<int32_t *>(ws + b_clear);
    double *loss_parts = reinterpret_cast<double *>(ws + b_clear + b_counts);
    a.partial = reinterpret_cast<float *>(ws + b_clear + b_counts + b_loss);
    a.counts = counts, a.totals = totals;

    if (n <= kHistHosts && a.group_rows * k <= kClusterIds) {
        int cs = 1;
        while (cs < kMaxCluster && a.group_rows > 512ll * cs) cs *= 2;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(cs, groups);
        cfg.blockDim = dim3(512);
        cfg.dynamicSmemBytes = n * sizeof(int);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = cs;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, count_cluster_kernel, hosts, (int)a.group_rows, (int)k, a.n, cs, counts, totals, tickets);
    } else {
        e = cudaMemsetAsync(ws, 0, b_clear + b_counts, stream);
        if (e == cudaSuccess && out_counts) e = cudaMemsetAsync(out_counts, 0, cells * sizeof(int32_t), stream);
        if (e == cudaSuccess) {
            // counters of a block's own keep the hot hosts' additions apart; they pay where a block counts more than it has to clear
            // and hand on, so large groups get no more blocks than that allows beyond one an SM
            long long bx = (a.group_rows + 255) / 256;
            const long long cap = (8ll * sms + groups - 1) / groups, one = (sms + groups - 1) / groups;
            const long long worth = a.group_rows * k / (4ll * (long long)n) > one ? a.group_rows * k / (4ll * (long long)n) : one;
            if (bx > cap) bx = cap;
            if (bx > worth) bx = worth;
            const bool in_shared = n <= kHistHosts && a.group_rows * k / bx >= (long long)n / 4;
            count_kernel<<<dim3((unsigned int)bx, groups), 256, in_shared ? n * sizeof(int) : 0, stream>>>(hosts, a.group_rows, k, a.n, in_shared,
                                                                                                           counts, totals);
            e = cudaGetLastError();
        }
    }
    if (e == cudaSuccess)
        e = l->dtype == NBOS_F32    ? dispatch<float>(a, groups, p, stream)
            : l->dtype == NBOS_BF16 ? dispatch<__nv_bfloat16>(a, groups, p, stream)
                                    : dispatch<__half>(a, groups, p, stream);
    if (e == cudaSuccess && forward) {
        finish_kernel<<<dim3(col_blocks, groups), dim3(finish_cols, finish_rows), 0, stream>>>(a, out_shares, out_loss, loss_parts, tickets);
        e = cudaGetLastError();
    }
    cudaFreeAsync(ws, stream);
    if (e != cudaSuccess) return cuda_fail(e, "balance loss launch");
    return NBOS_OK;
}

}  // namespace
}  // namespace nbos

using namespace nbos;

extern "C" int nbos_policy_balance(const nbos_logits *logits, int32_t n_groups, const int32_t *hosts, int32_t k,
                                   const float *grad_loss, float grad_scale, float *out_loss, int32_t *out_counts,
                                   float *out_shares, float *out_stats, void *out_grad, int64_t grad_stride,
                                   void *cuda_stream)
{
    if (!out_loss || !out_counts) return fail(NBOS_ERR_INVALID_ARG, "out_loss / out_counts is NULL");
    return balance(logits, n_groups, hosts, k, nullptr, grad_loss, grad_scale, out_loss, out_counts, out_shares, out_stats,
                   out_grad, grad_stride, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int nbos_policy_balance_backward(const nbos_logits *logits, int32_t n_groups, const int32_t *hosts, int32_t k,
                                            const float *stats, const float *grad_loss, float grad_scale, void *out_grad,
                                            int64_t grad_stride, void *cuda_stream)
{
    if (logits && logits->rows > 0 && (!stats || !out_grad)) return fail(NBOS_ERR_INVALID_ARG, "stats / out_grad is NULL");
    if (logits && logits->rows == 0) stats = nullptr;
    return balance(logits, n_groups, hosts, k, stats, grad_loss, grad_scale, nullptr, nullptr, nullptr, nullptr, out_grad,
                   grad_stride, static_cast<cudaStream_t>(cuda_stream));
}
