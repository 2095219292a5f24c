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
#include <math.h>

#include "nbos_policy.cuh"

namespace nbos {
namespace {

using namespace policy;

constexpr int kWarpRow = 1024;      // longest row of the warp form: 32 elements a lane
constexpr int kElems = 16;          // row elements a thread holds in the block form (as many column sums beside them)
constexpr int kMaxCluster = 8;
constexpr int kWarps = 8;           // of a block of the warp form
constexpr int kHistHosts = 8192;    // counters kept in shared memory while counting

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
    int parts;
};

// counts[g][h] += ..., totals[g] += (valid ids, rows that have one); grid (blocks, groups)
__global__ void __launch_bounds__(256) count_kernel(const int32_t *hosts, long long group_rows, int k, int n,
                                                    int32_t *counts, int2 *totals)
{
    extern __shared__ int s_hist[];
    __shared__ int s_tot[2];
    const bool in_shared = n <= kHistHosts;
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

// does any of the row's ids name a host? over `lanes` lanes
__device__ __forceinline__ bool row_live(const BalanceArgs &a, long long row, bool active, int sub, int lanes)
{
    float some = 0.0f;
    for (int j = sub; active && j < a.k; j += lanes) {
        const int h = a.hosts[row * a.k + j];
        if (h >= 0 && h < a.n) some = 1.0f;
    }
    return lanes_max(some, lanes) > 0.0f;
}

// ---- warp form: `lanes` lanes per row; grid (parts, groups) ------------------------------------------------
template <typename T, int VEC, int CH, bool GRAD, bool SAVED>
__global__ void __launch_bounds__(kWarps * 32) balance_warp_kernel(BalanceArgs a, int lanes)
{
    extern __shared__ float s_f[];   // f of the group's hosts, padded to lanes * CH * VEC; then the column sums
    const int lane = threadIdx.x & 31, sub = lane & (lanes - 1), warp = threadIdx.x >> 5;
    const int group = blockIdx.y, width = lanes * CH * VEC;
    const GroupScale gs = group_scale(a, group);
    for (int i = threadIdx.x; i < width; i += blockDim.x) s_f[i] = i < a.n ? (float)a.counts[(size_t)group * a.n + i] * gs.inv_total : 0.0f;
    __syncthreads();
    float acc[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[c][i] = 0.0f;
    const int rows_at_once = 32 / lanes;
    const long long first = (long long)group * a.group_rows;
    for (long long r0 = ((long long)blockIdx.x * kWarps + warp) * rows_at_once; r0 < a.group_rows;
         r0 += (long long)gridDim.x * kWarps * rows_at_once) {
        const bool active = r0 + lane / lanes < a.group_rows;
        const long long row = first + r0 + (active ? lane / lanes : 0);
        const T *x = static_cast<const T *>(a.x) + row * a.stride;
        float v[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) load_cols<T, VEC>(x, (c * lanes + sub) * VEC, active ? a.n : 0, neg_inf(), v[c]);
        const bool live = row_live(a, row, active, sub, lanes);
        float m = neg_inf(), s = 0.0f, dot = 0.0f;
        if (SAVED) {
            m = live ? a.stats_in[2 * row] : 0.0f;
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) m = fmaxf(m, v[c][i]);
            m = lanes_max(m, lanes);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] = exp_from(v[c][i], m, kLog2e);
                s += v[c][i];
                if (GRAD) dot += v[c][i] * s_f[(c * lanes + sub) * VEC + i];
            }
        s = SAVED ? (live ? a.stats_in[2 * row + 1] : 1.0f) : lanes_sum(s, lanes);
        if (GRAD) dot = lanes_sum(dot, lanes);
        // a row of -inf has sum 0 and no probabilities
        const float inv = live && s != 0.0f ? 1.0f / s : 0.0f;
        if (!SAVED) {
            if (live && a.stats && sub == 0) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[c][i] += live ? v[c][i] * inv : 0.0f;
        }
        if (GRAD) {
            T *grad = static_cast<T *>(a.grad) + row * a.gstride;
            dot *= inv;
            const float fac = gs.grad * inv;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    v[c][i] = live ? v[c][i] * fac * (s_f[(c * lanes + sub) * VEC + i] - dot) : 0.0f;
                store_cols<T, VEC>(grad, (c * lanes + sub) * VEC, active ? a.n : 0, v[c]);
            }
        }
    }
    if constexpr (!SAVED) {
        // the block's column sums: rows of one warp, then warp after warp
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                for (int off = 16; off >= lanes; off >>= 1) acc[c][i] += __shfl_xor_sync(kFull, acc[c][i], off);
        for (int w = 0; w < kWarps; ++w) {
            __syncthreads();
            if (warp == w && lane < lanes) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        float *to = &s_f[(c * lanes + sub) * VEC + i];
                        *to = w ? *to + acc[c][i] : acc[c][i];
                    }
            }
        }
        __syncthreads();
        float *out = a.partial + ((size_t)group * a.parts + blockIdx.x) * a.n;
        for (int i = threadIdx.x; i < a.n; i += blockDim.x) out[i] = s_f[i];
    }
}

// ---- block form: one block or cluster of cs blocks per row at a time; grid (parts * cs, groups) -------------
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
        const bool live = row_live(a, row, true, lane, 32);
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
                if (GRAD) store_cols<T, VEC>(grad, first_col + c * chunk + threadIdx.x * VEC, end_col, v[c]);
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
                if (GRAD) store_cols<T, VEC>(grad, col, end_col, w);
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

// shares = column sums over the parts / live; loss = n sum f share. blockDim (32 columns, L parts at a time);
// grid (column blocks, groups). The group's last block adds the column blocks' shares of the loss, in order.
__global__ void __launch_bounds__(1024) finish_kernel(BalanceArgs a, float *shares, float *loss, double *loss_parts,
                                                      unsigned int *tickets)
{
    __shared__ double s_sum[32][33];
    __shared__ unsigned int s_last;
    const int group = blockIdx.y, col = blockIdx.x * 32 + threadIdx.x;
    double sum = 0.0;
    if (col < a.n)
        for (int p = threadIdx.y; p < a.parts; p += blockDim.y) sum += (double)a.partial[((size_t)group * a.parts + p) * a.n + col];
    s_sum[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y != 0) return;
    for (int y = 1; y < blockDim.y; ++y) sum += s_sum[y][threadIdx.x];
    const int2 t = a.totals[group];
    const double share = t.y > 0 ? sum / (double)t.y : 0.0;
    double part = 0.0;
    if (col < a.n) {
        if (shares) shares[(size_t)group * a.n + col] = (float)share;
        if (t.x > 0) part = share * ((double)a.counts[(size_t)group * a.n + col] / (double)t.x);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) part += __shfl_xor_sync(kFull, part, off);
    double *mine = loss_parts + (size_t)group * gridDim.x;
    if (threadIdx.x == 0) {
        mine[blockIdx.x] = part;
        __threadfence();
        s_last = atomicAdd(&tickets[group], 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncwarp();
    if (!s_last) return;
    double total = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 32) total += __ldcg(&mine[i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(kFull, total, off);
    if (threadIdx.x == 0) loss[group] = (float)(total * (double)a.n);
}

struct Plan {
    bool warp_form, keep;
    int lanes, need;        // warp form: lanes per row, chunks per lane
    int cs, threads, span;  // block form
    int parts;
};

// VEC elements per load; rows of one group
Plan make_plan(const BalanceArgs &a, int groups, int vec, int sms)
{
    Plan p = {};
    p.warp_form = a.n <= kWarpRow;
    long long wanted;
    if (p.warp_form) {
        p.lanes = 1;
        while (p.lanes < 32 && p.lanes * vec < a.n) p.lanes *= 2;
        p.need = (a.n + p.lanes * vec - 1) / (p.lanes * vec);
        const long long at_once = kWarps * (32 / p.lanes);
        wanted = (a.group_rows + at_once - 1) / at_once;
        const long long fill = (3ll * sms + groups - 1) / groups;
        p.parts = (int)(wanted < fill ? wanted : fill);
    } else {
        auto threads_for = [&](int c) { return ((a.n + c * kElems - 1) / (c * kElems) + 31) / 32 * 32; };
        p.keep = a.n <= kMaxCluster * 1024 * kElems;
        p.cs = 1;
        while (p.cs < kMaxCluster && (threads_for(p.cs) > 1024 || (a.group_rows * groups * p.cs < 2 * sms && threads_for(p.cs) > 128)))
            p.cs *= 2;
        p.threads = p.keep ? threads_for(p.cs) : 1024;
        p.span = ((a.n + p.cs - 1) / p.cs + vec - 1) / vec * vec;
        const int resident = p.threads > 512 ? 1 : (1024 / p.threads);
        const long long fill = ((long long)sms * resident / p.cs + groups - 1) / groups;
        p.parts = (int)(a.group_rows < fill ? a.group_rows : (fill > 1 ? fill : 1));
    }
    if (p.parts < 1) p.parts = 1;
    return p;
}

template <typename T, int VEC, int CH, bool GRAD, bool SAVED>
cudaError_t launch_warp(const BalanceArgs &a, int groups, const Plan &p, cudaStream_t stream)
{
    const size_t smem = (size_t)p.lanes * CH * VEC * sizeof(float);
    balance_warp_kernel<T, VEC, CH, GRAD, SAVED><<<dim3(p.parts, groups), kWarps * 32, smem, stream>>>(a, p.lanes);
    return cudaGetLastError();
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
cudaError_t launch(const BalanceArgs &a, int groups, const Plan &p, cudaStream_t stream)
{
    if (!p.warp_form)
        return p.keep ? launch_block<T, VEC, true, GRAD, SAVED>(a, groups, p, stream)
                      : launch_block<T, VEC, false, GRAD, SAVED>(a, groups, p, stream);
    if (p.need <= 1) return launch_warp<T, VEC, 1, GRAD, SAVED>(a, groups, p, stream);
    if (p.need <= 2) return launch_warp<T, VEC, 2, GRAD, SAVED>(a, groups, p, stream);
    if (VEC >= 4 || p.need <= 4) return launch_warp<T, VEC, (VEC == 4 ? 8 : 4), GRAD, SAVED>(a, groups, p, stream);
    if constexpr (VEC == 1) {
        if (p.need <= 8) return launch_warp<T, VEC, 8, GRAD, SAVED>(a, groups, p, stream);
        if (p.need <= 16) return launch_warp<T, VEC, 16, GRAD, SAVED>(a, groups, p, stream);
        return launch_warp<T, VEC, 32, GRAD, SAVED>(a, groups, p, stream);
    }
    return cudaErrorUnknown;   // not reached
}

template <typename T>
cudaError_t dispatch(const BalanceArgs &a, int groups, const Plan &p, bool vec, cudaStream_t stream)
{
    constexpr int V = kPer16<T>;
    if (a.stats_in) return vec ? launch<T, V, true, true>(a, groups, p, stream) : launch<T, 1, true, true>(a, groups, p, stream);
    if (a.grad) return vec ? launch<T, V, true, false>(a, groups, p, stream) : launch<T, 1, true, false>(a, groups, p, stream);
    return vec ? launch<T, V, false, false>(a, groups, p, stream) : launch<T, 1, false, false>(a, groups, p, stream);
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
    const bool vec = rows_aligned16(a.x, l->rows, a.stride, elem) && (!a.grad || rows_aligned16(a.grad, l->rows, a.gstride, elem));
    const Plan p = make_plan(a, groups, vec ? (int)(16 / elem) : 1, sms);
    a.parts = p.parts;

    // workspace: totals and tickets (cleared), the counts if the caller takes none, the loss and column sums in parts
    auto round256 = [](size_t b) { return (b + 255) & ~(size_t)255; };
    const int col_blocks = (int)((n + 31) / 32);
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

    e = cudaMemsetAsync(ws, 0, b_clear + b_counts, stream);
    if (e == cudaSuccess && out_counts) e = cudaMemsetAsync(out_counts, 0, cells * sizeof(int32_t), stream);
    if (e == cudaSuccess) {
        long long bx = (a.group_rows + 1023) / 1024;
        const long long cap = (4ll * sms + groups - 1) / groups;
        if (bx > cap) bx = cap;
        const size_t hist = n <= kHistHosts ? n * sizeof(int) : 0;
        count_kernel<<<dim3((unsigned int)bx, groups), 256, hist, stream>>>(hosts, a.group_rows, k, a.n, counts, totals);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess)
        e = l->dtype == NBOS_F32    ? dispatch<float>(a, groups, p, vec, stream)
            : l->dtype == NBOS_BF16 ? dispatch<__nv_bfloat16>(a, groups, p, vec, stream)
                                    : dispatch<__half>(a, groups, p, vec, stream);
    if (e == cudaSuccess && forward) {
        int at_once = 1;
        while (at_once < 32 && at_once < p.parts) at_once *= 2;
        finish_kernel<<<dim3(col_blocks, groups), dim3(32, at_once), 0, stream>>>(a, out_shares, out_loss, loss_parts, tickets);
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
