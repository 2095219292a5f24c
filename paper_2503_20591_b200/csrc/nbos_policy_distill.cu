// Distillation of a placement policy from a teacher's k best hosts per row (nbos_policy_distill).
//
// Per row with logits x, m = max x, S = sum_j 2^((x_j - m) c), c = log2(e) / T, p_j = 2^((x_j - m) c) / S and the
// teacher's q over its counting entries:
//   loss = T^2 sum_k q_k (ln q_k - ln p_k),  d loss / d x_j = T (p_j - q_j).
// What bounds it: the logits' bytes, read once, and as many written for the gradient. So a row stays in registers
// between its reduction and its gradient (32 to 64 elements a thread): 4 to 32 lanes of a warp share a short row (up to
// 1,024 hosts), a block a longer one (up to 16,384). Both stay on their SM and walk over the rows, the next ones on their
// way to shared memory by asynchronous copies. Longer rows, or few of them, take a cluster of up to 8 blocks each; only
// rows of more than 262,144 hosts are read twice. Each exponential is computed once; threads keep it relative to their
// warp's maximum and scale it by 2^((m_warp - m) c) / S when the row's statistics are known.
// Measured (B200, 6,464 GB/s copied): 262,144 x 1,024 bf16 loss and gradient back to back 202 us = 5,330 GB/s (218 us a call
// at a time), f32 375 us = 5,730 GB/s;
// 65,536 x 4,096 bf16 238 us = 4,510 GB/s. 16-bit logits are bound by instruction issue beside the bytes.
#include <math.h>

#include "nbos_policy.cuh"

namespace nbos {
namespace {

using namespace policy;

constexpr int kElems = 32;             // row elements a thread holds in the block form
constexpr int kBlockStages = 3;        // rows of the block form on their way or in use
constexpr int kMaxCluster = 8;
constexpr int kWarpRow = 32 * kElems;  // longest row of the warp form

struct DistillArgs {
    const void *x;
    long long rows, stride;
    int n;
    const int32_t *hosts;
    const float *teacher;
    long long tstride;
    int k;
    float T, c, inv_t;
    const float *grad_loss;
    float grad_scale;
    float *loss;
    float *stats;
    const float *stats_in;
    void *grad;
    long long gstride;
    bool wide;   // the gradient's rows lie on 16-byte boundaries where the logits' do: it is written 16 bytes at a time
};

struct Entry {
    int host;   // -1: does not count
    float t, x;
};

template <typename T>
__device__ __forceinline__ Entry load_entry(const DistillArgs &a, long long row, const T *x, int k)
{
    Entry e;
    e.host = a.hosts[row * a.k + k];
    e.t = a.teacher ? a.teacher[row * a.tstride + k] : 0.0f;
    e.x = neg_inf();
    if (e.host >= 0 && e.host < a.n) e.x = to_float(x[e.host]);
    // comparisons with NaN are false: a NaN teacher logit does not count; a NaN student logit does (its row is NaN)
    if (!(e.t > neg_inf()) || e.x == neg_inf()) e.host = -1;
    return e;
}

// The teacher's softmax over `lanes` lanes: largest teacher logit of the row (-inf: no entry counts) and the sum.
template <typename T>
__device__ __forceinline__ void teacher_stats(const DistillArgs &a, long long row, const T *x, bool active, int sub,
                                              int lanes, const Entry &first, float &tm, float &z)
{
    tm = neg_inf();
    for (int k = sub; active && k < a.k; k += lanes) {
        const Entry e = k == sub ? first : load_entry(a, row, x, k);
        if (e.host >= 0) tm = fmaxf(tm, e.t);
    }
    tm = lanes_max(tm, lanes);
    z = 0.0f;
    for (int k = sub; active && k < a.k; k += lanes) {
        const Entry e = k == sub ? first : load_entry(a, row, x, k);
        if (e.host >= 0) z += exp_from(e.t, tm, a.c);
    }
    z = lanes_sum(z, lanes);
}

template <typename T>
__device__ __forceinline__ float row_loss(const DistillArgs &a, long long row, const T *x, bool active, int sub, int lanes,
                                          const Entry &first, float tm, float z, float m, float s)
{
    const float shift = logf(s) - logf(z);
    float l = 0.0f;
    for (int k = sub; active && k < a.k; k += lanes) {
        const Entry e = k == sub ? first : load_entry(a, row, x, k);
        if (e.host < 0) continue;
        const float q = exp_from(e.t, tm, a.c) * reciprocal(z);
        // q underflows to 0 before ln q leaves the range of 32 bits; 0 * -inf is kept out
        const float v = q * (((e.t - tm) - (e.x - m)) * a.inv_t + shift);
        l += q == 0.0f ? 0.0f : v;
    }
    return lanes_sum(l, lanes) * a.T * a.T;
}

// The gradient at the listed hosts, written over what the row's owner wrote there: p - (all of q that goes there).
template <typename T>
__device__ __forceinline__ void fix_entries(const DistillArgs &a, long long row, const T *x, const Entry &e, T *grad,
                                            float tm, float z, float m, float s, float gmul)
{
    float q = 0.0f;
    for (int k = 0; k < a.k; ++k) {
        if (a.hosts[row * a.k + k] != e.host) continue;
        const float t = a.teacher ? a.teacher[row * a.tstride + k] : 0.0f;
        if (t > neg_inf()) q += exp_from(t, tm, a.c) * reciprocal(z);
    }
    grad[e.host] = from_float<T>(gmul * (exp_from(e.x, m, a.c) * reciprocal(s) - q));
}

__device__ __forceinline__ float grad_multiplier(const DistillArgs &a, long long row)
{
    return a.T * a.grad_scale * (a.grad_loss ? a.grad_loss[row] : 1.0f);
}

// ---- rows that a warp or a block holds, staged -------------------------------------------------------------
// What a team needs of one row, in shared memory: the row, its entries, (grad_loss, m, S).
template <typename T>
struct Staged {
    const T *x;
    const int *hosts;
    const float *teacher, *given;
    int n, k;
    bool has_teacher;
    __device__ __forceinline__ Entry entry(int i) const
    {
        Entry e;
        e.host = hosts[i];
        e.t = has_teacher ? teacher[i] : 0.0f;
        e.x = neg_inf();
        if (e.host >= 0 && e.host < n) e.x = to_float(x[e.host]);
        // comparisons with NaN are false: a NaN teacher logit does not count; a NaN student logit does
        if (!(e.t > neg_inf()) || e.x == neg_inf()) e.host = -1;
        return e;
    }
};
struct Layout {   // bytes of a stage: rows, then entries, then what is given per row
    int row_bytes, rows, k;
    bool aligned;   // every row starts on a 16-byte boundary
    int whole;      // n if, besides, the gradient is written 16 bytes at a time: columns below it need no look; else 0
    __host__ __device__ int hosts_at() const { return row_bytes * rows; }
    __host__ __device__ int teacher_at() const { return hosts_at() + rows * k * 4; }
    __host__ __device__ int given_at() const { return teacher_at() + rows * k * 4; }
    __host__ __device__ int bytes() const { return (given_at() + rows * 12 + 15) & ~15; }
};

template <typename T, bool GRAD, bool SAVED>
__device__ __forceinline__ void stage_rest(const DistillArgs &a, const Layout &lay, char *at, int slot, long long row, int sub, int team)
{
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(at));
    for (int i = sub; i < a.k; i += team) {
        copy_async4(to + lay.hosts_at() + (slot * a.k + i) * 4, a.hosts + row * a.k + i);
        if (a.teacher) copy_async4(to + lay.teacher_at() + (slot * a.k + i) * 4, a.teacher + row * a.tstride + i);
    }
    if (sub == 0) {
        if (GRAD && a.grad_loss) copy_async4(to + lay.given_at() + slot * 12, a.grad_loss + row);
        if (SAVED) {
            copy_async4(to + lay.given_at() + slot * 12 + 4, a.stats_in + 2 * row);
            copy_async4(to + lay.given_at() + slot * 12 + 8, a.stats_in + 2 * row + 1);
        }
    }
}
template <typename T>
__device__ __forceinline__ Staged<T> staged_row(const DistillArgs &a, const Layout &lay, const char *at, int slot, long long row)
{
    Staged<T> s;
    s.x = reinterpret_cast<const T *>(at + slot * lay.row_bytes + row_shift(static_cast<const T *>(a.x) + row * a.stride));
    s.hosts = reinterpret_cast<const int *>(at + lay.hosts_at()) + slot * a.k;
    s.teacher = reinterpret_cast<const float *>(at + lay.teacher_at()) + slot * a.k;
    s.given = reinterpret_cast<const float *>(at + lay.given_at()) + slot * 3;
    s.n = a.n, s.k = a.k, s.has_teacher = a.teacher != nullptr;
    return s;
}

// largest teacher logit of the row (-inf: no entry counts) and the sum of its softmax, over `lanes` lanes
template <typename T>
__device__ __forceinline__ void teacher_sums(const DistillArgs &a, const Staged<T> &r, bool active, int sub, int lanes, float &tm, float &z)
{
    tm = neg_inf();
    for (int i = sub; active && i < a.k; i += lanes) {
        const Entry e = r.entry(i);
        if (e.host >= 0) tm = fmaxf(tm, e.t);
    }
    tm = lanes_max(tm, lanes);
    z = 0.0f;
    for (int i = sub; active && i < a.k; i += lanes) {
        const Entry e = r.entry(i);
        if (e.host >= 0) z += exp_from(e.t, tm, a.c);
    }
    z = lanes_sum(z, lanes);
}
template <typename T>
__device__ __forceinline__ float entries_loss(const DistillArgs &a, const Staged<T> &r, bool active, int sub, int lanes, float tm, float z, float m, float s)
{
    const float shift = logf(s) - logf(z);
    float l = 0.0f;
    for (int i = sub; active && i < a.k; i += lanes) {
        const Entry e = r.entry(i);
        if (e.host < 0) continue;
        const float q = exp_from(e.t, tm, a.c) * reciprocal(z);
        // q underflows to 0 before ln q leaves the range of 32 bits; 0 * -inf is kept out
        const float v = q * (((e.t - tm) - (e.x - m)) * a.inv_t + shift);
        l += q == 0.0f ? 0.0f : v;
    }
    return lanes_sum(l, lanes) * a.T * a.T;
}
// the gradient at an entry's host: p - (all of q that goes there)
template <typename T>
__device__ __forceinline__ float entry_grad(const DistillArgs &a, const Staged<T> &r, const Entry &e, float tm, float z, float m, float s, float gmul)
{
    float q = 0.0f;
    for (int i = 0; i < a.k; ++i) {
        const float t = r.has_teacher ? r.teacher[i] : 0.0f;
        if (r.hosts[i] == e.host && t > neg_inf()) q += exp_from(t, tm, a.c) * reciprocal(z);
    }
    return gmul * (exp_from(e.x, m, a.c) * reciprocal(s) - q);
}

// At most one entry a lane (e, host -1 where there is none), in the first entry_lanes of `lanes` lanes: the row's loss (if
// LOSS) and, if GRAD, the gradient at the lane's entry.
template <bool LOSS, bool GRAD>
__device__ __forceinline__ void entry_math(const DistillArgs &a, const Entry &e, int lanes, int entry_lanes, float m0, float s, float inv_s,
                                           float gmul, float &loss, float &grad)
{
    const float tm = lanes_max(e.host >= 0 ? e.t : neg_inf(), entry_lanes);
    float q = e.host >= 0 ? exp2_fast((e.t - tm) * a.c) : 0.0f;
    const float inv_z = reciprocal(lanes_sum(q, entry_lanes));
    q *= inv_z;
    if (LOSS) {
        // q underflows to 0 before ln q leaves the range of 32 bits; 0 * -inf is kept out
        const float l = q * (((e.t - tm) - (e.x - m0)) * a.inv_t + logf(s * inv_z));
        loss = lanes_sum(e.host < 0 || q == 0.0f ? 0.0f : l, entry_lanes) * a.T * a.T;
    }
    if (GRAD) {
        float all = 0.0f;   // a host may be listed more than once
        for (int i = 0; i < a.k; ++i) {
            const float other = __shfl_sync(kFull, q, i, lanes);
            if (__shfl_sync(kFull, e.host, i, lanes) == e.host) all += other;
        }
        grad = gmul * (exp2_fast((e.x - m0) * a.c) * inv_s - all);
    }
}

// ---- warp form: LANES lanes per row, CH * VEC elements each; the grid stays and walks over the rows -------
constexpr int kWarps = 8;
// Elements a lane holds at most. 64 (at two thirds of the warps an SM) is worth it where instructions bound: 262,144 x 1,024 bf16
// 202 us against 218; not for 32-bit logits, bound by their bytes: 441 us against 380.
template <typename T> constexpr int kMostElems = sizeof(T) == 2 ? 64 : 40;

template <typename T, int LANES, int CH, bool GRAD, bool SAVED>
__global__ void __launch_bounds__(kWarps * 32, CH * kPer16<T> > 32 ? 2 : 3) distill_warp_kernel(DistillArgs a, int entry_lanes, Layout lay)
{
    constexpr int VEC = kPer16<T>;
    extern __shared__ __align__(16) char s_mem[];
    constexpr int lanes = LANES;
    const int lane = threadIdx.x & 31, sub = lane & (lanes - 1), slot = lane / lanes, at_once = 32 / lanes;
    const int stage_bytes = lay.bytes();
    char *mine = s_mem + (threadIdx.x >> 5) * kStages * stage_bytes;
    const long long step = (long long)gridDim.x * kWarps * at_once;
    const long long row0 = ((long long)blockIdx.x * kWarps + (threadIdx.x >> 5)) * at_once;
    auto queue = [&](long long base, int st) {
        if (base + slot < a.rows) {
            stage_row(mine + st * stage_bytes + slot * lay.row_bytes, static_cast<const T *>(a.x) + (base + slot) * a.stride, a.n,
                      (base + slot) * a.stride * (long long)sizeof(T), sub, lanes);
            stage_rest<T, GRAD, SAVED>(a, lay, mine + st * stage_bytes, slot, base + slot, sub, lanes);
        }
        copies_commit();
    };
#pragma unroll
    for (int st = 0; st < kStages - 1; ++st) queue(row0 + st * step, st);
    int st = 0;
    for (long long base = row0; base < a.rows; base += step) {
        queue(base + (kStages - 1) * step, st == 0 ? kStages - 1 : st - 1);
        copies_wait();
        __syncwarp();
        const bool active = base + slot < a.rows;
        const long long row = active ? base + slot : base;
        const Staged<T> r = staged_row<T>(a, lay, mine + st * stage_bytes, active ? slot : 0, row);
        const int first = sub * VEC - row_shift(r.x) / (int)sizeof(T);
        float v[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if ((c + 1) * lanes * VEC <= lay.whole)
                unpack16(*reinterpret_cast<const uint4 *>(r.x + first + c * lanes * VEC), v[c], T());
            else
                staged_cols<T, VEC>(r.x, first + c * lanes * VEC, a.n, v[c]);
        }
        const float m = SAVED ? r.given[1] : lanes_max(max_all<VEC, CH>(v), lanes);
        const float m0 = m == neg_inf() ? 0.0f : m;
        const float mine_sum = exp_all<VEC, CH>(v, m0, a.c);
        const float s = SAVED ? r.given[2] : lanes_sum(mine_sum, lanes);
        const float inv_s = reciprocal(s);
        const float gmul = GRAD ? a.T * a.grad_scale * (a.grad_loss ? r.given[0] : 1.0f) : 0.0f;
        float tm = neg_inf(), z = 0.0f, entry_g = 0.0f, l = 0.0f;
        Entry e{-1, 0.0f, 0.0f};   // k <= lanes: the lane's entry
        bool any;
        if (a.k <= lanes) {
            if (active && sub < a.k) e = r.entry(sub);
            const unsigned int group = lanes == 32 ? kFull : ((1u << lanes) - 1) << (slot * lanes);
            any = (__ballot_sync(kFull, e.host >= 0) & group) != 0;
            entry_math<!SAVED, GRAD>(a, e, lanes, entry_lanes, m0, s, inv_s, gmul, l, entry_g);
        } else {
            teacher_sums(a, r, active, sub, lanes, tm, z);
            any = tm > neg_inf();
            if (!SAVED) l = entries_loss(a, r, active && any, sub, lanes, tm, z, m, s);
        }
        if (!SAVED && active && sub == 0) {
            if (a.loss) a.loss[row] = any ? l : 0.0f;
            if (a.stats) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
        }
        if (GRAD) {
            T *grad = static_cast<T *>(a.grad) + row * a.gstride;
            const float fac = gmul * inv_s;
            if (__any_sync(kFull, !any)) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[c][i] = any ? v[c][i] : 0.0f;
            }
            const float fac0 = any ? fac : 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                scale_all<VEC>(v[c], fac0);
                if ((c + 1) * lanes * VEC <= lay.whole) {
                    if (active) __stcs(reinterpret_cast<uint4 *>(grad + first + c * lanes * VEC), pack16(v[c], T()));
                } else {
                    store_cols<T, VEC>(grad, first + c * lanes * VEC, active ? a.n : 0, v[c], a.wide);
                }
            }
            __syncwarp();   // the listed hosts' gradients go over what their columns' lanes wrote
            if (a.k <= lanes) {
                if (e.host >= 0) grad[e.host] = from_float<T>(entry_g);
            } else {
                for (int i = sub; active && i < a.k; i += lanes) {
                    const Entry o = r.entry(i);
                    if (o.host >= 0) grad[o.host] = from_float<T>(entry_grad(a, r, o, tm, z, m, s, gmul));
                }
            }
        }
        __syncwarp();   // the stage may be filled again
        st = st == kStages - 1 ? 0 : st + 1;
    }
}

// ---- block form: one row at a time per block, kElems elements a thread -------------------------------------
template <typename T, bool GRAD, bool SAVED>
__global__ void __maxnreg__(80) distill_staged_kernel(DistillArgs a, int entry_lanes, Layout lay)
{
    constexpr int VEC = kPer16<T>, CH = kElems / VEC;
    extern __shared__ __align__(16) char s_mem[];
    __shared__ float2 s_stats[2][16];
    __shared__ float s_fix[NBOS_POLICY_MAX_K];
    __shared__ int s_fix_host[NBOS_POLICY_MAX_K];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    // a warp has one stretch of columns: offsets are known when compiled
    constexpr int chunk = 32 * VEC;
    const int pieces = warp * 32 * CH, base = pieces * VEC, stage_bytes = lay.bytes();
    auto queue = [&](long long row, int st) {
        if (row < a.rows) {
            stage_row(s_mem + st * stage_bytes, static_cast<const T *>(a.x) + row * a.stride, a.n, row * a.stride * (long long)sizeof(T), lane, 32,
                      pieces, pieces + 32 * CH);
            stage_rest<T, GRAD, SAVED>(a, lay, s_mem + st * stage_bytes, 0, row, threadIdx.x, blockDim.x);
        }
        copies_commit();
    };
    // The listed hosts' gradients go over what their columns' threads wrote; the first warp writes them once all threads
    // have come to the next row's barrier. That barrier also frees the stage of the row before: three stages.
    T *fix_grad = nullptr;
    auto fix = [&]() {
        if (GRAD && warp == 0 && fix_grad) {
            for (int i = lane; i < a.k; i += 32)
                if (s_fix_host[i] >= 0) fix_grad[s_fix_host[i]] = from_float<T>(s_fix[i]);
            fix_grad = nullptr;
        }
    };
#pragma unroll
    for (int st = 0; st < kBlockStages - 1; ++st) queue(blockIdx.x + (long long)st * gridDim.x, st);
    int st = 0, turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const long long ahead = row + (kBlockStages - 1) * (long long)gridDim.x;
        const int ahead_st = st == 0 ? kBlockStages - 1 : st - 1;
        copies_wait<kBlockStages - 2>();
        const Staged<T> r = staged_row<T>(a, lay, s_mem + st * stage_bytes, 0, row);
        // its 16 bytes a thread has copied itself; the first elements of an unaligned table came through other threads
        if (!lay.aligned || SAVED) __syncthreads();
        if (SAVED) {
            fix();
            queue(ahead, ahead_st);
        }
        const int first = base + lane * VEC - row_shift(r.x) / (int)sizeof(T);
        float v[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if ((c + 1) * chunk <= lay.whole - base)
                unpack16(*reinterpret_cast<const uint4 *>(r.x + first + c * chunk), v[c], T());
            else
                staged_cols<T, VEC>(r.x, first + c * chunk, a.n, v[c]);
        }
        float m = SAVED ? r.given[1] : lanes_max(max_all<VEC, CH>(v), 32);
        const float m_warp = m;
        float s = exp_all<VEC, CH>(v, m == neg_inf() ? 0.0f : m, a.c);
        if (SAVED) {
            s = r.given[2];
        } else {
            s = lanes_sum(s, 32);
            if (lane == 0) s_stats[turn][warp] = make_float2(m, s);
            __syncthreads();
            fix();
            queue(ahead, ahead_st);
            const float2 w = lane < warps ? s_stats[turn][lane] : make_float2(neg_inf(), 0.0f);
            m = lanes_max(w.x, 16);
            m = __shfl_sync(kFull, m, 0);
            s = lanes_sum(w.y * exp_from(w.x, m, a.c), 16);
            s = __shfl_sync(kFull, s, 0);
        }
        const float inv_s = reciprocal(s);
        const float gmul = GRAD ? a.T * a.grad_scale * (a.grad_loss ? r.given[0] : 1.0f) : 0.0f;
        // every warp finds out whether an entry counts; the first one does what is to be done with them
        bool any = false;
        for (int i = lane; i < a.k; i += 32) any = any || r.entry(i).host >= 0;
        any = __any_sync(kFull, any);
        if (warp == 0) {
            float l = 0.0f;
            if (a.k <= 32) {
                Entry e{-1, 0.0f, 0.0f};
                if (lane < a.k) e = r.entry(lane);
                float g = 0.0f;
                entry_math<!SAVED, GRAD>(a, e, 32, entry_lanes, m == neg_inf() ? 0.0f : m, s, inv_s, gmul, l, g);
                if (GRAD && lane < a.k) s_fix_host[lane] = e.host, s_fix[lane] = g;
            } else {
                float tm, z;
                teacher_sums(a, r, true, lane, 32, tm, z);
                if (!SAVED) l = entries_loss(a, r, any, lane, 32, tm, z, m, s);
                for (int i = lane; GRAD && i < a.k; i += 32) {
                    const Entry e = r.entry(i);
                    s_fix_host[i] = e.host;
                    if (e.host >= 0) s_fix[i] = entry_grad(a, r, e, tm, z, m, s, gmul);
                }
            }
            if (!SAVED && lane == 0) {
                if (a.loss) a.loss[row] = any ? l : 0.0f;
                if (a.stats) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
            }
        }
        if (GRAD) {
            T *grad = static_cast<T *>(a.grad) + row * a.gstride;
            const float fac = gmul * inv_s * (SAVED ? 1.0f : exp_from(m_warp, m, a.c));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (any) {
                    scale_all<VEC>(v[c], fac);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[c][i] = 0.0f;
                }
                if ((c + 1) * chunk <= lay.whole - base)
                    __stcs(reinterpret_cast<uint4 *>(grad + first + c * chunk), pack16(v[c], T()));
                else
                    store_cols<T, VEC>(grad, first + c * chunk, a.n, v[c], a.wide);
            }
            if (any) fix_grad = grad;
        }
        st = st == kBlockStages - 1 ? 0 : st + 1;
    }
    __syncthreads();
    fix();
}

// (m, s) with s relative to m, merged with (m2, s2)
__device__ __forceinline__ void merge_stats(float &m, float &s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2);
    s = s * exp_from(m, top, c) + s2 * exp_from(m2, top, c);
    m = top;
}

// ---- block form: blockDim.x * CS threads per row, CS = cluster size ----------------------------------------
// KEEP: the row stays in registers; otherwise (rows too long) it is read once more for the gradient.
template <typename T, int VEC, bool KEEP, bool GRAD, bool SAVED>
__global__ void __launch_bounds__(1024, 1) distill_block_kernel(DistillArgs a, int cs, int span)
{
    constexpr int CH = kElems / VEC;
    __shared__ float2 s_stats[kMaxCluster * 32];
    __shared__ float s_teacher[2];
    __shared__ float s_entry_x[NBOS_POLICY_MAX_K];
    const int rank = cluster_rank(cs);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const long long row = blockIdx.x / cs;
    const T *x = static_cast<const T *>(a.x) + row * a.stride;
    const long long first_col = (long long)rank * span, end_col = min((long long)a.n, first_col + span);
    const long long chunk = (long long)blockDim.x * VEC;

    cluster_arrive(cs);
    float v[CH][VEC];
    float m = neg_inf(), s = 0.0f;
    if (KEEP) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            load_cols<T, VEC>(x, first_col + c * chunk + threadIdx.x * VEC, end_col, neg_inf(), v[c]);
    }
    if (SAVED) {
        m = a.stats_in[2 * row];
        s = a.stats_in[2 * row + 1];
    } else if (KEEP) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) m = fmaxf(m, v[c][i]);
        m = lanes_max(m, 32);
    }
    if (KEEP) {
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] = exp_from(v[c][i], m, a.c);
                sum += v[c][i];
            }
        if (!SAVED) s = lanes_sum(sum, 32);
    } else if (!SAVED) {
        for (long long col = first_col + threadIdx.x * VEC; col < end_col; col += chunk) {
            float w[VEC];
            load_cols<T, VEC>(x, col, end_col, neg_inf(), w);
            float top = m;
#pragma unroll
            for (int i = 0; i < VEC; ++i) top = fmaxf(top, w[i]);
            s *= exp_from(m, top, a.c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += exp_from(w[i], top, a.c);
            m = top;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1)
            merge_stats(m, s, __shfl_xor_sync(kFull, m, off), __shfl_xor_sync(kFull, s, off), a.c);
    }
    const float m_warp = m;
    Entry first{-1, 0.0f, 0.0f};
    float tm = neg_inf(), z = 0.0f;
    if (warp == 0) {
        if (lane < a.k) first = load_entry(a, row, x, lane);
        teacher_stats(a, row, x, true, lane, 32, first, tm, z);
        if (lane == 0) s_teacher[0] = tm, s_teacher[1] = z;
    }
    // the listed hosts' logits, before a gradient may be written over them
    for (int k = threadIdx.x; GRAD && k < a.k; k += blockDim.x) s_entry_x[k] = load_entry(a, row, x, k).x;
    cluster_wait(cs);   // the other blocks run: their shared memory may be written
    if (!SAVED) {
        // every warp's (m, s) goes to every block of the cluster; each warp then merges all of them
        if (lane < cs) {
            float2 *dst = cluster_peer(s_stats, lane, cs);
            dst[rank * warps + warp] = make_float2(m, s);
        }
    }
    cluster_sync(cs);   // also: no block writes its gradient before the others have read the entries
    if (!SAVED) {
        m = neg_inf(), s = 0.0f;
        for (int i = lane; i < cs * warps; i += 32) merge_stats(m, s, s_stats[i].x, s_stats[i].y, a.c);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1)
            merge_stats(m, s, __shfl_xor_sync(kFull, m, off), __shfl_xor_sync(kFull, s, off), a.c);
    }
    tm = s_teacher[0], z = s_teacher[1];
    const bool any = tm > neg_inf();
    if (!SAVED && warp == 0 && rank == 0) {
        // listed hosts beyond the first 32 are re-read here: with a gradient the loss is taken before the barrier below
        const float l = row_loss(a, row, x, any, lane, 32, first, tm, z, m, s);
        if (lane == 0) {
            if (a.loss) a.loss[row] = any ? l : 0.0f;
            if (a.stats) a.stats[2 * row] = m, a.stats[2 * row + 1] = s;
        }
    }
    if (GRAD) {
        T *grad = static_cast<T *>(a.grad) + row * a.gstride;
        const float gmul = grad_multiplier(a, row);
        const float fac = gmul * reciprocal(s) * (KEEP ? exp_from(m_warp, m, a.c) : 1.0f);
        if (a.k > 32) cluster_sync(cs);   // row_loss has re-read logits that the next lines may write over
        if (KEEP) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[c][i] = any ? v[c][i] * fac : 0.0f;
                store_cols<T, VEC>(grad, first_col + c * chunk + threadIdx.x * VEC, end_col, v[c], a.wide);
            }
        } else {
            for (long long col = first_col + threadIdx.x * VEC; col < end_col; col += chunk) {
                float w[VEC];
                load_cols<T, VEC>(x, col, end_col, neg_inf(), w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) w[i] = any ? exp_from(w[i], m, a.c) * fac : 0.0f;
                store_cols<T, VEC>(grad, col, end_col, w, a.wide);
            }
        }
        __syncthreads();
        for (int k = threadIdx.x; any && k < a.k; k += blockDim.x) {
            Entry e;
            e.host = a.hosts[row * a.k + k];
            e.t = a.teacher ? a.teacher[row * a.tstride + k] : 0.0f;
            e.x = s_entry_x[k];
            if (e.host < first_col || e.host >= end_col || !(e.t > neg_inf()) || e.x == neg_inf()) continue;
            fix_entries(a, row, x, e, grad, tm, z, m, s, gmul);
        }
    }
}

int power_of_two(int n, int most)   // the first that is not below n
{
    int p = 1;
    while (p < n && p < most) p *= 2;
    return p;
}

template <typename T, int LANES, int CH, bool GRAD, bool SAVED>
cudaError_t launch_warp(const DistillArgs &a, const Layout &lay, int sms, cudaStream_t stream)
{
    auto *kernel = distill_warp_kernel<T, LANES, CH, GRAD, SAVED>;
    static const int regs = kernel_registers(kernel);
    const int shared = kWarps * kStages * lay.bytes();
    const cudaError_t e = allow_shared(kernel, shared);
    if (e != cudaSuccess) return e;
    const long long per_block = kWarps * (32 / LANES), wanted = (a.rows + per_block - 1) / per_block;
    const long long fit = (long long)sms * resident_blocks(regs, kWarps * 32, shared);
    kernel<<<(unsigned int)(wanted < fit ? wanted : fit), kWarps * 32, shared, stream>>>(a, power_of_two(a.k, LANES), lay);
    return cudaGetLastError();
}

template <typename T, int LANES, bool GRAD, bool SAVED>
cudaError_t launch_chunks(const DistillArgs &a, int chunks, const Layout &lay, int sms, cudaStream_t stream)
{
    constexpr int VEC = kPer16<T>;
    if (chunks == 1) return launch_warp<T, LANES, 1, GRAD, SAVED>(a, lay, sms, stream);
    if (chunks == 2) return launch_warp<T, LANES, 2, GRAD, SAVED>(a, lay, sms, stream);
    if (chunks == 32 / VEC) return launch_warp<T, LANES, 32 / VEC, GRAD, SAVED>(a, lay, sms, stream);
    if (chunks == 40 / VEC) return launch_warp<T, LANES, 40 / VEC, GRAD, SAVED>(a, lay, sms, stream);
    return launch_warp<T, LANES, kMostElems<T> / VEC, GRAD, SAVED>(a, lay, sms, stream);
}

// The staged forms; false: not for these sizes.
template <typename T, bool GRAD, bool SAVED>
bool launch_staged(const DistillArgs &a, int sms, cudaStream_t stream, cudaError_t &e)
{
    constexpr int VEC = kPer16<T>;
    const bool aligned = rows_aligned16(a.x, a.rows, a.stride, sizeof(T));
    const int columns = a.n + (aligned ? 0 : VEC - 1);   // with those before an unaligned row
    // Lanes per row and 16-byte chunks per lane. What a row costs besides its elements, about as much as 36 elements a lane,
    // is shared by the warp's rows: as few lanes as that makes cheapest, no fewer than entries; but enough to give every SM
    // eight warps. Why 40 elements are among the shapes (against the next one): 694,444 x 144 bf16 107 us / 137, 333,333 x 300 bf16
    // 134 / 164, 156,250 x 640 bf16 93 / 118; 757,575 x 132 f32 155 / 207, 312,500 x 320 f32 148 / 171, 156,250 x 640 f32 145 / 166.
    constexpr int kChunks[] = {1, 2, 32 / VEC, 40 / VEC, 64 / VEC};
    int lanes = 32, chunks = kChunks[2];
    long long best = 1ll << 40;
    for (int l = 4; l <= 32; l *= 2)
        for (int c : kChunks) {
            if (l * c * VEC < columns || (l < 32 && l < a.k) || c * VEC > kMostElems<T>) continue;
            long long cost = (long long)l * (36 + c * VEC);
            if (l < 32 && a.rows * l < 32ll * 8 * sms) cost += (1ll << 30) / l;
            if (cost < best) best = cost, lanes = l, chunks = c;
        }
    const Layout warp_lay{staged_row_bytes(a.n, sizeof(T), aligned), 32 / lanes, a.k, aligned, aligned && a.wide ? a.n : 0};
    // (long lists of entries would leave room for one block only)
    if (columns <= kWarpRow && kWarps * kStages * warp_lay.bytes() <= 112 * 1024) {
        switch (lanes) {
        case 4: e = launch_chunks<T, 4, GRAD, SAVED>(a, chunks, warp_lay, sms, stream); break;
        case 8: e = launch_chunks<T, 8, GRAD, SAVED>(a, chunks, warp_lay, sms, stream); break;
        case 16: e = launch_chunks<T, 16, GRAD, SAVED>(a, chunks, warp_lay, sms, stream); break;
        default: e = launch_chunks<T, 32, GRAD, SAVED>(a, chunks, warp_lay, sms, stream); break;
        }
        return true;
    }
    const int threads = ((columns + kElems - 1) / kElems + 31) / 32 * 32;
    auto *kernel = distill_staged_kernel<T, GRAD, SAVED>;
    static const int regs = kernel_registers(kernel);
    const Layout lay{staged_row_bytes(a.n, sizeof(T), aligned), 1, a.k, aligned, aligned && a.wide ? a.n : 0};
    const int shared = kBlockStages * lay.bytes();
    // (fewer rows than that leave SMs without one, or with one block: the other form has several blocks to a row. Up to 592 rows of
    // 1,040 to 16,384 hosts both wait for the call on the host, 10 us; 444 x 16,384 bf16 12.3 us here, 16.3 there)
    if (threads > 512 || shared > kMostShared || a.rows < 2 * sms) return false;
    e = allow_shared(kernel, shared);
    if (e != cudaSuccess) return true;
    const long long fit = (long long)sms * resident_blocks(regs, threads, shared + 2560);
    kernel<<<(unsigned int)(a.rows < fit ? a.rows : fit), threads, shared, stream>>>(a, power_of_two(a.k, 32), lay);
    e = cudaGetLastError();
    return true;
}

template <typename T, int VEC, bool GRAD, bool SAVED>
cudaError_t launch(const DistillArgs &a, int sms, cudaStream_t stream)
{
    cudaError_t staged = cudaSuccess;
    if (launch_staged<T, GRAD, SAVED>(a, sms, stream, staged)) return staged;
    // One block per row while the rows fill the GPU; more blocks per row when they do not, or when the row needs them
    const bool keep = a.n <= kMaxCluster * 1024 * kElems;
    int cs = 1;
    auto threads_for = [&](int c) { return ((a.n + c * kElems - 1) / (c * kElems) + 31) / 32 * 32; };
    while (cs < kMaxCluster && (threads_for(cs) > 1024 || (a.rows * cs < 2 * sms && threads_for(cs) > 128))) cs *= 2;
    const int threads = keep ? threads_for(cs) : 1024;
    const int span = ((a.n + cs - 1) / cs + VEC - 1) / VEC * VEC;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    // grid.x holds rows * cs blocks: 2^31 - 1 at most, so very many rows go in several launches
    const long long rows_per_launch = 2147483647ll / kMaxCluster;
    for (long long r = 0; r < a.rows; r += rows_per_launch) {
        DistillArgs b = a;
        b.rows = a.rows - r < rows_per_launch ? a.rows - r : rows_per_launch;
        b.x = static_cast<const T *>(a.x) + r * a.stride;
        b.hosts += r * a.k;
        if (b.teacher) b.teacher += r * a.tstride;
        if (b.grad_loss) b.grad_loss += r;
        if (b.loss) b.loss += r;
        if (b.stats) b.stats += 2 * r;
        if (b.stats_in) b.stats_in += 2 * r;
        if (b.grad) b.grad = static_cast<T *>(a.grad) + r * a.gstride;
        cfg.gridDim = dim3((unsigned int)(b.rows * cs));
        cudaError_t e = keep ? cudaLaunchKernelEx(&cfg, distill_block_kernel<T, VEC, true, GRAD, SAVED>, b, cs, span)
                             : cudaLaunchKernelEx(&cfg, distill_block_kernel<T, VEC, false, GRAD, SAVED>, b, cs, span);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T>
cudaError_t dispatch(const DistillArgs &a, int sms, cudaStream_t stream)
{
    // the path, and with it every rounding, goes by the logits alone: the loss is the same with a gradient or without
    const bool vec = rows_aligned16(a.x, a.rows, a.stride, sizeof(T));
    constexpr int V = kPer16<T>;
    if (a.stats_in) return vec ? launch<T, V, true, true>(a, sms, stream) : launch<T, 1, true, true>(a, sms, stream);
    if (a.grad) return vec ? launch<T, V, true, false>(a, sms, stream) : launch<T, 1, true, false>(a, sms, stream);
    return vec ? launch<T, V, false, false>(a, sms, stream) : launch<T, 1, false, false>(a, sms, stream);
}

int distill(const nbos_logits *l, const int32_t *hosts, const float *teacher, int64_t tstride, int32_t k, float T,
            const float *stats_in, const float *grad_loss, float grad_scale, float *out_loss, float *out_stats,
            void *out_grad, int64_t gstride, cudaStream_t stream)
{
    int rc = check_logits(l);
    if (rc || (rc = check_k(k))) return rc;
    if (!(T > 0.0f) || !isfinite(T) || !isfinite(kLog2e / T) || !isfinite(T * T))
        return fail(NBOS_ERR_INVALID_ARG, "temperature must be finite and > 0 (as must 1 / T and T^2)");
    if (tstride != 0 && (tstride < k || tstride > ((int64_t)1 << 40)))
        return fail(NBOS_ERR_INVALID_ARG, "teacher_stride must be 0 or in k..2^40 (got %lld)", (long long)tstride);
    if (l->rows == 0) return NBOS_OK;
    if (!out_loss && !out_stats && !out_grad) return fail(NBOS_ERR_INVALID_ARG, "no output asked for");
    if (!hosts) return fail(NBOS_ERR_INVALID_ARG, "hosts is NULL");
    if (out_grad && (rc = check_grad(l, out_grad, gstride))) return rc;
    if (out_grad == l->data && out_grad && l->rows > 1 && gstride != l->row_stride)
        return fail(NBOS_ERR_INVALID_ARG, "a gradient written over the logits needs their row_stride");
    if (!aligned_to(hosts, 4) || !aligned_to(teacher, 4) || !aligned_to(grad_loss, 4) || !aligned_to(out_loss, 4) ||
        !aligned_to(out_stats, 4) || !aligned_to(stats_in, 4))
        return fail(NBOS_ERR_INVALID_ARG, "an int32 / float array is not 4-byte aligned");
    int sms = 0, device = 0;
    if ((rc = check_sm100(&sms, &device))) return rc;
    DistillArgs a{l->data, l->rows, l->row_stride, l->n_hosts, hosts, teacher, tstride, k, T, kLog2e / T, 1.0f / T,
                  grad_loss, grad_scale, out_loss, out_stats, stats_in, out_grad, gstride, false};
    if (a.rows == 1) a.stride = a.gstride = l->n_hosts;
    const long long apart = static_cast<const char *>(l->data) - static_cast<const char *>(out_grad);
    a.wide = !out_grad || (apart % 16 == 0 && (a.stride - a.gstride) * (long long)dtype_bytes(l->dtype) % 16 == 0);
    const cudaError_t e = l->dtype == NBOS_F32    ? dispatch<float>(a, sms, stream)
                          : l->dtype == NBOS_BF16 ? dispatch<__nv_bfloat16>(a, sms, stream)
                                                  : dispatch<__half>(a, sms, stream);
    if (e != cudaSuccess) return cuda_fail(e, "distillation launch");
    return NBOS_OK;
}

}  // namespace
}  // namespace nbos

using namespace nbos;

extern "C" int nbos_policy_distill(const nbos_logits *logits, const int32_t *hosts, const float *teacher_logits,
                                   int64_t teacher_stride, int32_t k, float temperature, const float *grad_loss,
                                   float grad_scale, float *out_loss, float *out_stats, void *out_grad,
                                   int64_t grad_stride, void *cuda_stream)
{
    return distill(logits, hosts, teacher_logits, teacher_stride, k, temperature, nullptr, grad_loss, grad_scale,
                   out_loss, out_stats, out_grad, grad_stride, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int nbos_policy_distill_backward(const nbos_logits *logits, const int32_t *hosts,
                                            const float *teacher_logits, int64_t teacher_stride, int32_t k,
                                            float temperature, const float *stats, const float *grad_loss,
                                            float grad_scale, void *out_grad, int64_t grad_stride, void *cuda_stream)
{
    if (logits && logits->rows > 0 && (!stats || !out_grad)) return fail(NBOS_ERR_INVALID_ARG, "stats / out_grad is NULL");
    return distill(logits, hosts, teacher_logits, teacher_stride, k, temperature, stats, grad_loss, grad_scale,
                   nullptr, nullptr, out_grad, grad_stride, static_cast<cudaStream_t>(cuda_stream));
}
