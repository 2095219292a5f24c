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

// sum over the warp of values below 2^52, by two 26-bit halves
__device__ __forceinline__ u64 warp_sum(u64 v)
{
    const unsigned int lo = __reduce_add_sync(kFull, (unsigned int)v & 0x3FFFFFFu);
    const unsigned int hi = __reduce_add_sync(kFull, (unsigned int)(v >> 26));
    return ((u64)hi << 26) + lo;
}

// floor(total * floor(share * 2^24) / 2^24) for a share in [0, 1]; total below 2^52
__device__ __forceinline__ u64 share_of(u64 total, unsigned int steps)
{
    return (u64)steps * (total >> 24) + (((u64)steps * (total & 0xFFFFFFu)) >> 24);
}

// The warps that share a row. MULTI = false: one warp, no shared memory.
template <bool MULTI>
struct Team {
    ulonglong2 (*slots)[kMaxCluster * 32];   // two sets, taken in turn
    int warps, cs, me, lane, turn;           // me: this warp's place among all of the row

    // every warp's (a, b), which the lanes of a warp agree on, to every warp; then slots[done]
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
    __device__ __forceinline__ float max(float v)
    {
        v = lanes_max(v, 32);
        if (!MULTI) return v;
        const int now = exchange(__float_as_uint(v), 0);
        v = neg_inf();
        for (int i = lane; i < warps; i += 32) v = fmaxf(v, __uint_as_float((unsigned int)slots[now][i].x));
        return lanes_max(v, 32);
    }
    // weight in the warps before this one
    __device__ __forceinline__ u64 before(u64 mine)
    {
        if (!MULTI) return 0;
        const int now = exchange(mine, 0);
        u64 sum = 0;
        for (int i = lane; i < me; i += 32) sum += slots[now][i].x;
        return warp_sum(sum);
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

// A lane's elements: registers (REGS), or the workspace for rows that do not fit. chunk c of the lane covers the
// columns base + (c * 32 + lane) * VEC ...
template <int VEC, int CH, bool REGS>
struct Elems {
    unsigned int r[REGS ? CH * VEC : 1];
    unsigned int *store;
    int chunks;
    long long base, n;   // first column of the lane's chunk 0; columns of the row
    template <typename F>
    __device__ __forceinline__ void each(F f)   // f(value &, column)
    {
        if (REGS) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) f(r[c * VEC + i], (int)base + c * 32 * VEC + i);
        } else {
            for (int c = 0; c < chunks; ++c)
                for (int i = 0; i < VEC; ++i) {
                    const long long col = base + (long long)c * 32 * VEC + i;
                    if (col >= n) return;
                    unsigned int v = store[col];
                    f(v, (int)col);
                    store[col] = v;
                }
        }
    }
    // the first column, in index order over the warp, at which the running sum of value(element, column) from `from`
    // exceeds t; the warp must hold it. Returns the column and the value there.
    template <typename F>
    __device__ __forceinline__ void find(u64 t, u64 from, int lane, F value, int &col_out, u64 &val_out)
    {
        u64 run = from, s_found = 0, run_found = 0;
        int c_found = -1;
        auto step = [&](int c) {
            if (c_found >= 0) return;
            u64 s = 0;
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += at(c, i, value);
            const u64 total = warp_sum(s);
            if (t < run + total) c_found = c, s_found = s, run_found = run;
            run += total;
        };
        if (REGS) {
#pragma unroll
            for (int c = 0; c < CH; ++c) step(c);
        } else {
            for (int c = 0; c < chunks; ++c) step(c);
        }
        u64 upto = s_found;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const u64 other = __shfl_up_sync(kFull, upto, off);
            if (lane >= off) upto += other;
        }
        upto += run_found;
        const unsigned int over = __ballot_sync(kFull, t < upto);
        const int owner = __ffs(over) - 1;
        u64 acc = upto - s_found, val = 0;
        int col = -1;
        auto look = [&](int c) {
            if (c != c_found) return;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const u64 v = at(c, i, value);
                acc += v;
                if (col < 0 && t < acc) col = (int)(base + (long long)c * 32 * VEC + i), val = v;
            }
        };
        if (REGS) {
#pragma unroll
            for (int c = 0; c < CH; ++c) look(c);
        } else {
            if (c_found >= 0) look(c_found);
        }
        col_out = __shfl_sync(kFull, col, owner);
        val_out = __shfl_sync(kFull, val, owner);
    }
    template <typename F>
    __device__ __forceinline__ u64 at(int c, int i, F value)
    {
        const long long col = base + (long long)c * 32 * VEC + i;
        if (REGS) return value(r[c * VEC + i], (int)col);
        return col < n ? value(store[col], (int)col) : 0;
    }
};

// The column of the m-th (from 0) element, in index order over the row, that `pick` accepts.
template <bool MULTI, typename E, typename F>
__device__ __forceinline__ int nth_column(Team<MULTI> &team, E &e, u64 m, F pick)
{
    auto one = [&](unsigned int v, int col) -> u64 { return pick(v, col) ? 1 : 0; };
    u64 mine = 0;
    e.each([&](unsigned int &v, int col) { mine += one(v, col); });
    mine = warp_sum(mine);
    const u64 before = team.before(mine);
    int col = -1;
    u64 val = 0, where = 0;
    const bool has = m >= before && m < before + mine;
    if (has) e.find(m, before, team.lane, one, col, val);
    where = (u64)(unsigned int)col;
    team.tell(has, where, val);
    return (int)(unsigned int)where;
}

template <typename T, int CH, bool MULTI, bool REGS>
__device__ __forceinline__ void sample_row(const SampleArgs &a, long long row, Team<MULTI> team, unsigned int *store, int chunks)
{
    constexpr int VEC = kPer16<T>;
    const T *x = static_cast<const T *>(a.x) + row * a.stride;
    const int lane = team.lane;
    Elems<VEC, CH, REGS> e;
    e.store = store, e.chunks = chunks, e.n = a.n;
    e.base = (long long)team.me * (REGS ? CH : chunks) * 32 * VEC + lane * VEC;

    // logits, NaN as -inf, +inf as the largest finite float
    auto clean = [](float v) { return fminf(fmaxf(v, neg_inf()), 3.402823466e38f); };
    float m = neg_inf();
    if (REGS) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const long long col = e.base + c * 32 * VEC;
            float v[VEC];
            if (a.aligned) {
                load_cols<T, VEC>(x, col, a.n, neg_inf(), v);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = col + i < a.n ? to_float(x[col + i]) : neg_inf();
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float f = clean(v[i]);
                m = fmaxf(m, f);
                e.r[c * VEC + i] = __float_as_uint(f);
            }
        }
    } else {
        e.each([&](unsigned int &v, int col) {
            const float f = clean(to_float(x[col]));
            m = fmaxf(m, f);
            v = __float_as_uint(f);
        });
    }
    m = team.max(m);
    const float temperature = a.temperature ? a.temperature[row] : 1.0f;
    const bool greedy = !(temperature > 0x1p-20f);
    const float scale = __fdiv_rn(kLog2e, greedy ? 1.0f : temperature);
    // no contraction of the subtraction and the product: each is rounded
    auto weight = [&](float v) -> unsigned int {
        return (unsigned int)(exp2f(__fmul_rn(__fsub_rn(v, m), scale)) * 0x1p31f);
    };
    int k = greedy ? 1 : (a.top_k ? a.top_k[row] : 0);
    const bool none = m == neg_inf();

    // top-k: cut_key = the k-th largest key; of its ties the first `ties` in index order stay. Hosts below m - 32 / c
    // have weight 0: if at most k are above that, top-k changes nothing.
    unsigned int cut_key = 0;   // keys above it stay
    int tie_col = -1;           // and of the keys equal to it the columns up to this one
    if (!none && k > 0 && k < a.n) {
        auto above = [&](unsigned int key) -> u64 {
            u64 c = 0, d = 0;
            e.each([&](unsigned int &v, int) { c += key_of(__uint_as_float(v)) > key; });
            team.sum2(c, d);
            return c;
        };
        float lo_f = __fsub_rn(m, __fdiv_rn(32.0f, scale)), hi_f = m;
        unsigned int lo = key_of(lo_f), hi = key_of(m);
        if (lo >= hi) lo = key_of(neg_inf());   // m so large that the distance vanishes
        u64 above_lo = above(lo), above_hi = 0;
        bool exact = above_lo <= (u64)k;
        // invariant: above(hi) < k <= above(lo)
        for (int it = 0; !exact && hi - lo > 1; ++it) {
            unsigned int mid = lo + (hi - lo) / 2;
            if (it < 24) {   // halving the values converges faster than halving the keys at first
                const float f = 0.5f * lo_f + 0.5f * hi_f;
                const unsigned int g = key_of(f);
                if (g > lo && g < hi) mid = g;
            }
            const unsigned int b = mid & 0x80000000u ? mid ^ 0x80000000u : ~mid;
            const u64 c = above(mid);
            if (c >= (u64)k) {
                lo = mid, lo_f = __uint_as_float(b), above_lo = c;
                exact = c == (u64)k;
            } else {
                hi = mid, hi_f = __uint_as_float(b), above_hi = c;
            }
        }
        if (exact) {
            cut_key = lo;
        } else {
            cut_key = hi;
            tie_col = nth_column(team, e, (u64)k - above_hi - 1, [&](unsigned int v, int) { return key_of(__uint_as_float(v)) == cut_key; });
        }
    }
    // weights from here on
    u64 total = 0, count = 0;
    e.each([&](unsigned int &v, int col) {
        const float f = __uint_as_float(v);
        const unsigned int key = key_of(f);
        v = !none && (key > cut_key || (key == cut_key && col <= tie_col)) ? weight(f) : 0u;
        total += v;
        count += v != 0;
    });
    team.sum2(total, count);

    const float p = a.top_p ? a.top_p[row] : 1.0f;
    if (p < 1.0f && !greedy && total > 0) {
        const unsigned int steps = (unsigned int)(fmaxf(p, 0.0f) * 0x1p24f);
        u64 limit = share_of(total, steps);
        if (limit == 0) limit = 1;
        // invariant: mass(w > hi) < limit <= mass(w > lo)
        unsigned int lo = 0, hi = 0x80000000u;
        u64 mass_hi = 0, count_hi = 0, count_lo = count;
        while (hi - lo > 1 && count_lo - count_hi > 1) {
            // halfway between the logarithms; at the ends of that, halfway between the values
            unsigned int mid = __float2uint_rd(__uint_as_float((__float_as_uint(__uint2float_rn(lo ? lo : 1)) + __float_as_uint(__uint2float_rn(hi))) / 2));
            if (mid <= lo || mid >= hi) mid = lo + (hi - lo) / 2;
            u64 mass = 0, c = 0;
            e.each([&](unsigned int &v, int) {
                if (v > mid) mass += v, ++c;
            });
            team.sum2(mass, c);
            if (mass < limit)
                hi = mid, mass_hi = mass, count_hi = c;
            else
                lo = mid, count_lo = c;
        }
        // One host between the bounds: it is the one that reaches the limit, and stays. Else all of them have
        // weight hi and the first ceil((limit - mass_hi) / hi) in (x descending, index ascending) stay.
        unsigned int cut = lo;   // weights above it stay
        const u64 ties = count_lo - count_hi;
        if (ties > 1) {
            const u64 keep = (limit - mass_hi + hi - 1) / hi;
            if (keep < ties) {
                // the ties' logits may still differ: bisection on their keys
                auto key_at = [&](int col) { return key_of(clean(to_float(x[col]))); };
                unsigned int klo = 0, khi = 0xFFFFFFFFu;   // above(khi) < keep <= above(klo) among the ties
                u64 above_khi = 0, above_klo = ties;
                while (khi - klo > 1 && above_klo > keep) {
                    const unsigned int mid = klo + (khi - klo) / 2;
                    u64 c = 0, d = 0;
                    e.each([&](unsigned int &v, int col) {
                        if (v == hi) c += key_at(col) > mid;
                    });
                    team.sum2(c, d);
                    if (c >= keep)
                        klo = mid, above_klo = c;
                    else
                        khi = mid, above_khi = c;
                }
                unsigned int kcut = klo;
                int kcol = -1;
                if (above_klo > keep) {
                    kcut = khi;
                    kcol = nth_column(team, e, keep - above_khi - 1, [&](unsigned int v, int col) { return v == hi && key_at(col) == kcut; });
                }
                e.each([&](unsigned int &v, int col) {
                    if (v != hi) return;
                    const unsigned int key = key_at(col);
                    if (!(key > kcut || (key == kcut && col <= kcol))) v = 0;
                });
            }
        }
        e.each([&](unsigned int &v, int) {
            if (v <= cut) v = 0;
        });
    }
    const float min_p = a.min_p ? a.min_p[row] : 0.0f;
    if (min_p > 0.0f) {
        const unsigned int least = (unsigned int)(fminf(min_p, 1.0f) * 0x1p31f);
        e.each([&](unsigned int &v, int) {
            if (v < least) v = 0;
        });
    }
    u64 mine = 0;
    e.each([&](unsigned int &v, int) { mine += v; });
    mine = warp_sum(mine);
    int found = 0;
    for (int d = 0; d < a.draws; ++d) {
        u64 before = 0, left = mine;
        if (MULTI) {
            const int now = team.exchange(mine, 0);
            u64 all = 0;
            for (int i = lane; i < team.warps; i += 32) {
                const u64 v = team.slots[now][i].x;
                all += v;
                if (i < team.me) before += v;
            }
            left = warp_sum(all), before = warp_sum(before);
        }
        int col = -1;
        if (left > 0) {
            const float u = a.u[row * a.draws + d];
            unsigned int steps = (unsigned int)(fminf(fmaxf(u, 0.0f), 1.0f) * 0x1p24f);
            if (steps > 0xFFFFFFu) steps = 0xFFFFFFu;
            const u64 t = share_of(left, steps);
            const bool has = t >= before && t < before + mine;
            u64 val = 0, where = 0;
            if (has) {
                e.find(t, before, lane, [](unsigned int v, int) -> u64 { return v; }, col, val);
                mine -= val;
                e.each([&](unsigned int &v, int at) {
                    if (at == col) v = 0;
                });
            }
            where = (u64)(unsigned int)col;
            team.tell(has, where, val);
            col = (int)(unsigned int)where;
            ++found;
        }
        if (team.me == 0 && lane == 0) a.hosts[row * a.draws + d] = col;
    }
    if (a.found && team.me == 0 && lane == 0) a.found[row] = found;
}

template <typename T, int CH>
__global__ void __launch_bounds__(128) sample_warp_kernel(SampleArgs a)
{
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= a.rows) return;
    Team<false> team{nullptr, 1, 1, 0, (int)(threadIdx.x & 31), 0};
    sample_row<T, CH, false, true>(a, row, team, nullptr, CH);
}

// grid: REGS one block / cluster per row; else `clusters` of them take the rows in turn
template <typename T, bool REGS>
__global__ void __launch_bounds__(1024, 1) sample_block_kernel(SampleArgs a, int cs, int chunks)
{
    __shared__ ulonglong2 s_slots[2][kMaxCluster * 32];
    const int rank = cluster_rank(cs), warps = blockDim.x >> 5;
    Team<true> team{s_slots, warps * cs, cs, rank * warps + (int)(threadIdx.x >> 5), (int)(threadIdx.x & 31), 0};
    cluster_sync(cs);   // all blocks of the cluster run
    const long long first = blockIdx.x / cs, step = gridDim.x / cs;
    for (long long row = first; row < a.rows; row += step) {
        sample_row<T, kElems / kPer16<T>, true, REGS>(a, row, team, REGS ? nullptr : a.store + first * a.n, chunks);
        cluster_sync(cs);   // slots are free again
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
    const cudaError_t e = regs ? cudaLaunchKernelEx(&cfg, sample_block_kernel<T, true>, a, cs, chunks)
                               : cudaLaunchKernelEx(&cfg, sample_block_kernel<T, false>, a, cs, chunks);
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
