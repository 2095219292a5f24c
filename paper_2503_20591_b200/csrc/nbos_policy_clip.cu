// The global norm over many tensors, and clipping by it (nbos_policy_clip).
//
//   norm = (sum over all values of x^2)^(1/2), or max |x|;   x *= min(1, max_norm / (norm + 1e-6))
// Bound by memory: the values are read for the norm, read again and written. Tensors are cut into chunks of 16 KB; a
// block takes a run of neighbouring chunks, forward for the norm and backward for the scaling, so that what it read last, and
// the L2 cache still holds, is what it reads first the second time. Blocks' sums are added up in a fixed order by every block
// of the second launch. Few values take one launch of one cluster instead, whose blocks exchange their sums.
#include <math.h>

#include "nbos_policy.cuh"

namespace nbos {
namespace {

using namespace policy;

constexpr int kThreads = 256;
constexpr int kLoads = 4;                                 // 16-byte pieces of a chunk per thread
constexpr int kChunkBytes = kThreads * kLoads * 16;
constexpr int kFewTensors = 64, kManyTensors = 1100;      // per launch: what a kernel's parameters (32,764 bytes) hold
constexpr int kBlocksPerSm = 8;
constexpr int kCluster = 8;
constexpr long long kClusterChunks = 4 * kCluster;        // up to 512 KB one cluster does it all

template <int MAX>
struct Batch {
    const void *data[MAX];
    void *out[MAX];
    unsigned long long numel[MAX];                        // the type in bits 60 and up
    unsigned int first[MAX + 1];                          // number of chunks before the tensor
    int n;
    double *partial;                                      // one per block of all launches of the norm
    int partials, partial0;                               // all of them; this launch's first
    float max_norm;
    float *norm;
    int kind;
    bool scale;
};

template <int MAX>
__device__ __forceinline__ int tensor_of(const Batch<MAX> &b, unsigned int chunk)
{
    int lo = 0, hi = b.n - 1;   // the last tensor that starts at or before the chunk (tensors of no chunks are left out)
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (b.first[mid] <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double larger(double a, double b) { return b > a || b != b ? b : a; }   // NaN stays

// Sum of squares of v: in 32 bits where that can neither overflow nor lose what counts, else in 64.
template <int N>
__device__ __forceinline__ double squares(const float (&v)[N])
{
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i + 3 < N; i += 4) fma2(s[0], s[1], v[i], v[i + 1], v[i], v[i + 1]), fma2(s[2], s[3], v[i + 2], v[i + 3], v[i + 2], v[i + 3]);
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    // below 2^-80 values of 2^-63 and less, whose squares leave the normal numbers, may be what counts
    if (sum < 1e38f && sum > 0x1p-80f) return (double)sum;
    double d = 0.0;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i]));
    if (sum == 0.0f && top == 0.0f) return 0.0;
    for (int i = 0; i < N; ++i) d = fma((double)v[i], (double)v[i], d);
    return d;
}
template <int N>
__device__ __forceinline__ double magnitude(const float (&v)[N])
{
    double m = 0.0;
    float top = 0.0f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i])), nan |= v[i] != v[i];
    m = nan ? (double)__int_as_float(0x7FC00000) : (double)top;
    return m;
}
template <typename T>
__device__ __forceinline__ void load_all(float (&v)[kLoads * kPer16<T>], const T *x, bool wide, long long left)
{
    constexpr int V = kPer16<T>;
    if (wide && left >= kThreads * kLoads * V) {
        uint4 u[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) u[k] = reinterpret_cast<const uint4 *>(x)[k * kThreads + threadIdx.x];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float w[V];
            unpack16(u[k], w, T());
#pragma unroll
            for (int i = 0; i < V; ++i) v[k * V + i] = w[i];
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const long long at = (long long)(k * kThreads + threadIdx.x) * V;
        float w[V];
        if (wide && at + V <= left) {
            unpack16(*reinterpret_cast<const uint4 *>(x + at), w, T());
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = at + i < left ? to_float(x[at + i]) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[k * V + i] = w[i];
    }
}
template <typename T>
__device__ __forceinline__ void store_all(const float (&v)[kLoads * kPer16<T>], T *x, bool wide, long long left)
{
    constexpr int V = kPer16<T>;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const long long at = (long long)(k * kThreads + threadIdx.x) * V;
        float w[V];
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = v[k * V + i];
        if (wide && at + V <= left) {
            __stcs(reinterpret_cast<uint4 *>(x + at), pack16(w, T()));
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (at + i < left) x[at + i] = from_float<T>(w[i]);
        }
    }
}

// The factor comes from the norm in 64 bits: it is right even where the norm is beyond 32. One below the normal numbers would
// have lost bits, so it is applied in two steps.
struct Factor {
    float first, then;
};
__device__ __forceinline__ Factor clip_factor(double norm, float max_norm)
{
    if (isinf(max_norm) && norm == norm) return {1.0f, 1.0f};   // inf / inf otherwise where a value is infinite
    const double f = (double)max_norm / (norm + 1e-6);
    if (f < 0x1p-100) return {(float)(f * 0x1p64), 0x1p-64f};
    return {f < 1.0 ? (float)f : (f != f ? __int_as_float(0x7FC00000) : 1.0f), 1.0f};
}

template <typename T>
__device__ __forceinline__ void norm_chunk(const void *data, long long chunk, long long numel, int kind, double &sum)
{
    constexpr int N = kChunkBytes / sizeof(T);
    const T *x = static_cast<const T *>(data) + chunk * N;
    float v[kLoads * kPer16<T>];
    load_all(v, x, (reinterpret_cast<uintptr_t>(data) & 15) == 0, numel - chunk * N);
    if (kind == NBOS_NORM_2)
        sum += squares(v);
    else
        sum = larger(sum, magnitude(v));
}
template <typename T>
__device__ __forceinline__ void scale_chunk(const void *data, void *out, long long chunk, long long numel, Factor f)
{
    constexpr int N = kChunkBytes / sizeof(T);
    float v[kLoads * kPer16<T>];
    load_all(v, static_cast<const T *>(data) + chunk * N, (reinterpret_cast<uintptr_t>(data) & 15) == 0, numel - chunk * N);
    scale_all(v, f.first);
    if (f.then != 1.0f) scale_all(v, f.then);
    store_all(v, static_cast<T *>(out) + chunk * N, (reinterpret_cast<uintptr_t>(out) & 15) == 0, numel - chunk * N);
}

// chunks [from, to) of the batch, first to last; the norm's part of them (per thread)
template <int MAX>
__device__ double norm_run(const Batch<MAX> &b, unsigned int from, unsigned int to)
{
    double sum = 0.0;
    if (from >= to) return sum;
    int t = tensor_of(b, from);
    for (unsigned int c = from; c < to; ++c) {
        while (c >= b.first[t + 1]) ++t;
        const long long numel = (long long)(b.numel[t] & ((1ull << 60) - 1)), chunk = c - b.first[t];
        const int dtype = (int)(b.numel[t] >> 60);
        if (dtype == NBOS_F32)
            norm_chunk<float>(b.data[t], chunk, numel, b.kind, sum);
        else if (dtype == NBOS_BF16)
            norm_chunk<__nv_bfloat16>(b.data[t], chunk, numel, b.kind, sum);
        else
            norm_chunk<__half>(b.data[t], chunk, numel, b.kind, sum);
    }
    return sum;
}
// last to first
template <int MAX>
__device__ void scale_run(const Batch<MAX> &b, unsigned int from, unsigned int to, Factor factor)
{
    if (from >= to) return;
    int t = tensor_of(b, to - 1);
    for (unsigned int c = to; c-- > from;) {
        while (c < b.first[t]) --t;
        if (factor.first == 1.0f && b.out[t] == b.data[t]) continue;
        const long long numel = (long long)(b.numel[t] & ((1ull << 60) - 1)), chunk = c - b.first[t];
        const int dtype = (int)(b.numel[t] >> 60);
        if (dtype == NBOS_F32)
            scale_chunk<float>(b.data[t], b.out[t], chunk, numel, factor);
        else if (dtype == NBOS_BF16)
            scale_chunk<__nv_bfloat16>(b.data[t], b.out[t], chunk, numel, factor);
        else
            scale_chunk<__half>(b.data[t], b.out[t], chunk, numel, factor);
    }
}

// every thread gets the block's sum (or largest)
__device__ double block_total(double v, int kind)
{
    __shared__ double warps[kThreads / 32];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const double other = __shfl_xor_sync(kFull, v, off);
        v = kind == NBOS_NORM_2 ? v + other : larger(v, other);
    }
    __syncthreads();
    if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = v;
    __syncthreads();
    v = warps[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v = kind == NBOS_NORM_2 ? v + warps[w] : larger(v, warps[w]);
    return v;
}
template <int MAX>
__device__ __forceinline__ void run_of(const Batch<MAX> &b, unsigned int &from, unsigned int &to)
{
    const unsigned long long chunks = b.first[b.n];
    from = (unsigned int)(chunks * blockIdx.x / gridDim.x), to = (unsigned int)(chunks * (blockIdx.x + 1) / gridDim.x);
}

template <int MAX>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Batch<MAX> b)
{
    unsigned int from, to;
    run_of(b, from, to);
    const double total = block_total(norm_run(b, from, to), b.kind);
    if (threadIdx.x == 0) b.partial[b.partial0 + blockIdx.x] = total;
}

template <int MAX>
__global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ Batch<MAX> b)
{
    double v = 0.0;
    for (int i = threadIdx.x; i < b.partials; i += kThreads) v = b.kind == NBOS_NORM_2 ? v + b.partial[i] : larger(v, b.partial[i]);
    v = block_total(v, b.kind);
    const double norm = b.kind == NBOS_NORM_2 ? sqrt(v) : v;
    if (blockIdx.x == 0 && threadIdx.x == 0 && b.norm) *b.norm = (float)norm;
    if (!b.scale) return;
    unsigned int from, to;
    run_of(b, from, to);
    scale_run(b, from, to, clip_factor(norm, b.max_norm));
}

// All of it in one cluster.
template <int MAX>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads) small_kernel(const __grid_constant__ Batch<MAX> b)
{
    __shared__ double parts[kCluster];
    const auto cluster = cooperative_groups::this_cluster();
    cluster_arrive(kCluster);
    unsigned int from, to;
    run_of(b, from, to);
    const double total = block_total(norm_run(b, from, to), b.kind);
    cluster_wait(kCluster);   // every block has started
    if (threadIdx.x < kCluster) *cluster.map_shared_rank(&parts[blockIdx.x], threadIdx.x) = total;
    cluster.sync();
    double v = parts[0];
#pragma unroll
    for (int i = 1; i < kCluster; ++i) v = b.kind == NBOS_NORM_2 ? v + parts[i] : larger(v, parts[i]);
    const double norm = b.kind == NBOS_NORM_2 ? sqrt(v) : v;
    if (blockIdx.x == 0 && threadIdx.x == 0 && b.norm) *b.norm = (float)norm;
    if (b.scale) scale_run(b, from, to, clip_factor(norm, b.max_norm));
}

struct Tensors {
    const void *const *data;
    void *const *out;
    const int64_t *numel;
    const int32_t *dtype;
};
long long chunks_of(int64_t numel, int dtype) { return (numel * (int64_t)dtype_bytes(dtype) + kChunkBytes - 1) / kChunkBytes; }

// Tensors from `i` on, as many as fit; empty ones are left out.
template <int MAX>
int fill(Batch<MAX> &b, const Tensors &t, int i, int n)
{
    b.n = 0;
    unsigned int chunks = 0;
    for (; i < n && b.n < MAX; ++i) {
        if (t.numel[i] == 0) continue;
        const long long more = chunks_of(t.numel[i], t.dtype[i]);
        if (b.n > 0 && chunks + more > 0xFFFFFFFFll) break;
        b.data[b.n] = t.data[i], b.out[b.n] = t.out ? t.out[i] : nullptr;
        b.numel[b.n] = (unsigned long long)t.numel[i] | (unsigned long long)t.dtype[i] << 60;
        b.first[b.n++] = chunks;
        chunks += (unsigned int)more;
    }
    b.first[b.n] = chunks;
    return i;
}

template <int MAX>
int clip(const Tensors &t, int n, long long chunks, int launches, float max_norm, int kind, float *out_norm, int sms, int device, cudaStream_t stream)
{
    Batch<MAX> b;
    b.max_norm = max_norm, b.kind = kind, b.norm = out_norm, b.scale = t.out != nullptr;
    b.partial = nullptr, b.partials = b.partial0 = 0;
    if (launches <= 1 && chunks <= kClusterChunks) {
        fill(b, t, 0, n);
        small_kernel<MAX><<<kCluster, kThreads, 0, stream>>>(b);
        const cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? NBOS_OK : cuda_fail(e, "clipping launch");
    }
    const int blocks = sms * kBlocksPerSm;
    cudaMemPool_t pool = nullptr;
    int rc = library_pool(device, &pool);
    if (rc) return rc;
    cudaError_t e = cudaMallocFromPoolAsync(reinterpret_cast<void **>(&b.partial), sizeof(double) * blocks * launches, pool, stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(NBOS_ERR_NO_MEMORY, "device allocation failed: %s", cudaGetErrorString(e));
    }
    double *const partial = b.partial;
    for (int i = 0, k = 0; e == cudaSuccess && k < launches; ++k) {
        i = fill(b, t, i, n);
        b.partial0 = k * blocks;
        norm_kernel<MAX><<<blocks, kThreads, 0, stream>>>(b);
        e = cudaGetLastError();
    }
    b.partials = blocks * launches;
    for (int i = 0, k = 0; e == cudaSuccess && k < (b.scale ? launches : 1); ++k) {
        if (launches > 1) i = fill(b, t, i, n);
        scale_kernel<MAX><<<b.scale ? blocks : 1, kThreads, 0, stream>>>(b);
        e = cudaGetLastError();
        b.norm = nullptr;
    }
    cudaFreeAsync(partial, stream);
    return e == cudaSuccess ? NBOS_OK : cuda_fail(e, "clipping launch");
}

}  // namespace
}  // namespace nbos

using namespace nbos;
using namespace nbos::policy;

extern "C" int nbos_policy_clip(const void *const *data, void *const *out, const int64_t *numel, const int32_t *dtype, int32_t n_tensors,
                                float max_norm, int32_t norm_kind, float *out_norm, void *cuda_stream)
{
    if (n_tensors < 0) return fail(NBOS_ERR_INVALID_ARG, "n_tensors must be >= 0 (got %d)", n_tensors);
    if (n_tensors > 0 && (!data || !numel || !dtype)) return fail(NBOS_ERR_INVALID_ARG, "data / numel / dtype is NULL");
    if (norm_kind != NBOS_NORM_2 && norm_kind != NBOS_NORM_INF) return fail(NBOS_ERR_INVALID_ARG, "norm_kind must be NBOS_NORM_2 or NBOS_NORM_INF (got %d)", norm_kind);
    if (!(max_norm >= 0.0f)) return fail(NBOS_ERR_INVALID_ARG, "max_norm must be >= 0");
    if (!out && !out_norm) return fail(NBOS_ERR_INVALID_ARG, "no output asked for");
    if (!aligned_to(out_norm, 4)) return fail(NBOS_ERR_INVALID_ARG, "out_norm is not 4-byte aligned");
    long long chunks = 0, batch = 0;
    int filled = 0, launches = 1, used = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (dtype[i] != NBOS_F32 && dtype[i] != NBOS_BF16 && dtype[i] != NBOS_F16) return fail(NBOS_ERR_INVALID_ARG, "tensor %d: unknown dtype %d", i, dtype[i]);
        if (numel[i] < 0 || numel[i] > (int64_t)1 << 40) return fail(NBOS_ERR_INVALID_ARG, "tensor %d: numel must be in 0..2^40 (got %lld)", i, (long long)numel[i]);
        if (numel[i] == 0) continue;
        if (!data[i] || (out && !out[i])) return fail(NBOS_ERR_INVALID_ARG, "tensor %d is NULL", i);
        if (!aligned_to(data[i], dtype_bytes(dtype[i])) || (out && !aligned_to(out[i], dtype_bytes(dtype[i]))))
            return fail(NBOS_ERR_INVALID_ARG, "tensor %d is not aligned to its element type", i);
        const long long more = chunks_of(numel[i], dtype[i]);
        if (filled == kManyTensors || (filled > 0 && batch + more > 0xFFFFFFFFll)) ++launches, filled = 0, batch = 0;
        ++filled, ++used, batch += more, chunks += more;
    }
    int sms = 0, device = 0;
    const int rc = check_sm100(&sms, &device);
    if (rc) return rc;
    const Tensors t{data, out, numel, dtype};
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return used <= kFewTensors && launches == 1 ? clip<kFewTensors>(t, n_tensors, chunks, launches, max_norm, norm_kind, out_norm, sms, device, stream)
                                                : clip<kManyTensors>(t, n_tensors, chunks, launches, max_norm, norm_kind, out_norm, sms, device, stream);
}
