// Shared by the learned-policy kernels (distillation, balance loss, sampling): element types, loads and
// stores of a row, reductions over the lanes, warps and clustered blocks that share a row, and the argument
// checks the entry points have in common.
#ifndef NBOS_POLICY_CUH_
#define NBOS_POLICY_CUH_

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <utility>

#include "nbos_internal.h"

namespace nbos {
namespace policy {

constexpr float kLog2e = 1.4426950408889634f;
constexpr unsigned int kFull = 0xFFFFFFFFu;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xFF800000); }

// ---- elements: 32-bit arithmetic whatever the type, one rounding (to nearest even) at a store -------------
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

template <typename T> constexpr int kPer16 = 16 / (int)sizeof(T);

__device__ __forceinline__ void unpack16(const uint4 &u, float (&v)[4], float)
{
    v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack16(const uint4 &u, float (&v)[8], __nv_bfloat16)
{
    const unsigned int w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack16(const uint4 &u, float (&v)[8], __half)
{
    const unsigned int w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack16(const float (&v)[4], float)
{
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack16(const float (&v)[8], __nv_bfloat16)
{
    unsigned int w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned int *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack16(const float (&v)[8], __half)
{
    unsigned int w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned int *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// four neighbouring elements as they are in memory, from a boundary of four elements
template <typename T> struct Raw4;
template <> struct Raw4<float> {
    float4 v;
    __device__ __forceinline__ void load(const float *p) { v = __ldcs(reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void set(int i, float x) { (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w) = x; }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w; }
};
template <typename T> struct Raw4Half {
    uint2 v;
    __device__ __forceinline__ void load(const T *p) { v = __ldcs(reinterpret_cast<const uint2 *>(p)); }
    __device__ __forceinline__ void set(int i, T x)
    {
        const unsigned int b = *reinterpret_cast<const unsigned short *>(&x);
        unsigned int &w = i < 2 ? v.x : v.y;
        w = i % 2 ? (w & 0xFFFFu) | (b << 16) : (w & 0xFFFF0000u) | b;
    }
};
template <> struct Raw4<__nv_bfloat16> : Raw4Half<__nv_bfloat16> {
    __device__ __forceinline__ void get(float (&f)[4]) const
    {
        f[0] = __uint_as_float(v.x << 16), f[1] = __uint_as_float(v.x & 0xFFFF0000u);
        f[2] = __uint_as_float(v.y << 16), f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
};
template <> struct Raw4<__half> : Raw4Half<__half> {
    __device__ __forceinline__ void get(float (&f)[4]) const
    {
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2 *>(&v.y));
        f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
    }
};

// VEC consecutive elements of a row from column `col`; columns from `end` on read as `fill`. VEC is 16 bytes'
// worth (the row then starts on a 16-byte boundary and col is a multiple of VEC) or 1 (any alignment).
// Loads are plain (not through the read-only path): the gradient may be written over the logits.
template <typename T, int VEC>
__device__ __forceinline__ void load_cols(const T *row, long long col, long long end, float fill, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        v[0] = col < end ? to_float(__ldcs(row + col)) : fill;
    } else {
        if (col + VEC <= end) {
            unpack16(__ldcs(reinterpret_cast<const uint4 *>(row + col)), v, T());
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = col + i < end ? to_float(__ldcs(row + col + i)) : fill;
        }
    }
}
__device__ __forceinline__ void store_pair(unsigned short *at, unsigned int w, bool first, bool second);
// `wide`: row + col lies on a 16-byte boundary
template <typename T, int VEC, typename I>
__device__ __forceinline__ void store_cols(T *row, I col, I end, const float (&v)[VEC], bool wide = true)
{
    if constexpr (VEC == 1) {
        if (col < end) __stcs(row + col, from_float<T>(v[0]));
    } else {
        if (wide && col >= 0 && col + VEC <= end) {
            __stcs(reinterpret_cast<uint4 *>(row + col), pack16(v, T()));
        } else if (col >= end) {
        } else if (sizeof(T) == 2 && wide) {
            const uint4 u = pack16(v, T());
            const unsigned int w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) {
                const I c = col + 2 * i;
                store_pair(reinterpret_cast<unsigned short *>(row + c), w[i % 4], c >= 0 && c < end, c + 1 >= 0 && c + 1 < end);
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (col + i >= 0 && col + i < end) __stcs(row + col + i, from_float<T>(v[i]));
        }
    }
}

// ---- reductions over `lanes` neighbouring lanes (a power of two; every lane gets the result) ---------------
__device__ __forceinline__ float warp_max(float v)   // NaN is never the larger
{
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}
__device__ __forceinline__ float lanes_max(float v, int lanes)
{
    if (lanes == 32) return warp_max(v);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        if (off < lanes) v = fmaxf(v, __shfl_xor_sync(kFull, v, off));
    return v;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        if (off < lanes) v += __shfl_xor_sync(kFull, v, off);
    return v;
}

// 2^y to 2 ulp; results below the smallest normal number are 0
__device__ __forceinline__ float exp2_fast(float y)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y));
    return e;
}
// 2^((x - m) c); 0 where x is -inf even if m is -inf (a row without a finite logit). The subtraction comes
// first: near the row's maximum, where the result matters, it is exact or nearly so.
__device__ __forceinline__ float exp_from(float x, float m, float c)
{
    return exp2_fast((x - (m == neg_inf() ? 0.0f : m)) * c);
}
// two 32-bit operations in one instruction, each rounded to nearest as the single ones are
__device__ __forceinline__ void add2(float &a0, float &a1, float b0, float b1)   // a += b
{
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}
__device__ __forceinline__ void mul2(float &a0, float &a1, float b0, float b1)   // a *= b
{
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}
__device__ __forceinline__ void fma2(float &d0, float &d1, float a0, float a1, float b0, float b1)   // d += a b
{
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\t"
        "fma.rn.f32x2 x, y, z, x;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(d0), "+f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// v = 2^((v - m0) c) over a lane's elements; returns their sum (single elements: an even number of chunks, or one). Two sums
// in turn: one would have every addition wait for the one before.
template <int VEC, int CH>
__device__ __forceinline__ float exp_all(float (&v)[CH][VEC], float m0, float c)
{
    float s[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        if constexpr (VEC == 1 && CH == 1) {
            s[0][0] = v[0][0] = exp2_fast((v[0][0] - m0) * c);
        } else if constexpr (VEC == 1) {
            if (k % 2) continue;
            add2(v[k][0], v[k + 1][0], -m0, -m0);
            mul2(v[k][0], v[k + 1][0], c, c);
            v[k][0] = exp2_fast(v[k][0]), v[k + 1][0] = exp2_fast(v[k + 1][0]);
            add2(s[k / 2 % 2][0], s[k / 2 % 2][1], v[k][0], v[k + 1][0]);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                add2(v[k][i], v[k][i + 1], -m0, -m0);
                mul2(v[k][i], v[k][i + 1], c, c);
                v[k][i] = exp2_fast(v[k][i]), v[k][i + 1] = exp2_fast(v[k][i + 1]);
                add2(s[i / 2 % 2][0], s[i / 2 % 2][1], v[k][i], v[k][i + 1]);
            }
        }
    }
    return (s[0][0] + s[0][1]) + (s[1][0] + s[1][1]);
}
// v *= f
template <int VEC>
__device__ __forceinline__ void scale_all(float (&v)[VEC], float f)
{
    if constexpr (VEC == 1) {
        v[0] *= f;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) mul2(v[i], v[i + 1], f, f);
    }
}
template <int VEC, int CH>
__device__ __forceinline__ float max_all(const float (&v)[CH][VEC])
{
    float m[4] = {neg_inf(), neg_inf(), neg_inf(), neg_inf()};
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) m[(k * VEC + i) % 4] = fmaxf(m[(k * VEC + i) % 4], v[k][i]);
    return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

__device__ __forceinline__ float reciprocal(float x) { return __fdividef(1.0f, x); }   // 2 ulp

// ---- rows staged in shared memory by asynchronous copies ----------------------------------------------------
constexpr int kStages = 2;   // rows on their way or in use per team (a warp, or a block); 3 and 4 measured the same

__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src, int bytes)   // the rest of the 16 becomes 0
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_drain() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int PENDING = kStages - 1>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
}

// Bytes between the 16-byte boundary before a row and the row itself; they are staged along.
template <typename T>
__device__ __forceinline__ int row_shift(const T *row)
{
    return (int)(reinterpret_cast<uintptr_t>(row) & 15);
}
// Queues the copies of n elements from `row` to `dst` (16-byte aligned; the row itself lands row_shift bytes further),
// thread `sub` of `team`. The bytes before an unaligned row belong to the rows before it (or the gaps between them);
// where the table does not have that many (`offset`: the row's, in bytes), the first, partial 16 bytes go element by
// element.
// Only the 16-byte pieces from, ..., until - 1; piece `origin` lands at `dst`.
template <typename T>
__device__ __forceinline__ void stage_row(char *dst, const T *row, int n, long long offset, int sub, int team, int from = 0, int until = 1 << 30,
                                          int origin = 0)
{
    const int shift = row_shift(row), total = shift + n * (int)sizeof(T);
    const char *src = reinterpret_cast<const char *>(row) - shift;
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(dst)) - origin * 16;
    int g = from + sub;
    if (offset < shift && from == 0) {
        for (int i = sub; i < n && shift + (i + 1) * (int)sizeof(T) <= 16; i += team) reinterpret_cast<T *>(dst + shift)[i] = row[i];
        if (sub == 0) g = team;   // the pieces of 16 bytes after it
    }
    const int whole = min(total >> 4, until);
#pragma unroll 4
    for (; g < whole; g += team) copy_async16(to + g * 16, src + g * 16);
    if (g == total >> 4 && g < until && (total & 15)) copy_async16(to + g * 16, src + g * 16, total & 15);
}
// Bytes of a staged row, with what precedes an unaligned one.
inline int staged_row_bytes(int n, int elem, bool aligned) { return (n * elem + (aligned ? 0 : 15) + 15) & ~15; }
// VEC elements (16 bytes) of a staged row from column `col`, which lies on a 16-byte boundary and may be below 0: columns
// outside the row read as -inf
template <typename T, int VEC>
__device__ __forceinline__ void staged_cols(const T *row, int col, int n, float (&v)[VEC])
{
    if (col < n) {   // the boundary before a row and its last 16 bytes are staged whole
        unpack16(*reinterpret_cast<const uint4 *>(row + col), v, T());
        if (col < 0 || col + VEC > n) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = (unsigned int)(col + i) < (unsigned int)n ? v[i] : neg_inf();
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = neg_inf();
    }
}
// two neighbours on a 4-byte boundary, either of them perhaps outside the row
__device__ __forceinline__ void store_pair(unsigned short *at, unsigned int w, bool first, bool second)
{
    if (first && second)
        __stcs(reinterpret_cast<unsigned int *>(at), w);
    else if (first)
        __stcs(at, (unsigned short)w);
    else if (second)
        __stcs(at + 1, (unsigned short)(w >> 16));
}

// ---- blocks that share a row: a cluster of `cs` blocks, or one block (cs = 1) ------------------------------
__device__ __forceinline__ int cluster_rank(int cs)
{
    return cs > 1 ? (int)cooperative_groups::this_cluster().block_rank() : 0;
}
// arrive + wait: every block of the cluster has started, so its shared memory may be written from outside
__device__ __forceinline__ void cluster_arrive(int cs)
{
    if (cs > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait(int cs)
{
    if (cs > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync(int cs)
{
    if (cs > 1)
        cooperative_groups::this_cluster().sync();
    else
        __syncthreads();
}
template <typename V>
__device__ __forceinline__ V *cluster_peer(V *shared, int rank, int cs)
{
    return cs > 1 ? cooperative_groups::this_cluster().map_shared_rank(shared, rank) : shared;
}

// 16 of the 32 bytes lo, hi, from byte `from` on
__device__ __forceinline__ uint4 window16(const uint4 &lo, const uint4 &hi, int from)
{
    unsigned int w[7] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z};
    if (from & 8) w[0] = w[2], w[1] = w[3], w[2] = w[4], w[3] = w[5], w[4] = w[6], w[5] = hi.w;
    if (from & 4) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = w[4], w[4] = w[5];
    if (from & 3) {
        const int bits = (from & 3) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- kernels in a row --------------------------------------------------------------------------------------
// A kernel launched by launch_next may start while the one before it in the stream still runs: it sets itself up and
// then waits, before it touches memory, until that one has finished and its results can be seen. Every kernel of such a row waits.
__device__ __forceinline__ void previous_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- host side --------------------------------------------------------------------------------------------
template <typename... P, typename... A>
inline cudaError_t launch_next(void (*kernel)(P...), dim3 grid, int threads, size_t shared, cudaStream_t stream, A &&...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}
inline size_t dtype_bytes(int dtype) { return dtype == NBOS_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int check_logits(const nbos_logits *l)
{
    if (!l) return fail(NBOS_ERR_INVALID_ARG, "logits is NULL");
    if (l->dtype != NBOS_F32 && l->dtype != NBOS_BF16 && l->dtype != NBOS_F16)
        return fail(NBOS_ERR_INVALID_ARG, "unknown dtype %d", l->dtype);
    if (l->n_hosts < 1 || l->n_hosts > NBOS_MAX_HOSTS)
        return fail(NBOS_ERR_INVALID_ARG, "n_hosts must be in 1..%d (got %d)", NBOS_MAX_HOSTS, l->n_hosts);
    if (l->rows < 0 || l->rows > NBOS_POLICY_MAX_ROWS)
        return fail(NBOS_ERR_INVALID_ARG, "rows must be in 0..2^31 - 1 (got %lld)", (long long)l->rows);
    if (l->rows > 1 && (l->row_stride < l->n_hosts || l->row_stride > ((int64_t)1 << 40)))
        return fail(NBOS_ERR_INVALID_ARG, "row_stride must be in n_hosts..2^40 (got %lld)", (long long)l->row_stride);
    if (l->rows > 0 && !l->data) return fail(NBOS_ERR_INVALID_ARG, "logits->data is NULL");
    if (!aligned_to(l->data, dtype_bytes(l->dtype)))
        return fail(NBOS_ERR_INVALID_ARG, "logits->data is not aligned to its element type");
    return NBOS_OK;
}
inline int check_grad(const nbos_logits *l, const void *grad, int64_t grad_stride)
{
    if (!aligned_to(grad, dtype_bytes(l->dtype)))
        return fail(NBOS_ERR_INVALID_ARG, "out_grad is not aligned to its element type");
    if (l->rows > 1 && (grad_stride < l->n_hosts || grad_stride > ((int64_t)1 << 40)))
        return fail(NBOS_ERR_INVALID_ARG, "grad_stride must be in n_hosts..2^40 (got %lld)", (long long)grad_stride);
    return NBOS_OK;
}
inline int check_k(int32_t k)
{
    if (k < 1 || k > NBOS_POLICY_MAX_K) return fail(NBOS_ERR_INVALID_ARG, "k must be in 1..%d (got %d)", NBOS_POLICY_MAX_K, k);
    return NBOS_OK;
}
inline int check_sm100(int *sms, int *device)
{
    int major = 0;
    NBOS_CUDA_TRY(cudaGetDevice(device));
    NBOS_CUDA_TRY(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *device));
    if (major != 10) return fail(NBOS_ERR_UNSUPPORTED_DEVICE, "device %d has compute capability %d.x", *device, major);
    NBOS_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *device));
    return NBOS_OK;
}
// Dynamic shared memory that a block of any form takes at most; with the kernels' static part, less than 7 KB, what an SM has.
constexpr int kMostShared = 220 * 1024;
// Before a launch with `bytes` of it. A launch has 48 KB, static and dynamic together, unless the kernel has been allowed more. What is
// allowed belongs to the kernel, not to the launch, and another host thread may be about to launch it with another size: so
// it is the same for every size.
template <typename K>
inline cudaError_t allow_shared(K *kernel, int bytes)
{
    return bytes > 40 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared) : cudaSuccess;
}
// Blocks of a kernel that an SM holds at once: what a persistent grid is sized by. regs: the kernel's registers.
inline int resident_blocks(int regs, int threads, size_t shared)
{
    // a quarter of the SM has 16,384 registers for whole warps
    const int by_regs = 4 * (512 / ((regs + 7) & ~7)) / ((threads + 31) / 32);
    const int by_shared = (int)((228 * 1024) / (shared + 1024));
    const int by_threads = 2048 / threads;
    int n = by_regs < by_shared ? by_regs : by_shared;
    n = n < by_threads ? n : by_threads;
    return n < 1 ? 1 : n;
}
template <typename K>
inline int kernel_registers(K *kernel)
{
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, kernel) != cudaSuccess) {
        cudaGetLastError();
        return 128;
    }
    return attr.numRegs;
}
// every row of `p` starts on a 16-byte boundary
inline bool rows_aligned16(const void *p, int64_t rows, int64_t stride, size_t elem)
{
    return aligned_to(p, 16) && (rows <= 1 || (stride * elem) % 16 == 0);
}

}  // namespace policy
}  // namespace nbos
#endif
