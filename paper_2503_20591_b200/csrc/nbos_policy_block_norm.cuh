// The norms around a residual block with its gate and scaled residual (nbos_policy_block_norm, nbos_policy_block_norm_backward).
//
//   y^ = y / sqrt(mean y^2 + eps),  n = y^ w_post,  r = alpha x + gate n,  r^ = r / sqrt(mean r^2 + eps),  h = r^ w_pre
//   e  = dh w_pre,  d = dr + (e - r^ mean(e r^)) / sqrt(mean r^2 + eps)             (the whole gradient of r)
//   dx = alpha d,  dgate = sum d n,  dw_post = sum d gate y^,  dw_pre = sum dh r^
//   f  = d gate w_post,  dy = (f - y^ mean(f y^)) / sqrt(mean y^2 + eps)
// Bound by memory: each table is read and written once. A row lives in registers, 8 or 16 values a thread, from its first load to
// its last store; forward and backward take two sums over a row each (the two roots are saved). r is computed again from x and y
// rather than read: the same traffic, without its rounding. Sums over rows stay in registers while a block goes through its
// rows; with a gate that many rows share, dgate and dw_post come from one sum: S = sum d y^ over those rows gives
// dgate = w_post S and gate S, the rows' part of dw_post.
#ifndef NBOS_POLICY_BLOCK_NORM_CUH_
#define NBOS_POLICY_BLOCK_NORM_CUH_

#include <math.h>
#include <type_traits>

#include "nbos_policy.cuh"

namespace nbos {
namespace block_norm {

using namespace policy;

constexpr int kTeams = 256;   // threads of a block whose rows take a warp or less

struct BlockArgs {
    const void *x, *y, *gate, *post, *pre;
    long long x_stride, y_stride, gate_stride;
    long long rows, rows_per_gate;
    int width;
    bool gate_f32, weight_f32;
    float alpha, eps, per_width;
    // forward
    void *out, *normed;
    long long out_stride, normed_stride;
    float *stats;
    // backward
    const float *saved;
    const void *dr, *dh;
    long long dr_stride, dh_stride;
    void *dx, *dy, *dgate;
    long long dx_stride, dy_stride;
    long long dgate_stride;
    float *partial;               // [blocks][2][width]
    int blocks_per_gate;          // > 1: several blocks share a gate's rows, each has one stretch of them; 1: a block has whole gates
};

__device__ __forceinline__ float one_value(const void *p, long long i, bool f32, float) { (void)f32; return static_cast<const float *>(p)[i]; }
template <typename T>
__device__ __forceinline__ float one_value(const void *p, long long i, bool f32, T)
{
    return f32 ? static_cast<const float *>(p)[i] : to_float(static_cast<const T *>(p)[i]);
}

// VEC neighbours that lie in memory as 16 bytes, 4 bytes or one value
template <typename T, int VEC>
__device__ __forceinline__ void unpack(float (&v)[VEC], const void *at)
{
    if constexpr (VEC == kPer16<T>) {
        unpack16(*static_cast<const uint4 *>(at), v, T());
    } else if constexpr (VEC == 2 && sizeof(T) == 2) {
        const unsigned int w = *static_cast<const unsigned int *>(at);
        const unsigned short lo = (unsigned short)w, hi = (unsigned short)(w >> 16);
        v[0] = to_float(*reinterpret_cast<const T *>(&lo)), v[1] = to_float(*reinterpret_cast<const T *>(&hi));
    } else {
        v[0] = to_float(*static_cast<const T *>(at));
    }
}
// The columns of a thread: pieces of VEC, `team` of them apart. Piece k is whole, or the row's last and cut off, or behind it.
struct Columns {
    int team, t, width, whole, rest;
    __device__ __forceinline__ Columns(int team_, int t_, int width_, int vec) : team(team_), t(t_), width(width_), whole(width_ / vec - t_), rest(width_ % vec) {}
    __device__ __forceinline__ bool is_whole(int k) const { return k * team < whole; }
    __device__ __forceinline__ bool is_cut(int k) const { return rest != 0 && k * team == whole; }
};
// piece k of a row, 0 behind its end
template <typename T, int VEC>
__device__ __forceinline__ void get(float (&v)[VEC], const T *row, int k, const Columns &c)
{
    const T *at = row + (k * c.team + c.t) * VEC;
    if (c.is_whole(k)) {
        unpack<T, VEC>(v, at);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = 0.0f;
        if (VEC > 1 && c.is_cut(k)) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i < c.rest) v[i] = to_float(at[i]);
        }
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void get_either(float (&v)[VEC], const void *row, bool f32, int k, const Columns &c)
{
    if (sizeof(T) == 2 && f32) {
        const float *p = static_cast<const float *>(row) + (k * c.team + c.t) * VEC;
        if (VEC % 4 == 0 && c.is_whole(k)) {
            if constexpr (VEC % 4 == 0) {
#pragma unroll
                for (int i = 0; i < VEC; i += 4) {
                    const float4 w = *reinterpret_cast<const float4 *>(p + i);
                    v[i] = w.x, v[i + 1] = w.y, v[i + 2] = w.z, v[i + 3] = w.w;
                }
            }
            return;
        }
        const int n = c.is_whole(k) ? VEC : c.is_cut(k) ? c.rest : 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = i < n ? p[i] : 0.0f;
    } else {
        get<T, VEC>(v, static_cast<const T *>(row), k, c);
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void put(T *row, const float (&v)[VEC], int k, const Columns &c)
{
    T *at = row + (k * c.team + c.t) * VEC;
    if (c.is_whole(k)) {
        if constexpr (VEC == kPer16<T>) {
            *reinterpret_cast<uint4 *>(at) = pack16(v, T());
        } else if constexpr (VEC == 2 && sizeof(T) == 2) {
            const T lo = from_float<T>(v[0]), hi = from_float<T>(v[1]);
            *reinterpret_cast<unsigned int *>(at) =
                *reinterpret_cast<const unsigned short *>(&lo) | (unsigned int)*reinterpret_cast<const unsigned short *>(&hi) << 16;
        } else {
            at[0] = from_float<T>(v[0]);
        }
    } else if (VEC > 1 && c.is_cut(k)) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < c.rest) at[i] = from_float<T>(v[i]);
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void put_either(void *row, bool f32, const float (&v)[VEC], int k, const Columns &c)
{
    if (sizeof(T) == 2 && f32) {
        const int n = c.is_whole(k) ? VEC : c.is_cut(k) ? c.rest : 0;
        float *at = static_cast<float *>(row) + (k * c.team + c.t) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < n) at[i] = v[i];
    } else {
        put<T, VEC>(static_cast<T *>(row), v, k, c);
    }
}

// Sum over the threads of a row: `team` lanes of a warp, or (BLOCK) the block, of 16 warps (WIDE: 32) at most. One barrier a sum: the
// next one uses the other half.
template <bool BLOCK, bool WIDE>
__device__ __forceinline__ float row_sum(float v, int team, float4 (*warps)[8], int &half)
{
    if (!BLOCK) return lanes_sum(v, team);
    v = lanes_sum(v, 32);
    const int n = blockDim.x / 32;
    if (threadIdx.x % 32 == 0) reinterpret_cast<float *>(warps[half])[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < (WIDE ? 8 : 4); ++w) {   // (what lies behind the last warp is 0)
        if (4 * w >= n) break;
        const float4 f = warps[half][w];
        v += (f.x + f.y) + (f.z + f.w);
    }
    half ^= 1;
    return v;
}

// Rows to come, copied ahead into shared memory: each thread copies the pieces that it will read itself, so no barrier is needed, and
// reads them again in each pass over the row rather than keep them. (Loads into registers: 8 x 8,192 x 2,048 bf16 forward
// 316 us, backward 651; staged, with 8 values a thread, 256 and 511; with 16 values, 217 and 545, and then as below.) Single values of 16 bits cannot be
// copied like that: they are loaded and put there. Rows beyond 8,192 values do not fit: they come from memory and then from the L1 cache.
template <typename T, int VEC, int CH, bool WIDE>
struct Ahead {
    static constexpr int kPiece = VEC * (int)sizeof(T);
    static constexpr bool kStaged = !WIDE;
    static constexpr int kRowBytes = kStaged ? CH * kPiece : 0;   // a thread's, per table

    // Two rows where a thread's pieces are 16 bytes and there is room for two blocks, else one: more rows take shared memory from more
    // blocks (8 x 8,192 x 2,048 bf16 backward one row ahead 321 us, two 312, three 339; 4,099 x 2,050 f16 112, 116, 147).
    static int rows(int tables, int threads) { return kPiece == 16 && 2 * tables * kRowBytes * threads <= 100 * 1024 ? 2 : 1; }
    static __device__ __forceinline__ void wait(int rows)
    {
        if (!kStaged) return;
        if (rows == 2)
            copies_wait<1>();
        else
            copies_wait<0>();
    }
    static __device__ __forceinline__ int slot(int table, int k)   // table: of all rows' tables
    {
        return ((table * CH + k) * (int)blockDim.x + (int)threadIdx.x) * kPiece;
    }
    // what lies behind a row's end stays 0 in all of them
    static __device__ __forceinline__ void clear(char *shared, int tables)
    {
        if constexpr (kStaged) {
            for (int n = 0; n < tables * CH; ++n) {
                char *at = shared + (n * (int)blockDim.x + (int)threadIdx.x) * kPiece;
                if constexpr (kPiece == 16)
                    *reinterpret_cast<uint4 *>(at) = make_uint4(0, 0, 0, 0);
                else if constexpr (kPiece == 4)
                    *reinterpret_cast<unsigned int *>(at) = 0u;
                else
                    *reinterpret_cast<unsigned short *>(at) = 0;
            }
        }
    }
    // two tables' rows at a time (either may be NULL)
    static __device__ __forceinline__ void copy(char *shared, int table, const T *row, const T *row2, const Columns &c)
    {
        if constexpr (kStaged && kPiece == 2) {   // single values: loaded, all under way together, and put there
            unsigned short v[2][CH];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const T *from = (n == 0 ? row : row2);
#pragma unroll
                for (int k = 0; k < CH; ++k) v[n][k] = from && c.is_whole(k) ? reinterpret_cast<const unsigned short *>(from)[k * c.team + c.t] : (unsigned short)0;
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int k = 0; k < CH; ++k) *reinterpret_cast<unsigned short *>(shared + slot(table + n, k)) = v[n][k];
        } else {
            if (row) copy_one(shared, table, row, c);
            if (row2) copy_one(shared, table + 1, row2, c);
        }
    }
    static __device__ __forceinline__ void copy_one(char *shared, int table, const T *row, const Columns &c)
    {
        if constexpr (kStaged && kPiece >= 4) {
            const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(shared + slot(table, 0)));
            const T *from = row + c.t * VEC;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const uint32_t at = to + k * (int)blockDim.x * kPiece;
                if (c.is_whole(k)) {
                    if constexpr (kPiece == 16)
                        copy_async16(at, from + k * c.team * VEC);
                    else
                        copy_async4(at, from + k * c.team * VEC);
                } else if (VEC > 1 && c.is_cut(k)) {
                    const int bytes = c.rest * (int)sizeof(T);
                    if constexpr (kPiece == 16)
                        copy_async16(at, from + k * c.team * VEC, bytes);
                    else
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at), "l"(from + k * c.team * VEC), "r"(bytes) : "memory");
                }
            }
        }
    }
    static __device__ __forceinline__ void read(float (&v)[VEC], const char *shared, int table, int k, const T *row, const Columns &c)
    {
        if constexpr (kStaged)
            unpack<T, VEC>(v, shared + slot(table, k));
        else
            get<T, VEC>(v, row, k, c);
    }
};

// v *= w;  v *= f (above);  s += a b, two sums side by side
template <int VEC>
__device__ __forceinline__ void mul_all(float (&v)[VEC], const float (&w)[VEC])
{
    if constexpr (VEC == 1) {
        v[0] *= w[0];
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) mul2(v[i], v[i + 1], w[i], w[i + 1]);
    }
}
template <int VEC>
__device__ __forceinline__ void dot_all(float (&s)[2], const float (&a)[VEC], const float (&b)[VEC])
{
    if constexpr (VEC == 1) {
        s[0] = fmaf(a[0], b[0], s[0]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) fma2(s[0], s[1], a[i], a[i + 1], b[i], b[i + 1]);
    }
}
template <int VEC>
__device__ __forceinline__ void add_product(float (&s)[VEC], const float (&a)[VEC], const float (&b)[VEC])   // s += a b
{
    if constexpr (VEC == 1) {
        s[0] = fmaf(a[0], b[0], s[0]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) fma2(s[i], s[i + 1], a[i], a[i + 1], b[i], b[i + 1]);
    }
}
template <int VEC>
__device__ __forceinline__ void add_scaled(float (&s)[VEC], const float (&a)[VEC], float f)   // s += a f
{
    if constexpr (VEC == 1) {
        s[0] = fmaf(a[0], f, s[0]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) fma2(s[i], s[i + 1], a[i], a[i + 1], f, f);
    }
}


enum Gate { NO_GATE, SHARED_GATE, ROW_GATE };

// Registers: what leaves room for enough threads to keep the memory busy. Weights are not among them: they lie in shared memory as
// 32-bit floats, those of the branch's norm multiplied by the gate that the block's rows share. (Taken from the L1 cache row by row:
// 8 x 8,192 x 2,048 bf16 forward 191 us, backward 414; this 188 and 312.)
template <bool WIDE> constexpr int kForwardRegs = 64;
template <bool WIDE> constexpr int kBackwardRegs = WIDE ? 64 : 112;

// The rows of a block: part of one gate's, or whole gates (without a shared gate all rows are one gate's).
struct Rows {
    unsigned int per_gate, gate_from, gate_to, part_from, part_to;
    __device__ __forceinline__ Rows(const BlockArgs &a, bool shared_gate)
    {
        per_gate = (unsigned int)(shared_gate ? a.rows_per_gate : a.rows), part_from = 0, part_to = per_gate;
        if (a.blocks_per_gate > 1) {
            gate_from = blockIdx.x / a.blocks_per_gate, gate_to = gate_from + 1;
            const unsigned int part = blockIdx.x % a.blocks_per_gate;
            part_from = (unsigned int)((long long)per_gate * part / a.blocks_per_gate);
            part_to = (unsigned int)((long long)per_gate * (part + 1) / a.blocks_per_gate);
        } else {
            const long long gates = (unsigned int)a.rows / per_gate;
            gate_from = (unsigned int)(gates * blockIdx.x / gridDim.x), gate_to = (unsigned int)(gates * (blockIdx.x + 1) / gridDim.x);
        }
    }
};
// Blocks that share a gate's rows: as many as fill the GPU, each with rows for all its teams. Without a shared gate there is one gate.
struct Split {
    int share;
    long long blocks;
};
inline Split split_rows(long long rows, long long per_gate, bool shared_gate, int teams, long long fit)
{
    if (!shared_gate) per_gate = rows;
    const long long gates = rows / per_gate, most = (per_gate + teams - 1) / teams;
    long long share = (fit + gates - 1) / gates;
    if (gates > 1 && gates * share > fit && share > 1) --share;
    if (share > most) share = most;
    return {(int)share, share > 1 ? gates * share : gates < fit ? gates : fit};
}

// v = the gate of gate row / row `at`
template <typename T>
__device__ __forceinline__ const void *gate_at(const BlockArgs &a, long long at)
{
    return static_cast<const char *>(a.gate) + at * a.gate_stride * (a.gate_f32 ? 4 : (int)sizeof(T));
}
// Weights as the thread that reads them finds them without bank conflicts: its pieces of four (or fewer) lie `team` pieces apart.
template <int VEC>
__device__ __forceinline__ int weight_slot(int k, int i, int team, int t)
{
    constexpr int P = VEC < 4 ? VEC : 4;
    return ((k * (VEC / P) + i / P) * team + t) * P + i % P;
}
// weight * gate (1 where there is none) of the thread's columns
template <typename T, int VEC, int CH>
__device__ __forceinline__ void fill_weights(float *to, const void *weight, bool f32, const void *gate, bool gate_f32, int team, int t, int width)
{
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int col = (k * team + t) * VEC + i;
            float w = weight && col < width ? one_value(weight, col, f32, T()) : 1.0f;
            if (gate && col < width) w *= one_value(gate, col, gate_f32, T());
            to[weight_slot<VEC>(k, i, team, t)] = w;
        }
}
template <int VEC>
__device__ __forceinline__ void weights(float (&v)[VEC], const float *from, int k, int team, int t)
{
    if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            const float4 w = *reinterpret_cast<const float4 *>(from + weight_slot<VEC>(k, i, team, t));
            v[i] = w.x, v[i + 1] = w.y, v[i + 2] = w.z, v[i + 3] = w.w;
        }
    } else if constexpr (VEC == 2) {
        const float2 w = *reinterpret_cast<const float2 *>(from + weight_slot<VEC>(k, 0, team, t));
        v[0] = w.x, v[1] = w.y;
    } else {
        v[0] = from[weight_slot<VEC>(k, 0, team, t)];
    }
}

// How a row is spread: VEC neighbours at a time as the alignment of all tables allows; 8 values a thread up to 256 (32 lanes), 16 beyond
// (what a thread does besides its values weighs half as much); up to 512 values a warp's lanes, or fewer, have a row. Beyond
// 8,192 values that means 1,024 threads, whose 64 registers each do not hold all that a row needs.
struct Shape {
    int vec, chunks, team;
    bool block, wide;
    int threads;
};
inline Shape plan(int width, int elem, int align)
{
    Shape s;
    s.vec = align >= 16 ? 16 / elem : align >= 4 && elem == 2 ? 2 : 1;
    const int values = width > 256 ? 16 : 8;
    s.chunks = values / s.vec;
    const int need = (width + values - 1) / values;
    s.block = need > 32, s.wide = need > 512;
    s.team = 1;
    if (s.block)
        s.team = (need + 31) / 32 * 32;
    else
        while (s.team < need) s.team *= 2;
    s.threads = s.block ? s.team : kTeams;
    return s;
}
inline int table_align(const void *p, int64_t rows, int64_t stride, int elem)
{
    if (!p) return 16;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (rows > 1 ? (uintptr_t)(stride * elem) : 0);
    return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

template <typename T, typename F>
cudaError_t by_shape(const Shape &s, F launch)
{
    constexpr int V = kPer16<T>;
#define NBOS_SHAPE(VEC, CH, BLOCK, WIDE) \
    if (s.vec == VEC && s.chunks == CH && s.block == BLOCK && s.wide == WIDE) \
        return launch(std::integral_constant<int, VEC>(), std::integral_constant<int, CH>(), std::integral_constant<bool, BLOCK>(), std::integral_constant<bool, WIDE>());
#define NBOS_SHAPES(VEC) NBOS_SHAPE(VEC, 8 / VEC, false, false) NBOS_SHAPE(VEC, 16 / VEC, false, false) \
    NBOS_SHAPE(VEC, 16 / VEC, true, false) NBOS_SHAPE(VEC, 16 / VEC, true, true)
    NBOS_SHAPES(V)
    NBOS_SHAPES(1)
    if constexpr (sizeof(T) == 2) { NBOS_SHAPES(2) }
#undef NBOS_SHAPES
#undef NBOS_SHAPE
    return cudaErrorInvalidConfiguration;
}


// The backward launches (nbos_policy_block_norm_backward.cu); c: which sums over rows are wanted
struct ColumnArgs {
    const float *partial;
    int blocks, blocks_per_gate, width;
    const void *gate, *post;
    long long gate_stride;
    bool gate_f32, weight_f32, weigh;   // weigh: the blocks' S have yet to be multiplied by their gate
    void *dpost, *dpre, *dgate;
    long long dgate_stride;
};
cudaError_t launch_backward(int dtype, const BlockArgs &a, const Shape &s, int sms, ColumnArgs &c, cudaMemPool_t pool, cudaStream_t stream);

}  // namespace block_norm
}  // namespace nbos
#endif
