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

// The columns of a thread: pieces of 16 bytes' worth of values (VEC), `team` of them apart. Piece k is whole, or the row's last and cut off,
// or behind it. `mine`: which of the block's teams the thread is in.
struct Columns {
    int team, t, width, whole, rest, mine, teams;
    __device__ __forceinline__ Columns(int team_, int t_, int width_, int vec, int mine_, int teams_)
        : team(team_), t(t_), width(width_), whole(width_ / vec - t_), rest(width_ % vec), mine(mine_), teams(teams_)
    {
    }
    __device__ __forceinline__ bool is_whole(int k) const { return k * team < whole; }
    __device__ __forceinline__ bool is_cut(int k) const { return rest != 0 && k * team == whole; }
};
// Piece k of a row, 0 behind its end. ANY: the row may start anywhere, else on a 16-byte boundary.
template <typename T, int VEC, bool ANY>
__device__ __forceinline__ void get(float (&v)[VEC], const T *row, int k, const Columns &c)
{
    const T *at = row + (k * c.team + c.t) * VEC;
    if (!ANY && c.is_whole(k)) {
        unpack16(*reinterpret_cast<const uint4 *>(at), v, T());
    } else {
        const int n = c.is_whole(k) ? VEC : c.is_cut(k) ? c.rest : 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = i < n ? to_float(at[i]) : 0.0f;
    }
}
template <typename T, int VEC, bool ANY>
__device__ __forceinline__ void get_either(float (&v)[VEC], const void *row, bool f32, int k, const Columns &c)
{
    if (sizeof(T) == 2 && f32) {
        const float *p = static_cast<const float *>(row) + (k * c.team + c.t) * VEC;
        if (!ANY && c.is_whole(k)) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const float4 w = *reinterpret_cast<const float4 *>(p + i);
                v[i] = w.x, v[i + 1] = w.y, v[i + 2] = w.z, v[i + 3] = w.w;
            }
        } else {
            const int n = c.is_whole(k) ? VEC : c.is_cut(k) ? c.rest : 0;
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = i < n ? p[i] : 0.0f;
        }
    } else {
        get<T, VEC, ANY>(v, static_cast<const T *>(row), k, c);
    }
}
template <typename T, int VEC, bool ANY>
__device__ __forceinline__ void put(T *row, const float (&v)[VEC], int k, const Columns &c)
{
    T *at = row + (k * c.team + c.t) * VEC;
    if (!ANY && c.is_whole(k)) {
        *reinterpret_cast<uint4 *>(at) = pack16(v, T());
    } else {
        const int n = c.is_whole(k) ? VEC : c.is_cut(k) ? c.rest : 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < n) at[i] = from_float<T>(v[i]);
    }
}
template <typename T, int VEC, bool ANY>
__device__ __forceinline__ void put_either(void *row, bool f32, const float (&v)[VEC], int k, const Columns &c)
{
    if (sizeof(T) == 2 && f32) {
        const int n = c.is_whole(k) ? VEC : c.is_cut(k) ? c.rest : 0;
        float *at = static_cast<float *>(row) + (k * c.team + c.t) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < n) at[i] = v[i];
    } else {
        put<T, VEC, ANY>(static_cast<T *>(row), v, k, c);
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

template <bool BLOCK>
__device__ __forceinline__ void team_sync()
{
    if (BLOCK)
        __syncthreads();
    else
        __syncwarp();
}

// Rows to come, copied ahead into shared memory and read there again in each pass rather than kept. (Loads into registers, 8 x
// 8,192 x 2,048 bf16: forward 316 us, backward 651; staged, with 8 values a thread, 256 and 511; with 16 values, 217 and 545, and then as
// below.) Rows on 16-byte boundaries: each thread copies the pieces that it reads itself, so no barrier is needed. ANY, rows that start
// anywhere: a team copies the row with the bytes from the boundary before it, a thread puts its pieces together from two neighbours of 16 bytes,
// and results go the same way back (single values from and to memory instead: 32,768 x 2,051 f16 without a gate, forward 373 us, backward
// 1,018; this 202 and 550). Rows that do not fit (beyond 8,192 values, or nearly that many of 32 bits) come from memory and then from the L1
// cache.
template <typename T, int VEC, int CH, bool BLOCK, bool WIDE, bool ANY>
struct Ahead {
    static constexpr bool kStaged = !WIDE;

    static __host__ __device__ __forceinline__ int region(int team) { return (CH * team + (ANY ? 2 : 0)) * 16; }   // bytes of a row
    static __host__ __device__ __forceinline__ int bytes(int rows, int tables, int team, int teams)
    {
        return kStaged ? rows * tables * teams * region(team) : 0;
    }
    // Two rows where there is room for two blocks, else one: more rows take shared memory from more blocks (8 x 8,192 x 2,048 bf16
    // backward one row ahead 321 us, two 312, three 339).
    static int rows(int tables, int team, int teams) { return bytes(2, tables, team, teams) <= 100 * 1024 ? 2 : 1; }

    static __device__ __forceinline__ char *row_at(char *shared, int table, const Columns &c)   // table: of all rows' tables
    {
        return shared + (table * c.teams + c.mine) * region(c.team);
    }
    // what lies behind a row's end stays 0 in all of them
    static __device__ __forceinline__ void clear(char *shared, int bytes)
    {
        if constexpr (kStaged) {
            for (int i = threadIdx.x; i < bytes / 16; i += blockDim.x) reinterpret_cast<uint4 *>(shared)[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
        }
    }
    // offset: of the row in its table
    static __device__ __forceinline__ void copy(char *shared, int table, const T *row, long long offset, const Columns &c)
    {
        if constexpr (kStaged && ANY) {
            stage_row(row_at(shared, table, c), row, c.width, offset * (long long)sizeof(T), c.t, c.team);
        } else if constexpr (kStaged) {
            const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(row_at(shared, table, c))) + c.t * 16;
            const T *from = row + c.t * VEC;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (c.is_whole(k))
                    copy_async16(to + k * c.team * 16, from + k * c.team * VEC);
                else if (c.is_cut(k))
                    copy_async16(to + k * c.team * 16, from + k * c.team * VEC, c.rest * (int)sizeof(T));
            }
        }
    }
    static __device__ __forceinline__ void read(float (&v)[VEC], char *shared, int table, int k, const T *row, const Columns &c)
    {
        if constexpr (!kStaged) {
            get<T, VEC, ANY>(v, row, k, c);
        } else {
            const uint4 *at = reinterpret_cast<const uint4 *>(row_at(shared, table, c)) + k * c.team + c.t;
            if constexpr (!ANY) {
                unpack16(*at, v, T());
            } else {
                if (c.is_whole(k) || c.is_cut(k)) {
                    const int shift = row_shift(row);
                    uint4 piece = *at;
                    if (shift) piece = window16(piece, at[1], shift);
                    unpack16(piece, v, T());
                }
                if (!c.is_whole(k)) {
                    const int n = c.is_cut(k) ? c.rest : 0;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] = i < n ? v[i] : 0.0f;
                }
            }
        }
    }
    // A result's piece: to memory at once, or (ANY) to shared memory, in place of a table that has been read, and from there by row_out.
    static __device__ __forceinline__ void write(T *row, char *shared, int table, const float (&v)[VEC], int k, const Columns &c)
    {
        if constexpr (kStaged && ANY) {
            if (c.is_whole(k) || c.is_cut(k)) reinterpret_cast<uint4 *>(row_at(shared, table, c))[k * c.team + c.t] = pack16(v, T());
        } else {
            put<T, VEC, ANY>(row, v, k, c);
        }
    }
    static __device__ __forceinline__ void row_out(T *row, char *shared, int table, const Columns &c)
    {
        if constexpr (kStaged && ANY) {
            const char *from = row_at(shared, table, c);
            const int shift = row_shift(row), total = shift + c.width * (int)sizeof(T);
            char *to = reinterpret_cast<char *>(row) - shift;
            for (int g = c.t; g * 16 < total; g += c.team) {
                if (g * 16 >= shift && g * 16 + 16 <= total) {
                    const uint4 *at = reinterpret_cast<const uint4 *>(from) + g;
                    uint4 piece = *at;
                    if (shift) piece = window16(at[-1], piece, 16 - shift);
                    *reinterpret_cast<uint4 *>(to + g * 16) = piece;
                } else {
                    for (int i = g * 16; i < g * 16 + 16; i += (int)sizeof(T))
                        if (i >= shift && i < total) *reinterpret_cast<T *>(to + i) = *reinterpret_cast<const T *>(from + i - shift);
                }
            }
        }
    }
};

// v *= w;  v *= f (above);  s += a b, two sums side by side
template <int VEC>
__device__ __forceinline__ void mul_all(float (&v)[VEC], const float (&w)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC; i += 2) mul2(v[i], v[i + 1], w[i], w[i + 1]);
}
template <int VEC>
__device__ __forceinline__ void dot_all(float (&s)[2], const float (&a)[VEC], const float (&b)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC; i += 2) fma2(s[0], s[1], a[i], a[i + 1], b[i], b[i + 1]);
}
template <int VEC>
__device__ __forceinline__ void add_product(float (&s)[VEC], const float (&a)[VEC], const float (&b)[VEC])   // s += a b
{
#pragma unroll
    for (int i = 0; i < VEC; i += 2) fma2(s[i], s[i + 1], a[i], a[i + 1], b[i], b[i + 1]);
}
template <int VEC>
__device__ __forceinline__ void add_scaled(float (&s)[VEC], const float (&a)[VEC], float f)   // s += a f
{
#pragma unroll
    for (int i = 0; i < VEC; i += 2) fma2(s[i], s[i + 1], a[i], a[i + 1], f, f);
}


enum Gate { NO_GATE, SHARED_GATE, ROW_GATE };

// Registers: what leaves room for enough threads to keep the memory busy (backward with 96: 280 -> 320 us for 32,768 x 2,048 f16, a gate for each of
// eight groups). Some backward forms do not fit: rows of 257 to 512 values spill 100 to 820 bytes a thread at 112 (4 groups, 512 bf16, 134 million values: 346 us, 71 % of the
// tables' bytes; a gate a row 538, 61 %), rows beyond 8,192 values 250 to 890 at 64 (12,288 bf16: 732 us, 34 %). Weights are not among them: they lie in shared memory as
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
// Weights as the thread that reads them finds them without bank conflicts: its pieces of four lie `team` pieces apart.
template <int VEC>
__device__ __forceinline__ int weight_slot(int k, int i, int team, int t)
{
    return ((k * (VEC / 4) + i / 4) * team + t) * 4 + i % 4;
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
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
        const float4 w = *reinterpret_cast<const float4 *>(from + weight_slot<VEC>(k, i, team, t));
        v[i] = w.x, v[i + 1] = w.y, v[i + 2] = w.z, v[i + 3] = w.w;
    }
}

// How a row is spread: pieces of 16 bytes; 8 values a thread up to 256 (32 lanes), 16 beyond (what a thread does besides its values weighs
// half as much); up to 512 values a warp's lanes, or fewer, have a row. Beyond 8,192 values that means 1,024 threads, whose 64
// registers each do not hold all that a row needs.
struct Shape {
    int chunks, team;
    bool block, wide, any;   // any: some table's rows do not start on 16-byte boundaries
    int threads;
};
inline Shape plan(int width, int elem, bool any)
{
    Shape s;
    s.any = any;
    const int values = width > 256 ? 16 : 8;
    s.chunks = values * elem / 16;
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
// whether some row of a table starts off 16-byte boundaries
inline bool rows_anywhere(const void *p, int64_t rows, int64_t stride, int elem)
{
    return p && ((reinterpret_cast<uintptr_t>(p) | (rows > 1 ? (uintptr_t)(stride * elem) : 0)) & 15) != 0;
}

template <typename T, typename F>
cudaError_t by_shape(const Shape &s, F launch)
{
    constexpr int V = kPer16<T>;
#define NBOS_SHAPE(CH, BLOCK, WIDE, ANY)                                                                                            \
    if (s.chunks == CH && s.block == BLOCK && s.wide == WIDE && s.any == ANY)                                                       \
        return launch(std::integral_constant<int, CH>(), std::integral_constant<bool, BLOCK>(), std::integral_constant<bool, WIDE>(), \
                      std::integral_constant<bool, ANY>());
#define NBOS_SHAPES(ANY) \
    NBOS_SHAPE(8 / V, false, false, ANY) NBOS_SHAPE(16 / V, false, false, ANY) NBOS_SHAPE(16 / V, true, false, ANY) NBOS_SHAPE(16 / V, true, true, ANY)
    NBOS_SHAPES(false)
    NBOS_SHAPES(true)
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
