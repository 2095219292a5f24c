// Distillation of a two-tower policy without its table of logits (nbos_policy_towers, nbos_policy_towers_backward).
//
// With a the requests' vectors, b the hosts', c = log2(e) / T, and x_rh = a_r . b_h where the request fits the host, else -inf:
//   forward   m_r = max_h x_rh,  S_r = sum_h 2^((x_rh - m_r) c)      a matrix product whose tiles never leave the chip
//             y_rj = x at the row's hosts, taken from the same tiles,  loss_r = T^2 sum_j q_j (ln q_j - (y_rj - m_r) / T + ln S_r)
//   backward  G_rh = g_r T (p_rh - q_rh), p_rh = 2^((x_rh - m_r) c) / S_r    the product once more
//             da = G b,  db = G^T a                                           two more products
// G exists in pieces (groups, or runs of a group's longer side), its entries as two values of the operands' type: about kPieceBytes of it.
#include <math.h>

#include <atomic>

#include "nbos_policy.cuh"
#include "nbos_probe.h"
#include "nbos_tensor.cuh"

namespace nbos {
namespace {

using namespace policy;
using namespace tensor;

constexpr int kTileM = 256;           // rows of a pair's tile; each of its two blocks has 128 of them
constexpr int kTileN = 256;           // columns; narrower tiles of 128 for gradients of at most 128 columns
constexpr int kBlockK = 64;           // values of the contraction per stage: one 128-byte row
constexpr int kParts = 4;             // a tile's columns are read in this many parts, each by four warps (32 rows a warp)
constexpr int kEpilogue = 128 * kParts;
constexpr int kThreads = kEpilogue + 64;   // and a warp that copies, a warp that multiplies
constexpr int kTmemColumns = 512;     // two tiles of 32-bit products
constexpr int kBand = 16;             // tiles of hosts that G's rows go through together
constexpr int kFewEntries = 4;        // a row's entries that are put into G on its way out; more of them by a kernel of their own
constexpr size_t kPieceBytes = 512u << 20;   // 65,536 x 4,096 at width 256, gradients: 48 MB 950 us, 128 MB 650, 256 MB 586, 512 MB 567 (one value an entry): launches fill the GPU

enum Kind { STATS, GRAD, GRAD_REQUESTS, GRAD_HOSTS };

struct Tiles {                        // what one launch covers
    int groups, m_tiles, n_tiles, k_blocks;
    int splits, split_blocks;         // the contraction in parts, whose sums are added up afterwards
    long long units;                  // groups * m_tiles * n_tiles * splits
};
// G is held in 16 bits, so all of it is multiplied by one factor, and what comes of it divided by it again: the largest |g_r T| becomes
// `top`, the value of both types just below a power of two. A row's largest entries, p - q near -1, then lose least (values just above
// a power of two lose twice the share), those of a p near 0 nothing; and 16-bit floats use their whole range: p of 2^-29 is still a
// normal number.
struct Range {
    const unsigned int *largest;      // bits of the largest finite |grad_loss| of a row that counts; NULL: 1
    float scale, top;                 // grad_scale T; 1 - 2^-8, in 16-bit floats times 2^15
    __device__ __forceinline__ float factor() const
    {
        const float g = (largest ? __uint_as_float(*largest) : 1.0f) * fabsf(scale);
        return g > 0.0f && g < __int_as_float(0x7F800000) ? fminf(top / g, 0x1p100f) : 1.0f;
    }
};
struct TowerArgs {
    Tiles t;
    int a_z0, a_z, b_z0, b_z;         // group g is slice z0 + g * z of the operand
    int a_m0, b_n0, b_k0;             // first row of the operand
    int k_shift, plane_z;             // gradients: 1 if G has two planes, which take turns in the contraction (what both are multiplied with
                                      // is then read from memory once), and the slices from one to the next
    int group0, row0, rows, hosts, width;   // rows: of a group
    int col0, col_end;                // scores: the launch's first host, and how many it has
    const int4 *asks, *room;
    float c;                          // log2(e) / T
    float2 *partial;                  // STATS: [groups][rows][slots] (m, S) of parts of a row
    int slots;
    const unsigned int *keys;         // STATS: [groups][rows][k], each 32 rows' entries in the order of their tiles (NULL: at most kFewEntries a row)
    const int *key_starts;            // of each 32 rows' list, five
    float *entries;                   // STATS: x at a row's entries, rows entry_stride apart
    int entry_stride;
    const float *stats;               // GRAD: [groups][rows][stats_stride]: m, S, ...
    int stats_stride;
    const int32_t *ids;               // the rows' entries, k of them (GRAD: NULL: too many)
    const float *teacher;
    long long teacher_stride;
    int k;
    const float *grad_loss;
    Range range;
    void *out;                        // gradients: the result itself (one part), or
    float *sums;                      // [splits][groups][m_rows][width to a multiple of 4] of 32-bit sums, added to those there if `add`
    long long out_stride, out_group_stride;
    bool out_wide;                    // rows of the result lie on 16-byte boundaries
    int m_rows, out_row0, add;        // m_rows: rows that the launch writes, per group
    unsigned long long limit_ns;      // of a wait
    bool stall;                       // self-test: nothing is copied, so that the waits run out
};

__device__ unsigned int tower_status;   // STATUS_WAIT_TIMEOUT once a wait ran out, until nbos_policy_towers_status is asked

// Scores: pair p of `pairs` takes units [first_unit(p), first_unit(p + 1)), hosts innermost: a pair stays with its rows as long
// as it can, and all pairs have equally much to do.
__device__ __host__ __forceinline__ long long first_unit(long long units, int pairs, int p)
{
    const long long q = units / pairs, r = units % pairs;
    return p * q + (p < r ? p : r);
}
__device__ __host__ __forceinline__ int pair_of(long long units, int pairs, long long unit)
{
    const long long q = units / pairs, r = units % pairs;
    return (int)(unit < r * (q + 1) ? unit / (q + 1) : r + (unit - r * (q + 1)) / q);
}

struct Unit {
    int g, m, n, split, k0, k1;       // k0 .. k1: blocks of the contraction
};
// Every thread that has a part in a unit goes through the same schedule, so its steps are 32-bit ones: scores count on from where the
// pair starts, the others (fewer than 2^31 units) divide.
template <Kind KIND>
struct Schedule {
    unsigned int left, at, step;
    int n, m, g, band, band_end;   // scores: the next unit's, and which columns its band has
    __device__ __forceinline__ Schedule(const Tiles &t, int pair, int pairs)
    {
        if (KIND == STATS || KIND == GRAD) {
            const long long from = first_unit(t.units, pairs, pair), per_group = (long long)t.m_tiles * t.n_tiles;
            left = (unsigned int)(first_unit(t.units, pairs, pair + 1) - from);
            g = (int)(from / per_group);
            // GRAD goes through bands of columns, each for all rows: pairs in flight at one time read the same hosts, and still a pair
            // stays with its rows for a band's width. (STATS would leave a part of each row's statistics for each band.)
            const long long in = from % per_group;
            const int wide = KIND == GRAD ? kBand : t.n_tiles;
            band = (int)(in / ((long long)t.m_tiles * wide)) * wide;
            band_end = min(band + wide, t.n_tiles);
            const long long rest = in - (long long)t.m_tiles * band;
            m = (int)(rest / (band_end - band)), n = band + (int)(rest % (band_end - band));
        } else {
            left = (unsigned int)t.units > (unsigned int)pair ? ((unsigned int)t.units - pair + pairs - 1) / pairs : 0;
            at = pair, step = pairs;
        }
    }
    __device__ __forceinline__ bool next(const Tiles &t, Unit &u)
    {
        if (left == 0) return false;
        --left;
        if (KIND == STATS || KIND == GRAD) {
            u.n = n, u.m = m, u.g = g, u.split = 0;
            if (++n == band_end) {
                n = band;
                if (++m == t.m_tiles) {
                    m = 0;
                    if (band_end == t.n_tiles) ++g, band_end = 0;
                    n = band = band_end;
                    band_end = KIND == GRAD ? min(band + kBand, t.n_tiles) : t.n_tiles;
                }
            }
        } else {
            // bands of 8 tiles along M, so that tiles in flight at one time share both operands
            const unsigned int per_split = (unsigned int)t.m_tiles * t.n_tiles, part = at / per_split, in = at % per_split;
            const unsigned int across = in / (8u * t.n_tiles), high = min(8u, t.m_tiles - 8 * across), rest = in - across * 8 * t.n_tiles;
            u.m = (int)(8 * across + rest % high), u.n = (int)(rest / high);
            u.split = (int)(part % t.splits), u.g = (int)(part / t.splits);
            at += step;
        }
        u.k0 = u.split * t.split_blocks;
        u.k1 = min(t.k_blocks, u.k0 + t.split_blocks);
        return true;
    }
};

template <Kind KIND, int BN>
struct Shape {
    static constexpr bool kAlongKA = KIND != GRAD_HOSTS, kAlongKB = KIND == STATS || KIND == GRAD;
    static constexpr int kBytesA = 128 * kBlockK * 2, kBytesB = BN / 2 * kBlockK * 2, kStageBytes = kBytesA + kBytesB;
    // what is on its way out, a box a warp: G, 32 rows x 64 columns; a gradient, 32 x 32
    static constexpr int kStaging = KIND == GRAD ? 4 * 128 * 128 : KIND == STATS ? 0 : 4 * 128 * 64;
    static constexpr int kRoom = KIND == STATS || KIND == GRAD ? 2 * kTileN * 16 : 0;
    static constexpr int kStages = KIND == GRAD ? 4 : 6;
    static constexpr int kBytes = kStages * kStageBytes + kStaging + kRoom + 256 /* barriers */ + 1024 /* alignment */;
};

__device__ __forceinline__ void bar_sync(int id, int threads)
{
    __syncwarp();   // the barrier counts whole warps
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// d = (a - m) b + c, two at a time. The subtraction comes first: near the row's maximum it is exact or nearly so, and nothing
// overflows at low temperatures.
__device__ __forceinline__ void apart2(float &d0, float &d1, uint32_t a0, uint32_t a1, float minus_m, float b)
{
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %4};\n\tmov.b64 z, {%5, %5};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmul.rn.f32x2 x, x, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d0), "=f"(d1) : "r"(a0), "r"(a1), "f"(minus_m), "f"(b));
}
__device__ __forceinline__ void apart2(float &d0, float &d1, uint32_t a0, uint32_t a1, float minus_m, float b, float c)
{
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %4};\n\tmov.b64 z, {%5, %5};\n\tmov.b64 w, {%6, %6};\n\t"
        "add.rn.f32x2 x, x, y;\n\tfma.rn.f32x2 x, x, z, w;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d0), "=f"(d1) : "r"(a0), "r"(a1), "f"(minus_m), "f"(b), "f"(c));
}
__device__ __forceinline__ bool fits(const int4 &ask, const int4 &room)
{
    return ask.x <= room.x && ask.y <= room.y && ask.z <= room.z && ask.w <= room.w;
}
__device__ __forceinline__ bool never_fits(const int4 &ask) { return (ask.x | ask.y | ask.z | ask.w) < 0; }

// v where the request fits, else -inf: four compares that hand on one predicate (&& became branches: forward of 65,536 x 4,096 hosts at
// width 256 494 us, this 239 then). The integer compares are what bounds the kernels with capacities now.
__device__ __forceinline__ uint32_t if_fits(uint32_t v, const int4 &ask, const int4 &room)
{
    uint32_t out;
    asm("{\n\t.reg .pred p;\n\tsetp.le.s32 p, %1, %5;\n\tsetp.le.and.s32 p, %2, %6, p;\n\tsetp.le.and.s32 p, %3, %7, p;\n\t"
        "setp.le.and.s32 p, %4, %8, p;\n\tselp.b32 %0, %9, 0xFF800000, p;\n\t}"
        : "=r"(out)
        : "r"(ask.x), "r"(ask.y), "r"(ask.z), "r"(ask.w), "r"(room.x), "r"(room.y), "r"(room.z), "r"(room.w), "r"(v));
    return out;
}

// 64 products of one row become logits: -inf behind the last host
__device__ __forceinline__ void cut64(uint32_t (&u)[32], uint32_t (&v)[32], int left)
{
    if (left < 64) {
#pragma unroll
        for (int i = 0; i < 32; ++i) u[i] = i < left ? u[i] : 0xFF800000u, v[i] = 32 + i < left ? v[i] : 0xFF800000u;
    }
}
// With capacities a thread has 8 of 32 columns of four rows (v[0]: rows t / 4 and t / 4 + 8, v[1]: 16 further) rather than 64 of one row: it
// reads a host's room once for four requests. `room`: of column 2 (t % 4).
__device__ __forceinline__ void mask_rows(uint32_t (&v)[2][16], const int4 *room, const int4 (&ask)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int4 has = room[8 * j + e];
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r / 2][4 * j + 2 * (r % 2) + e] = if_fits(v[r / 2][4 * j + 2 * (r % 2) + e], ask[r], has);
        }
}
// running (m, s) of row r of the four over 8 more logits
__device__ __forceinline__ void add8(float &m, float &s, const uint32_t (&v)[2][16], int r, float c)
{
    auto at = [&](int j, int e) { return __uint_as_float(v[r / 2][4 * j + 2 * (r % 2) + e]); };
    float top[2] = {m, m};
#pragma unroll
    for (int j = 0; j < 4; ++j) top[j % 2] = fmaxf(top[j % 2], fmaxf(at(j, 0), at(j, 1)));
    const float to = fmaxf(top[0], top[1]);
    const float base = to == neg_inf() ? 0.0f : to;
    s *= exp2_fast((m - base) * c);
    m = to;
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float e0, e1;
        apart2(e0, e1, __float_as_uint(at(j, 0)), __float_as_uint(at(j, 1)), -base, c);
        add2(sum[0], sum[1], exp2_fast(e0), exp2_fast(e1));
    }
    s += sum[0] + sum[1];
}

// running (m, s) of a row over 64 more logits
__device__ __forceinline__ void add64(float &m, float &s, uint32_t (&u)[32], uint32_t (&v)[32], float c)
{
    float top[4] = {m, m, m, m};
#pragma unroll
    for (int i = 0; i < 32; i += 4)
#pragma unroll
        for (int j = 0; j < 4; ++j) top[j] = fmaxf(top[j], fmaxf(__uint_as_float(u[i + j]), __uint_as_float(v[i + j])));
    const float to = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const float base = to == neg_inf() ? 0.0f : to;
    s *= exp2_fast((m - base) * c);
    m = to;
    float sum[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float e0, e1, f0, f1;
        apart2(e0, e1, u[i], u[i + 1], -base, c);
        apart2(f0, f1, v[i], v[i + 1], -base, c);
        add2(sum[0][0], sum[0][1], exp2_fast(e0), exp2_fast(e1));
        add2(sum[1][0], sum[1][1], exp2_fast(f0), exp2_fast(f1));
    }
    s += (sum[0][0] + sum[0][1]) + (sum[1][0] + sum[1][1]);
}

__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

// The entries of row `at`: their columns of this launch's hosts (-1: none) and G there. Entries that name one host add up, and
// each of them holds the sum.
template <int PLANES, typename T>
__device__ __forceinline__ void row_entries(const TowerArgs &a, long long at, bool inside, int (&column)[kFewEntries], T (&value)[PLANES][kFewEntries])
{
    const float *stats = a.stats + at * a.stats_stride;
    float t[kFewEntries], x[kFewEntries], top = neg_inf(), sum = 0.0f;
    int id[kFewEntries];
#pragma unroll
    for (int j = 0; j < kFewEntries; ++j) {
        const bool there = inside && j < a.k;
        id[j] = there ? a.ids[at * a.k + j] : -1;
        x[j] = there ? stats[2 + j] : neg_inf();
        t[j] = there && x[j] != neg_inf() ? (a.teacher ? a.teacher[at * a.teacher_stride + j] : 0.0f) : neg_inf();
        if (t[j] > top) top = t[j];
    }
#pragma unroll
    for (int j = 0; j < kFewEntries; ++j) {
        t[j] = t[j] > neg_inf() ? exp2_fast((t[j] - top) * a.c) : 0.0f;
        sum += t[j];
    }
    const bool some = sum != 0.0f;
    const float m = some ? stats[0] : 0.0f, minus = some ? -log2f(stats[1]) : 0.0f;
    const float factor = some ? a.range.scale * (a.grad_loss ? a.grad_loss[at] : 1.0f) * a.range.factor() : 0.0f;
#pragma unroll
    for (int j = 0; j < kFewEntries; ++j) {
        float q = 0.0f;
#pragma unroll
        for (int l = 0; l < kFewEntries; ++l) q += id[l] == id[j] ? t[l] : 0.0f;
        const bool put = some && x[j] != neg_inf() && id[j] >= a.col0 && id[j] < a.col0 + a.col_end;
        column[j] = put ? id[j] - a.col0 : -1;
        const float g = (exp2_fast(fmaf(x[j] - m, a.c, minus)) - q / sum) * factor;
        value[0][j] = from_float<T>(g);
        if (PLANES == 2) value[PLANES - 1][j] = from_float<T>(g - to_float(value[0][j]));
    }
}

// STATS: a row's entries are picked from the tiles as these pass, so that their x are the very values that m and S are made of. (Products of
// their own, summed in another order, are off by some 1e-5: below T of that size p was 0 or infinite at a row's best host.) A warp sees
// 32 rows, and one of a tile's four quarters, in ascending tiles.
constexpr unsigned int kNoEntry = 0xFFFFFFFFu;
// Up to kFewEntries a row (65,536 x 4,096, one entry: 94 us, sorted 99; four 102 / 107): a lane has its row's own, in order, as host << 8 | place in the row's list; at[0] is the next one.
struct RowEntries {
    unsigned int at[kFewEntries];
    float *x;
    __device__ __forceinline__ void start(const TowerArgs &a, long long row, bool inside, int quarter, int tile)
    {
        x = a.entries + row * a.entry_stride;
#pragma unroll
        for (int j = 0; j < kFewEntries; ++j) {
            const int id = inside && j < a.k ? a.ids[row * a.k + j] : -1;
            at[j] = id >= tile * kTileN && id < a.hosts && id / 64 % 4 == quarter ? (unsigned int)id << 8 | (unsigned int)j : kNoEntry;
        }
        auto order = [&](int i, int j) {
            const unsigned int low = min(at[i], at[j]), high = max(at[i], at[j]);
            at[i] = low, at[j] = high;
        };
        order(0, 1), order(2, 3), order(0, 2), order(1, 3), order(1, 2);
    }
    // those in the 64 columns from n0 on, whose products lie at `from` in tensor memory: one load a column, whichever rows have an entry there
    __device__ __forceinline__ void pick(int n0, uint32_t from)
    {
        const unsigned int first = (unsigned int)n0 << 8;
        for (;;) {
            const unsigned int column = __reduce_min_sync(kFull, at[0] - first) >> 8;
            if (column >= 64u) break;
            uint32_t v;
            tmem_load1(v, from + column);
            tmem_wait(v);
            while ((at[0] - first) >> 8 == column) {   // (a host may be listed twice)
                x[at[0] & 255u] = __uint_as_float(v);
#pragma unroll
                for (int j = 0; j + 1 < kFewEntries; ++j) at[j] = at[j + 1];
                at[kFewEntries - 1] = kNoEntry;
            }
            __syncwarp();
        }
    }
};
// More of them: the 32 rows' entries come sorted by quarter and tile (sort_entries_kernel); a lane has one of the next 32.
struct SortedEntries {
    const unsigned int *list;
    float *x;
    int at, end, stride;
    unsigned int key;                 // tile << 19 | column of the quarter << 13 | row << 8 | place in the row's list
    __device__ __forceinline__ void fetch()
    {
        key = at + (int)(threadIdx.x % 32) < end ? list[at + threadIdx.x % 32] : kNoEntry;
        __syncwarp();   // what follows reads tensor memory, which the warp does as one
    }
    __device__ __forceinline__ void start(const TowerArgs &a, int group, int row, int quarter, int tile)
    {
        at = end = 0;
        if (row < a.rows) {
            const int *const starts = a.key_starts + 5 * ((long long)group * (((unsigned int)a.rows + 31) / 32) + row / 32);
            list = a.keys + ((long long)group * a.rows + row) * a.k;
            x = a.entries + ((long long)group * a.rows + row) * a.entry_stride;
            stride = a.entry_stride;
            at = starts[quarter], end = starts[quarter + 1];
            for (int to = end; tile > 0 && at < to;) {   // a pair that starts inside a row
                const int mid = (at + to) / 2;
                if (list[mid] >> 19 < (unsigned int)tile)
                    at = mid + 1;
                else
                    to = mid;
            }
        }
        fetch();
    }
    __device__ __forceinline__ void pick(int tile, uint32_t from)
    {
        for (;;) {
            const bool mine = key >> 19 == (unsigned int)tile;
            const unsigned int all = __ballot_sync(kFull, mine);
            if (all == 0u) break;
            unsigned int column = mine ? key >> 13 & 63u : 64u;
            uint32_t got = 0u;
            for (;;) {
                const unsigned int least = __reduce_min_sync(kFull, column);
                if (least == 64u) break;
                uint32_t v;
                tmem_load1(v, from + least);
                tmem_wait(v);
                const uint32_t there = __shfl_sync(kFull, v, key >> 8 & 31u);
                if (column == least) got = there, column = 64u;
            }
            if (mine) x[(long long)(key >> 8 & 31u) * stride + (key & 255u)] = __uint_as_float(got);
            at += __popc(all);
            fetch();
            if (all != kFull) break;
        }
    }
};

// One launch covers its units with pairs of blocks, each a persistent pair: one thread a block copies operand tiles
// into a ring of stages, one thread of the pair multiplies them into one of two accumulators in tensor memory, 16 warps a
// block read the other. No wait is without a limit: when one runs out the block's flag goes up, copies and products stop, the
// readers go through the rest of their units without waiting (so that their barriers stay matched), and the status
// word says that the outputs are undefined.
template <Kind KIND, int BN, bool MASK, int PLANES, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    tower_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                 const __grid_constant__ CUtensorMap map_g, const __grid_constant__ TowerArgs args)
{
    using S = Shape<KIND, BN>;
    extern __shared__ char raw[];
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    char *const shared = raw + (base - smem_addr(raw));
    const uint32_t staging = base + S::kStages * S::kStageBytes;
    int4 *const room = reinterpret_cast<int4 *>(shared + S::kStages * S::kStageBytes + S::kStaging);
    char *const tail = shared + S::kStages * S::kStageBytes + S::kStaging + S::kRoom;
    const uint32_t full = smem_addr(tail), empty = full + 8 * S::kStages, tmem_full = empty + 8 * S::kStages, tmem_empty = tmem_full + 16;
    volatile unsigned int *const abort_flag = reinterpret_cast<volatile unsigned int *>(tail + 8 * (2 * S::kStages + 4));
    const uint32_t tmem_word = tmem_empty + 16 + 4;
    volatile const uint32_t *const tmem_at = reinterpret_cast<volatile const uint32_t *>(tail + 8 * (2 * S::kStages + 4) + 4);

    const Tiles &t = args.t;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = pair_rank();
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, 1);
        for (int b = 0; b < 2; ++b) mbar_init(tmem_full + 8 * b, 1), mbar_init(tmem_empty + 8 * b, 2 * kEpilogue / 32);
        *abort_flag = 0u;
        barriers_visible();
    }
    __syncthreads();
    cluster_barrier();   // tensor memory is allocated by the pair as one: its other block has to be there (without this a pair waited for good, once in thousands of launches)
    if (warp == kEpilogue / 32) {
        if (lane == 0) prefetch_map(&map_a), prefetch_map(&map_b);
        __syncwarp();
        tmem_alloc(tmem_word, kTmemColumns);
    }
    fence_before();
    __syncthreads();
    cluster_barrier();
    fence_after();
    const uint32_t tmem = *tmem_at;
    next_may_start();
    previous_done();

    Unit u;
    if (warp == kEpilogue / 32) {   // ---- copies
        if (lane == 0) {
            Schedule<KIND> todo(t, pair, pairs);
            int stage = 0;
            uint32_t phase = 0;
            bool ok = !args.stall;
            long long copied = 0;
            while (ok && todo.next(t, u)) {
                const int az = args.a_z0 + u.g * args.a_z, bz = args.b_z0 + u.g * args.b_z;
                const int m0 = u.m * kTileM + (int)rank * 128, n0 = u.n * BN + (int)rank * (BN / 2);
                for (int kb = u.k0; kb < u.k1; ++kb) {
                    ok = wait_cluster(empty + 8 * stage, phase ^ 1, abort_flag, args.limit_ns);
                    if (!ok) break;
                    const uint32_t bar = peer_addr(full + 8 * stage, 0);
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * stage, 2 * S::kStageBytes);
                    const uint32_t a = base + stage * S::kStageBytes, b = a + S::kBytesA;
                    const int k = (kb >> args.k_shift) * kBlockK, z = az + (kb & args.k_shift) * args.plane_z;
                    if (S::kAlongKA) {
                        load_box(a, &map_a, k, args.a_m0 + m0, z, bar);
                    } else {
                        load_box(a, &map_a, m0, k, z, bar);
                        load_box(a + 64 * 128, &map_a, m0 + 64, k, z, bar);
                    }
                    if (S::kAlongKB) {
                        load_box(b, &map_b, k, args.b_n0 + n0, bz, bar);
                    } else {
                        load_box(b, &map_b, n0, args.b_k0 + k, bz, bar);
                        if (BN == 256) load_box(b + 64 * 128, &map_b, n0 + 64, args.b_k0 + k, bz, bar);
                    }
                    ++copied;
                    if (++stage == S::kStages) stage = 0, phase ^= 1;
                }
            }
            // every stage has been read: no arrival is on its way to this block any more
            for (int s = 0; ok && s < S::kStages && s < copied; ++s) {
                if (stage == 0) stage = S::kStages, phase ^= 1;
                --stage;
                ok = wait_cluster(empty + 8 * stage, phase, abort_flag, args.limit_ns);
            }
        }
        __syncwarp();
    } else if (warp == kEpilogue / 32 + 1) {   // ---- products
        if (lane == 0 && rank == 0) {
            Schedule<KIND> todo(t, pair, pairs);
            constexpr uint32_t instr = instruction<T>(kTileM, BN, S::kAlongKA, S::kAlongKB);
            constexpr int step_a = S::kAlongKA ? 32 : 2048, step_b = S::kAlongKB ? 32 : 2048;
            const uint64_t base_a = operand_base(S::kAlongKA, 64 * 128), base_b = operand_base(S::kAlongKB, 64 * 128);
            int stage = 0, buffer = 0;
            uint32_t phase = 0, buffer_phase = 0;
            bool ok = true;
            while (ok && todo.next(t, u)) {
                ok = wait_cluster(tmem_empty + 8 * buffer, buffer_phase ^ 1, abort_flag, args.limit_ns);
                if (!ok) break;
                fence_after();
                const uint32_t d = tmem + buffer * kTileN;
                for (int kb = u.k0; kb < u.k1; ++kb) {
                    ok = wait_cluster(full + 8 * stage, phase, abort_flag, args.limit_ns);
                    if (!ok) break;
                    fence_after();
                    const uint32_t a = base + stage * S::kStageBytes, b = a + S::kBytesA;
#pragma unroll
                    for (int k = 0; k < kBlockK / 16; ++k)
                        mma(d, operand(base_a, a + k * step_a), operand(base_b, b + k * step_b), instr, kb > u.k0 || k > 0);
                    commit_pair(empty + 8 * stage);
                    if (++stage == S::kStages) stage = 0, phase ^= 1;
                }
                if (!ok) break;
                commit_pair(tmem_full + 8 * buffer);
                buffer ^= 1;
                if (buffer == 0) buffer_phase ^= 1;
            }
        }
        __syncwarp();
    } else {   // ---- reading the products: a quarter of the tile's columns a warp
        Schedule<KIND> todo(t, pair, pairs);
        const int quarter = warp / 4, row_in = (warp % 4) * 32 + lane;
        const uint32_t lane_at = tmem + ((uint32_t)(warp % 4 * 32) << 16) + quarter * (BN / kParts);
        const uint32_t freed = peer_addr(tmem_empty, 0);
        int buffer = 0, last_g = -1, last_m = -1, parity = 0;
        uint32_t buffer_phase = 0;
        // a row a thread, or four (see mask_rows); row i of them
        constexpr int ROWS = MASK ? 4 : 1;
        auto row_at = [&](int i) { return MASK ? warp % 4 * 32 + lane / 4 + 8 * i : row_in; };
        int4 ask[ROWS];
        // STATS: the rows' statistics so far; GRAD: -m (in run_m), -log2 S and the factor of p
        float run_m[ROWS], run_s[ROWS], minus[ROWS], factor[ROWS];
        bool dead[ROWS], some_dead = false;
        // GRAD: the few entries of the row that this lane puts in: columns, and what stands there, p - q rounded once
        const int entry_row = MASK ? lane / 4 + 8 * (lane % 4) : lane;
        int entry_at[kFewEntries];
        T entry[PLANES][kFewEntries];
        int slot = 0;
        RowEntries own_entries;
        SortedEntries sorted_entries;
        auto release = [&] {
            fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(freed + 8 * buffer);
        };
        auto flush = [&] {
            if (last_m < 0) return;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                if (MASK) {   // four lanes have a row
#pragma unroll
                    for (int off = 1; off < 4; off *= 2) {
                        const float m = __shfl_xor_sync(kFull, run_m[i], off), s = __shfl_xor_sync(kFull, run_s[i], off);
                        const float to = fmaxf(run_m[i], m), base = to == neg_inf() ? 0.0f : to;
                        run_s[i] = run_s[i] * exp2_fast((run_m[i] - base) * args.c) + s * exp2_fast((m - base) * args.c);
                        run_m[i] = to;
                    }
                    if (lane % 4 != i) continue;
                    if (never_fits(ask[i])) run_m[i] = neg_inf(), run_s[i] = 0.0f;
                }
                const int row = last_m * kTileM + (int)rank * 128 + row_at(i);
                if (row < args.rows)
                    args.partial[((long long)last_g * args.rows + row) * args.slots + kParts * slot + quarter] = make_float2(run_m[i], run_s[i]);
            }
        };
        // A gradient that a wait ran out on the way to is NaN: all of it after a launch before this one, the block's tiles after one of its own.
        float undo = KIND == GRAD_REQUESTS || KIND == GRAD_HOSTS ? (tower_status ? __int_as_float(0x7FC00000) : 1.0f / args.range.factor()) : 1.0f;
        while (todo.next(t, u)) {
            const int local = u.m * kTileM + (int)rank * 128 + row_in;   // row of the launch
            if (KIND == STATS || KIND == GRAD) {
                if (u.g != last_g || u.m != last_m) {
                    if (KIND == STATS) {
                        flush();
                        slot = pair - pair_of(t.units, pairs, ((long long)u.g * t.m_tiles + u.m) * t.n_tiles);
                        if (args.keys)
                            sorted_entries.start(args, u.g, local - lane, quarter, u.n);
                        else
                            own_entries.start(args, (long long)u.g * args.rows + local, local < args.rows, quarter, u.n);
                        __syncwarp();
                    }
                    some_dead = false;
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        const int row = args.row0 + u.m * kTileM + (int)rank * 128 + row_at(i);
                        const bool inside = row < args.rows;
                        const long long at = (long long)(args.group0 + u.g) * args.rows + row;
                        run_m[i] = neg_inf(), run_s[i] = minus[i] = factor[i] = 0.0f;
                        dead[i] = true;
                        if (KIND == GRAD && inside) {
                            const float m = args.stats[at * args.stats_stride], s = args.stats[at * args.stats_stride + 1];
                            dead[i] = s == __int_as_float(0x7F800000);
                            run_m[i] = -m, minus[i] = -log2f(s);
                            factor[i] = args.range.scale * (args.grad_loss ? args.grad_loss[at] : 1.0f) * args.range.factor();
                        }
                        ask[i] = MASK && inside ? args.asks[at] : make_int4(0, 0, 0, 0);
                        some_dead |= dead[i];
                    }
                    some_dead = __any_sync(kFull, some_dead);
                    if (KIND == GRAD && args.ids) {
                        const int row = args.row0 + u.m * kTileM + (int)rank * 128 + warp % 4 * 32 + entry_row;
                        row_entries(args, (long long)(args.group0 + u.g) * args.rows + row, row < args.rows, entry_at, entry);
                    }
                    last_g = u.g, last_m = u.m;
                }
                const int4 *columns = room + parity * kTileN;
                if (MASK) {
                    const int n = u.n * BN + (int)threadIdx.x;
                    if (threadIdx.x < kTileN)
                        room[parity * kTileN + threadIdx.x] =
                            n < args.col_end ? args.room[(long long)(args.group0 + u.g) * args.hosts + args.col0 + n] : make_int4(-1, -1, -1, -1);
                    bar_sync(1, kEpilogue);
                    columns += quarter * (BN / kParts) + 2 * (lane % 4);
                    parity ^= 1;
                }
                wait_cluster(tmem_full + 8 * buffer, buffer_phase, abort_flag, args.limit_ns);
                __syncwarp();   // (the loads are the whole warp's)
                fence_after();
                const uint32_t at = lane_at + buffer * kTileN;
                const int n0 = u.n * BN + quarter * 64;
                if constexpr (KIND == STATS) {
                    if (args.keys)
                        sorted_entries.pick(u.n, at);
                    else
                        own_entries.pick(n0, at);
                }
                if constexpr (KIND == STATS && !MASK) {
                    uint32_t v[2][32];
                    tmem_load32(v[0], at), tmem_load32(v[1], at + 32);
                    tmem_wait(v[0]);
                    tmem_wait(v[1]);
                    release();
                    cut64(v[0], v[1], args.col_end - n0);
                    add64(run_m[0], run_s[0], v[0], v[1], args.c);
                } else {
                    // 32 columns at a time. G: with two values, a box of each, of 32 rows x 32 columns; with one, a box of 64 columns
                    const uint32_t box = staging + warp * 32 * 128;   // the warp's own
                    constexpr int kLine = PLANES == 2 ? 64 : 128;
                    // where 16-byte piece j of a line lies: as the tensor copies swizzle lines of that length
                    auto piece_at = [&](int line, int j) { return box + line * kLine + ((PLANES == 2 ? j ^ (line / 2 & 3) : j ^ (line & 7)) << 4); };
#pragma unroll 1
                    for (int sub = 0; sub < 2; ++sub) {
                        const bool first = PLANES == 2 || sub == 0, last = PLANES == 2 || sub == 1;   // of a box
                        auto box_is_free = [&] {   // what was in it before has left (looked at as late as can be: the copy takes as long as the loads and compares)
                            if (KIND == GRAD && first) {
                                if (lane == 0) stores_read_wait<0>();
                                __syncwarp();
                            }
                        };
                        // p f of two columns in one word, and (PLANES == 2) what was rounded off in another
                        auto words = [&](uint32_t (&w)[PLANES], uint32_t x0, uint32_t x1, float from, float less, float by, bool none) {
                            float e0, e1;
                            apart2(e0, e1, x0, x1, from, args.c, less);
                            e0 = exp2_fast(e0), e1 = exp2_fast(e1);
                            mul2(e0, e1, by, by);
                            w[0] = pack2(e0, e1, T());
                            if (PLANES == 2) {
                                const float2 rounded = unpack2(w[0], T());
                                w[PLANES - 1] = pack2(e0 - rounded.x, e1 - rounded.y, T());
                            }
                            if (some_dead && none) {
#pragma unroll
                                for (int i = 0; i < PLANES; ++i) w[i] = 0u;
                            }
                        };
                        if constexpr (MASK) {
                            uint32_t v[2][16];
                            tmem_load16(v[0], at + 32 * sub), tmem_load16(v[1], at + 32 * sub + (16u << 16));
                            tmem_wait(v[0]);
                            tmem_wait(v[1]);
                            if (sub == 1) release();
                            mask_rows(v, columns + 32 * sub, ask);
                            box_is_free();
                            if constexpr (KIND == STATS) {
#pragma unroll
                                for (int i = 0; i < ROWS; ++i) add8(run_m[i], run_s[i], v, i, args.c);
                            } else {   // four lanes a word of a piece each
#pragma unroll
                                for (int i = 0; i < ROWS; ++i)
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        const int x = 4 * j + 2 * (i % 2);
                                        uint32_t w[PLANES];
                                        words(w, v[i / 2][x], v[i / 2][x + 1], run_m[i], minus[i], factor[i], dead[i]);
                                        const uint32_t to = piece_at(row_at(i) % 32, PLANES == 2 ? j : 4 * sub + j) + lane % 4 * 4;
#pragma unroll
                                        for (int q = 0; q < PLANES; ++q) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + q * 2048), "r"(w[q]) : "memory");
                                    }
                            }
                        } else if constexpr (KIND == GRAD) {
                            uint32_t v[32];
                            tmem_load32(v, at + 32 * sub);
                            tmem_wait(v);
                            if (sub == 1) release();
                            const int left = args.col_end - n0 - 32 * sub;
                            if (left < 32) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[i] = i < left ? v[i] : 0xFF800000u;
                            }
                            box_is_free();
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t w[4][PLANES];
#pragma unroll
                                for (int i = 0; i < 4; ++i) words(w[i], v[8 * j + 2 * i], v[8 * j + 2 * i + 1], run_m[0], minus[0], factor[0], dead[0]);
                                const uint32_t to = piece_at(lane, PLANES == 2 ? j : 4 * sub + j);
#pragma unroll
                                for (int q = 0; q < PLANES; ++q)
                                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + q * 2048), "r"(w[0][q]), "r"(w[1][q]), "r"(w[2][q]), "r"(w[3][q])
                                                 : "memory");
                            }
                        }
                        if (KIND == GRAD && last) {
                            const int x0 = n0 + (PLANES == 2 ? 32 * sub : 0);
                            if (args.ids) {
                                __syncwarp();
#pragma unroll
                                for (int j = 0; j < kFewEntries; ++j) {
                                    const int col = entry_at[j] - x0;
                                    if ((unsigned int)col < kLine / 2u) {
                                        const uint32_t to = piece_at(entry_row, col / 8) + col % 8 * 2;
#pragma unroll
                                        for (int q = 0; q < PLANES; ++q)
                                            asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + q * 2048), "h"(*reinterpret_cast<const unsigned short *>(&entry[q][j])) : "memory");
                                    }
                                }
                            }
                            async_proxy_fence();
                            __syncwarp();
                            if (lane == 0) {
                                const int y = u.m * kTileM + (int)rank * 128 + warp % 4 * 32;
                                if (x0 < args.col_end && y < args.m_rows) {
#pragma unroll
                                    for (int q = 0; q < PLANES; ++q) store_box(&map_g, x0, y, u.g + q * t.groups, box + q * 2048);
                                }
                                stores_commit();
                            }
                        }
                    }
                }
            } else {
                if (!wait_cluster(tmem_full + 8 * buffer, buffer_phase, abort_flag, args.limit_ns)) undo = __int_as_float(0x7FC00000);
                __syncwarp();
                fence_after();
                const int n_first = u.n * BN + quarter * (BN / kParts);
#pragma unroll 1
                for (int sub = 0; sub < BN / kParts / 32; ++sub) {
                    uint32_t v[32];
                    __syncwarp();   // lanes without a row went past the stores
                    tmem_load32(v, lane_at + buffer * kTileN + 32 * sub);
                    tmem_wait(v);
                    if (sub == BN / kParts / 32 - 1) release();
                    if (u.k0 >= u.k1) {   // a part behind the end of a shorter piece
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0u;
                    }
                    const int n0 = n_first + 32 * sub, first = u.m * kTileM + (int)rank * 128 + warp % 4 * 32, rows_here = min(32, args.m_rows - first);
                    if (rows_here <= 0 || n0 >= args.width) continue;
                    if (args.sums) {
                        const int wide = (args.width + 3) & ~3;
                        float *to = args.sums + (((long long)u.split * t.groups + u.g) * args.m_rows + local) * wide + n0;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            if (lane >= rows_here || n0 + i >= wide) break;
                            float4 w = make_float4(__uint_as_float(v[i]), __uint_as_float(v[i + 1]), __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
                            if (args.add) {
                                const float4 old = *reinterpret_cast<const float4 *>(to + i);
                                w.x += old.x, w.y += old.y, w.z += old.z, w.w += old.w;
                            }
                            *reinterpret_cast<float4 *>(to + i) = w;
                        }
                        continue;
                    }
                    T *const out = static_cast<T *>(args.out) + (args.group0 + u.g) * args.out_group_stride + (args.out_row0 + (long long)first) * args.out_stride + n0;
                    uint4 w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(v[8 * i + j]) * undo;
                        w[i] = pack16(x, T());
                    }
                    if (args.out_wide && n0 + 32 <= args.width) {
                        uint4 *const to = reinterpret_cast<uint4 *>(out + lane * args.out_stride);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (lane < rows_here) to[i] = w[i];
                    } else {
                        // Rows that start anywhere, and their ends: a row at a time, a column a lane, through shared memory. (A row a lane, value by
                        // value: 6 x 31,616 hosts at width 475, 790 us, this 105.)
                        const uint32_t box = staging + warp * 32 * 64;
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + lane * 64 + ((i ^ (lane / 2 & 3)) << 4)), "r"(w[i].x), "r"(w[i].y),
                                         "r"(w[i].z), "r"(w[i].w)
                                         : "memory");
                        __syncwarp();
                        const bool mine = n0 + lane < args.width;
#pragma unroll 8
                        for (int r = 0; r < rows_here; ++r) {
                            unsigned short x;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(box + r * 64 + ((lane / 8 ^ (r / 2 & 3)) << 4) + lane % 8 * 2) : "memory");
                            if (mine) reinterpret_cast<unsigned short *>(out)[r * args.out_stride + lane] = x;
                        }
                    }
                }
            }
            buffer ^= 1;
            if (buffer == 0) buffer_phase ^= 1;
        }
        if (KIND == STATS) flush();
        if (KIND == GRAD && lane == 0) stores_drain();
    }

    fence_before();
    __syncthreads();
    if (*abort_flag) {   // copies and products in flight end within microseconds where the device works at all
        if (threadIdx.x == 0) atomicOr(&tower_status, STATUS_WAIT_TIMEOUT);
        const unsigned long long t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 1000000ull) __nanosleep(1000);
    }
    cluster_barrier();
    fence_after();
    if (warp == kEpilogue / 32) tmem_free(tmem, kTmemColumns);
    cluster_barrier();   // and given back as one: neither leaves before
}

// ---- small kernels around the products ----------------------------------------------------------------------
// Operands that a tensor copy cannot read (rows off 16-byte boundaries) are laid out once a call: rows of `wide` values, a
// multiple of 8, zeros behind the last.
template <typename T>
__global__ void lay_out_kernel(const T *src, long long stride, long long group_stride, int rows, int width, int wide, T *dst)
{
    next_may_start();
    previous_done();
    const unsigned int chunks = wide / 8;
    const long long n = (long long)rows * chunks, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    src += blockIdx.y * group_stride;
    dst += (long long)blockIdx.y * rows * wide;
    // Eight values from the 16-byte pieces that hold them (6 x 31,616 rows of 475, value by value 214 us, this 66). The pieces at a table's ends
    // may reach up to 14 bytes beyond it, which nothing uses: a piece that holds one of its values lies on an aligned 16 bytes with it, and
    // memory is mapped, and protected, in far larger units.
#pragma unroll 4
    for (long long i = first; i < n; i += (long long)gridDim.x * blockDim.x) {
        const long long row = n <= 0xFFFFFFFFll ? (unsigned int)i / chunks : i / chunks;
        const int col = (int)(i - row * chunks) * 8, left = min(8, width - col);
        const uintptr_t from = reinterpret_cast<uintptr_t>(src + row * stride + col);
        const int shift = (int)(from & 15);
        const uint4 *const at = reinterpret_cast<const uint4 *>(from - shift);
        uint4 w = at[0];
        if (shift) w = window16(w, shift + 2 * left > 16 ? at[1] : make_uint4(0, 0, 0, 0), shift);
        if (left < 8) {
            unsigned int x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = 2 * j + 1 < left ? x[j] : 2 * j < left ? x[j] & 0xFFFFu : 0u;
            w = make_uint4(x[0], x[1], x[2], x[3]);
        }
        *reinterpret_cast<uint4 *>(dst + i * 8) = w;
    }
}

// The entries of 32 rows (of one group) in the order of their quarters and tiles: counted, placed. What comes first within a tile differs from
// run to run; what is done with it does not. Dynamic shared memory: a counter for each quarter of a tile, or (`fine`) for each of its 64 columns:
// where a quarter has more entries than columns, those that are read together are then on few columns.
__global__ void __launch_bounds__(256) sort_entries_kernel(const int32_t *ids, int rows, int k, int hosts, int tiles, bool fine, unsigned int *keys, int *starts)
{
    extern __shared__ unsigned int counters[];   // [4][tiles][1 or 64]
    __shared__ unsigned int warps[8];
    next_may_start();
    previous_done();
    const unsigned int lists = ((unsigned int)rows + 31) / 32;
    const int g = (int)(blockIdx.x / lists), row0 = (int)(blockIdx.x % lists) * 32, quarter = tiles * (fine ? 64 : 1), n = 4 * quarter;
    const int count = min(32, rows - row0) * k;
    ids += ((long long)g * rows + row0) * k, keys += ((long long)g * rows + row0) * k, starts += 5ll * blockIdx.x;
    auto counter = [&](int id) { return counters + id / 64 % 4 * quarter + (fine ? id / 256 * 64 + id % 64 : id / 256); };
    for (int i = threadIdx.x; i < n; i += 256) counters[i] = 0u;
    __syncthreads();
    for (int e = threadIdx.x; e < count; e += 256) {
        const int id = ids[e];
        if (id >= 0 && id < hosts) atomicAdd(counter(id), 1u);
    }
    __syncthreads();
    // how many come before each: a stretch of counters a thread
    const int stretch = (n + 255) / 256, from = min(n, (int)threadIdx.x * stretch), to = min(n, from + stretch);
    unsigned int own = 0u;
    for (int i = from; i < to; ++i) own += counters[i];
    unsigned int before = own;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const unsigned int v = __shfl_up_sync(kFull, before, off);
        if (threadIdx.x % 32 >= off) before += v;
    }
    if (threadIdx.x % 32 == 31) warps[threadIdx.x / 32] = before;
    __syncthreads();
    before -= own;
    for (int w = 0; w < (int)threadIdx.x / 32; ++w) before += warps[w];
    if (threadIdx.x == 255) starts[4] = (int)(before + own);
    for (int i = from; i < to; ++i) {
        const unsigned int here = counters[i];
        counters[i] = before;
        before += here;
    }
    __syncthreads();
    if (threadIdx.x < 4) starts[threadIdx.x] = (int)counters[threadIdx.x * quarter];
    __syncthreads();
    for (int e = threadIdx.x; e < count; e += 256) {
        const int id = ids[e], row = e / k;
        if (id >= 0 && id < hosts)
            keys[atomicAdd(counter(id), 1u)] = (unsigned int)(id / 256) << 19 | (unsigned int)(id % 64) << 13 | (unsigned int)row << 8 | (unsigned int)(e - row * k);
    }
}

struct FinishArgs {
    int groups, rows, hosts, k, slots, pairs, m_tiles, n_tiles;
    long long units;
    const int32_t *ids;
    const float *teacher;
    long long teacher_stride;
    const int4 *asks, *room;
    float T, c;
    const float2 *partial;
    float *entries;                   // x at the entries, rows entry_stride apart
    int entry_stride;
    float *loss, *stats;
};

// pair_of, in 32 bits where they do (a 64-bit division costs as much as a row's products)
__device__ __forceinline__ int pair_at(const FinishArgs &f, long long unit)
{
    if (f.units > 0x7FFFFFFF) return pair_of(f.units, f.pairs, unit);
    const unsigned int n = (unsigned int)f.units, q = n / f.pairs, r = n % f.pairs, u = (unsigned int)unit;
    return (int)(u < r * (q + 1) ? u / (q + 1) : r + (u - r * (q + 1)) / q);
}

// TEAM lanes a row: its parts' statistics become one, and the logits at its hosts the loss.
template <int TEAM>
__global__ void __launch_bounds__(256) finish_kernel(const __grid_constant__ FinishArgs f)
{
    next_may_start();
    previous_done();
    const int lane = threadIdx.x % TEAM;
    const long long team = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / TEAM;
    const bool inside = team < (long long)f.groups * f.rows;
    const long long at = inside ? team : 0;
    const int g = (int)(at / f.rows), row = (int)(at % f.rows);
    auto team_max = [](float v) {
#pragma unroll
        for (int off = TEAM / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, off));
        return v;
    };

    const int4 ask = f.asks ? f.asks[at] : make_int4(0, 0, 0, 0);
    const long long first = ((long long)g * f.m_tiles + row / kTileM) * f.n_tiles;
    const int parts = kParts * (pair_at(f, first + f.n_tiles - 1) - pair_at(f, first) + 1);
    float m = neg_inf(), s = 0.0f;
    for (int i = lane; i < parts; i += TEAM) {
        const float2 p = f.partial[at * f.slots + i];
        const float to = fmaxf(m, p.x), base = to == neg_inf() ? 0.0f : to;
        s = s * exp2_fast((m - base) * f.c) + p.y * exp2_fast((p.x - base) * f.c);
        m = to;
    }
    const float top = team_max(m), base = top == neg_inf() ? 0.0f : top;
    s = lanes_sum(s * exp2_fast((m - base) * f.c), TEAM);

    // over this lane's entries: largest teacher logit, sum of w = 2^((t - tm) c), sum of w ((t - tm) - (x - m))
    float tm = neg_inf(), ts = 0.0f, tx = 0.0f;
    for (int j = lane; j < f.k && inside; j += TEAM) {
        const int id = f.ids[at * f.k + j];
        const float t = f.teacher ? f.teacher[at * f.teacher_stride + j] : 0.0f;
        float *const to = f.entries + at * f.entry_stride + j;
        bool there = id >= 0 && id < f.hosts;
        if (there && f.asks) there = !never_fits(ask) && fits(ask, f.room[(long long)g * f.hosts + id]);
        const float x = there ? *to : neg_inf();
        if (f.stats && !there) *to = x;
        if (x != neg_inf() && t > neg_inf()) {   // a NaN logit counts, and spoils its row
            const float top_now = fmaxf(tm, t), keep = exp2_fast((tm - top_now) * f.c), w = exp2_fast((t - top_now) * f.c);
            tx = ts > 0.0f ? keep * (tx + ts * (tm - top_now)) : 0.0f;
            tx += w * ((t - top_now) - (x - base));
            ts = ts * keep + w;
            tm = top_now;
        }
    }
    const float teacher_top = team_max(tm), keep = ts > 0.0f ? exp2_fast((tm - teacher_top) * f.c) : 0.0f;
    tx = lanes_sum(ts > 0.0f ? keep * (tx + ts * (tm - teacher_top)) : 0.0f, TEAM);
    ts = lanes_sum(keep * ts, TEAM);
    if (lane != 0 || !inside) return;
    const bool some = ts != 0.0f;   // or NaN
    if (f.loss) {
        float loss = some ? f.T * (tx / ts) + f.T * f.T * (logf(s) - logf(ts)) : 0.0f;
        if (tower_status) loss = __int_as_float(0x7FC00000);
        f.loss[at] = loss;
    }
    // a row without a counting entry has no gradient: S = inf makes its p 0
    if (f.stats) f.stats[at * (2 + f.k)] = some ? top : 0.0f, f.stats[at * (2 + f.k) + 1] = some ? s : __int_as_float(0x7F800000);
}

// Rows without a counting entry (S is inf) have gradient 0 whatever arrives, and what is not finite spoils its row at any range: the
// range follows neither.
__global__ void largest_kernel(const float *grad_loss, const float *stats, int stats_stride, long long n, unsigned int *largest)
{
    next_may_start();
    previous_done();
    float m = 0.0f;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const float g = fabsf(grad_loss[i]);
        if (g < __int_as_float(0x7F800000) && stats[i * stats_stride + 1] != __int_as_float(0x7F800000)) m = fmaxf(m, g);
    }
    m = warp_max(m);
    if (threadIdx.x % 32 == 0) atomicMax(largest, __float_as_uint(m));   // of floats above 0 the order of their bits
}
struct PatchArgs {
    int groups, group0, row0, rows_here, rows, host0, hosts_here, hosts, k;
    const int32_t *ids;
    const float *teacher;
    long long teacher_stride;
    const float *stats, *grad_loss;
    Range range;
    float c;
    void *grad;
    long long grad_stride, grad_group_stride, plane_stride;   // plane_stride 0: one plane
};
// G at the teacher's hosts, p - q rounded once. `lanes` lanes a row (a power of two); entries that name one host add up.
template <typename T>
__global__ void __launch_bounds__(256) patch_kernel(const __grid_constant__ PatchArgs p, int lanes)
{
    next_may_start();
    previous_done();
    const long long n = (long long)p.groups * p.rows_here, i = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / lanes;
    const bool inside = i < n;
    const int sub = threadIdx.x % lanes, g = inside ? (int)(i / p.rows_here) : 0, row = inside ? (int)(i % p.rows_here) : 0;
    const long long at = (long long)(p.group0 + g) * p.rows + p.row0 + row;
    const float *stats = p.stats + at * (2 + p.k), *teacher = p.teacher ? p.teacher + at * p.teacher_stride : nullptr;
    const int32_t *ids = p.ids + at * p.k;
    float top = neg_inf(), sum = 0.0f;
    for (int j = sub; inside && j < p.k; j += lanes) {
        const float t = teacher ? teacher[j] : 0.0f;
        if (stats[2 + j] != neg_inf() && t > top) top = t;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        if (off < lanes) top = fmaxf(top, __shfl_xor_sync(kFull, top, off));
    for (int j = sub; inside && j < p.k; j += lanes) {
        const float t = teacher ? teacher[j] : 0.0f;
        if (stats[2 + j] != neg_inf() && t > neg_inf()) sum += exp2_fast((t - top) * p.c);
    }
    sum = lanes_sum(sum, lanes);
    if (!inside || sum == 0.0f) return;   // (a sum that is not a number spoils the row)
    const float m = stats[0], minus = -log2f(stats[1]);
    const float factor = p.range.scale * (p.grad_loss ? p.grad_loss[at] : 1.0f) * p.range.factor();
    for (int j = sub; j < p.k; j += lanes) {
        const int id = ids[j];
        if (id < p.host0 || id >= p.host0 + p.hosts_here || stats[2 + j] == neg_inf()) continue;
        float q = 0.0f;
        for (int l = 0; l < p.k; ++l) {
            const float t = teacher ? teacher[l] : 0.0f;
            if (ids[l] == id && t > neg_inf()) q += exp2_fast((t - top) * p.c);
        }
        const float prob = exp2_fast(fmaf(stats[2 + j] - m, p.c, minus));
        const float value = (prob - q / sum) * factor;
        T *const to = static_cast<T *>(p.grad) + g * p.grad_group_stride + row * p.grad_stride + id - p.host0;
        *to = from_float<T>(value);
        if (p.plane_stride) to[p.plane_stride] = from_float<T>(value - to_float(from_float<T>(value)));
    }
}

// The parts' sums become the gradient: [splits][groups][rows][width to a multiple of 4] -> rows `stride` apart.
template <typename T>
__global__ void sums_kernel(const float *sums, int splits, int groups, int rows, int width, Range range, T *out, long long stride,
                            long long group_stride)
{
    next_may_start();
    previous_done();
    const unsigned int quads = (width + 3) / 4;
    const long long n = (long long)groups * rows * quads;
    const float undo = tower_status ? __int_as_float(0x7FC00000) : 1.0f / range.factor();
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const float4 *const from = reinterpret_cast<const float4 *>(sums) + i;
        float4 s = from[0];
#pragma unroll 8
        for (int k = 1; k < splits; ++k) {
            const float4 v = from[k * n];
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const long long row = n <= 0xFFFFFFFFll ? (unsigned int)i / quads : i / quads;
        const int col = (int)(i - row * quads) * 4;
        T *const to = out + row / rows * group_stride + row % rows * stride + col;
        const float x[4] = {s.x * undo, s.y * undo, s.z * undo, s.w * undo};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < width) to[j] = from_float<T>(x[j]);
    }
}

// rows of zeros (a batch without requests leaves the hosts' gradient at 0)
template <typename T>
__global__ void zero_kernel(T *out, int rows, int width, long long stride)
{
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < (long long)rows * width; i += (long long)gridDim.x * blockDim.x)
        out[i / width * stride + i % width] = from_float<T>(0.0f);
}

// ---- host side ----------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static const EncodeTiled f = [] {
        void *at = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &at, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            at = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(at);
    }();
    return f;
}

// A table of 16-bit values [groups][rows][width] whose rows lie on 16-byte boundaries
struct Table {
    const void *data;
    long long stride, group_stride;   // elements; group_stride 0: one slice for all groups
    int groups, rows, width;
};
// boxes of 64 columns (128 bytes), or 32, swizzled, x box_rows rows
int make_map(CUtensorMap *map, const Table &t, int box_rows, int dtype, int box_columns = 64)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return fail(NBOS_ERR_CUDA, "cuTensorMapEncodeTiled is not there");
    const bool shared = t.group_stride == 0;
    const cuuint64_t dims[3] = {(cuuint64_t)t.width, (cuuint64_t)t.rows, shared ? 1u : (cuuint64_t)t.groups};
    const cuuint64_t strides[2] = {(cuuint64_t)t.stride * 2, shared ? (cuuint64_t)t.stride * 2 : (cuuint64_t)t.group_stride * 2};
    const cuuint32_t box[3] = {(cuuint32_t)box_columns, (cuuint32_t)box_rows, 1}, steps[3] = {1, 1, 1};
    const CUresult r = encode(map, dtype == NBOS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                              const_cast<void *>(t.data), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              box_columns == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(NBOS_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return NBOS_OK;
}
// whether a tensor copy can read the table as it lies
bool readable(const void *data, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride)
{
    return aligned_to(data, 16) && (rows <= 1 || stride % 8 == 0) && (groups <= 1 || group_stride % 8 == 0);
}

// One temporary allocation of a call, given back in stream order.
class Workspace {
public:
    size_t add(size_t bytes)
    {
        const size_t at = size_;
        size_ += (bytes + 1023) & ~(size_t)1023;
        return at;
    }
    int allocate(int device, cudaStream_t stream)
    {
        cudaMemPool_t pool = nullptr;
        const int rc = library_pool(device, &pool);
        if (rc) return rc;
        const cudaError_t e = cudaMallocFromPoolAsync(reinterpret_cast<void **>(&data_), size_ ? size_ : 1, pool, stream);
        if (e != cudaSuccess) {
            cudaGetLastError();
            data_ = nullptr;
            return fail(NBOS_ERR_NO_MEMORY, "device allocation failed: %s", cudaGetErrorString(e));
        }
        stream_ = stream;
        return NBOS_OK;
    }
    template <typename V> V *at(size_t offset) const { return reinterpret_cast<V *>(data_ + offset); }
    ~Workspace()
    {
        if (data_) cudaFreeAsync(data_, stream_);
    }

private:
    char *data_ = nullptr;
    size_t size_ = 0;
    cudaStream_t stream_ = nullptr;
};

// Self-test: the thread's next launch of that kind copies nothing (nbos_probe_towers_stall).
struct Stall {
    int kind;
    unsigned long long limit_ns;
};
thread_local Stall stall_next = {-1, 0};

template <Kind KIND, int BN, bool MASK, int PLANES, typename T>
cudaError_t launch_tower(const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &g, const TowerArgs &args, int pairs, cudaStream_t stream)
{
    auto *kernel = tower_kernel<KIND, BN, MASK, PLANES, T>;
    // once a device (a bit each; two threads that meet here set the same value twice)
    static std::atomic<unsigned long long> allowed{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = device < 64 ? 1ull << device : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<KIND, BN>::kBytes);
        if (e != cudaSuccess) return e;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    TowerArgs p = args;
    p.limit_ns = kWaitLimitNs;
    if (stall_next.kind == KIND) {
        p.limit_ns = stall_next.limit_ns, p.stall = true;
        stall_next.kind = -1;
    }
    return launch_next(kernel, dim3(2 * pairs), kThreads, Shape<KIND, BN>::kBytes, stream, a, b, g, p);
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// Parts of the contraction: as many as make the pairs finish soonest, in units of one stage's products of a pair (0.4 us). A unit
// costs three stages besides its own; parts cost a launch and their sums, 256 KB a tile written and read.
void plan_splits(Tiles &t, int pairs)
{
    const long long tiles = (long long)t.groups * t.m_tiles * t.n_tiles;
    double best = 1e300;
    int best_splits = 1;
    for (int s = 1; s <= t.k_blocks && s <= 64; ++s) {
        const int blocks = ceil_div(t.k_blocks, s);
        if (ceil_div(t.k_blocks, blocks) != s) continue;
        const double cost = (double)ceil_div(tiles * s, pairs) * (blocks + 3) + (s > 1 ? 6.0 + 0.2 * tiles * s : 0.0);
        if (cost < best) best = cost, best_splits = s;
    }
    t.split_blocks = ceil_div(t.k_blocks, best_splits);
    t.splits = best_splits;
    t.units = tiles * t.splits;
}

struct Call {
    const nbos_towers *in;
    const int32_t *ids;
    const float *teacher;
    int64_t teacher_stride;
    int32_t k;
    float T;
    int device, sms;
    cudaStream_t stream;
};

int check(const nbos_towers *in, const int32_t *ids, const float *teacher, int64_t tstride, int32_t k, float T)
{
    if (!in) return fail(NBOS_ERR_INVALID_ARG, "towers is NULL");
    if (in->dtype != NBOS_BF16 && in->dtype != NBOS_F16)
        return fail(NBOS_ERR_INVALID_ARG, "vectors must be NBOS_BF16 or NBOS_F16 (got dtype %d)", in->dtype);
    if (in->n_hosts < 1 || in->n_hosts > NBOS_MAX_HOSTS)
        return fail(NBOS_ERR_INVALID_ARG, "n_hosts must be in 1..%d (got %d)", NBOS_MAX_HOSTS, in->n_hosts);
    if (in->width < 1 || in->width > NBOS_POLICY_MAX_WIDTH)
        return fail(NBOS_ERR_INVALID_ARG, "width must be in 1..%d (got %d)", NBOS_POLICY_MAX_WIDTH, in->width);
    if (in->n_groups < 1 || in->n_groups > 65535) return fail(NBOS_ERR_INVALID_ARG, "n_groups must be in 1..65535 (got %d)", in->n_groups);
    if (in->rows < 0 || in->rows > NBOS_POLICY_MAX_ROWS / in->n_groups)
        return fail(NBOS_ERR_INVALID_ARG, "rows must be >= 0 and n_groups * rows below 2^31 (got %lld)", (long long)in->rows);
    const int64_t far = (int64_t)1 << 38;
    if (in->rows > 1 && (in->request_stride < in->width || in->request_stride > far))
        return fail(NBOS_ERR_INVALID_ARG, "request_stride must be in width..2^38 (got %lld)", (long long)in->request_stride);
    if (in->n_hosts > 1 && (in->host_stride < in->width || in->host_stride > far))
        return fail(NBOS_ERR_INVALID_ARG, "host_stride must be in width..2^38 (got %lld)", (long long)in->host_stride);
    if (in->n_groups > 1 && (in->request_group_stride < 0 || in->request_group_stride > far || in->host_group_stride < 0 || in->host_group_stride > far))
        return fail(NBOS_ERR_INVALID_ARG, "group strides must be in 0..2^38");
    if (in->rows > 0 && (!in->requests || !in->hosts)) return fail(NBOS_ERR_INVALID_ARG, "towers->requests / hosts is NULL");
    if (!aligned_to(in->requests, 2) || !aligned_to(in->hosts, 2)) return fail(NBOS_ERR_INVALID_ARG, "vectors are not aligned to their element type");
    if (in->gradient_values < 0 || in->gradient_values > 2) return fail(NBOS_ERR_INVALID_ARG, "gradient_values must be 1 or 2, or 0 for 2 (got %d)", in->gradient_values);
    if (!in->asks != !in->room) return fail(NBOS_ERR_INVALID_ARG, "asks and room come together");
    if (!aligned_to(in->asks, 16) || !aligned_to(in->room, 16)) return fail(NBOS_ERR_INVALID_ARG, "asks / room must be 16-byte aligned");
    const int rc = check_k(k);
    if (rc) return rc;
    if (!(T > 0.0f) || !isfinite(T) || !isfinite(kLog2e / T) || !isfinite(T * T))
        return fail(NBOS_ERR_INVALID_ARG, "temperature must be finite and > 0 (as must 1 / T and T^2)");
    if (tstride != 0 && (tstride < k || tstride > ((int64_t)1 << 40)))
        return fail(NBOS_ERR_INVALID_ARG, "teacher_stride must be 0 or in k..2^40 (got %lld)", (long long)tstride);
    if (in->rows > 0 && !ids) return fail(NBOS_ERR_INVALID_ARG, "hosts is NULL");
    if (!aligned_to(ids, 4) || !aligned_to(teacher, 4)) return fail(NBOS_ERR_INVALID_ARG, "an int32 / float array is not 4-byte aligned");
    return NBOS_OK;
}

// The two operands as the products read them; `offset`: where the workspace holds a copy that was laid out, else -1.
struct Operand {
    Table table;
    const void *src;
    long long src_stride, src_group_stride;
    bool copied;
    size_t offset;
};
Operand plan_operand(Workspace &ws, const void *data, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride, int width)
{
    Operand o;
    const int wide = (width + 7) & ~7;
    if (rows <= 1) stride = wide;
    if (groups <= 1) group_stride = 0;
    o.src = data, o.src_stride = stride, o.src_group_stride = group_stride;
    o.table = Table{data, stride, group_stride, (int)groups, (int)rows, width};
    o.copied = !readable(data, rows, stride, groups, group_stride);
    o.offset = 0;
    if (o.copied) {
        const int slices = group_stride == 0 ? 1 : (int)groups;
        o.offset = ws.add((size_t)slices * rows * wide * 2);
        o.table.stride = wide, o.table.group_stride = group_stride == 0 ? 0 : (long long)rows * wide;
    }
    return o;
}
template <typename T>
cudaError_t lay_out(const Workspace &ws, Operand &o, int sms, cudaStream_t stream)
{
    if (!o.copied) return cudaSuccess;
    T *to = ws.at<T>(o.offset);
    o.table.data = to;
    const int slices = o.table.group_stride == 0 ? 1 : o.table.groups, wide = (int)o.table.stride;
    const long long chunks = (long long)o.table.rows * (wide / 8), most = 8ll * sms;
    const long long blocks = (chunks + 255) / 256 < most ? (chunks + 255) / 256 : most;
    return launch_next(lay_out_kernel<T>, dim3((unsigned int)blocks, slices), 256, 0, stream, static_cast<const T *>(o.src), o.src_stride,
                       o.src_group_stride, o.table.rows, o.table.width, wide, to);
}

template <typename T>
int forward(const Call &c, float *out_loss, float *out_stats)
{
    const nbos_towers *in = c.in;
    Workspace ws;
    Operand a = plan_operand(ws, in->requests, in->rows, in->request_stride, in->n_groups, in->request_group_stride, in->width);
    Operand b = plan_operand(ws, in->hosts, in->n_hosts, in->host_stride, in->n_groups, in->host_group_stride, in->width);
    TowerArgs args = {};
    args.t.groups = in->n_groups, args.t.m_tiles = ceil_div(in->rows, kTileM), args.t.n_tiles = ceil_div(in->n_hosts, kTileN);
    args.t.k_blocks = args.t.split_blocks = ceil_div(in->width, kBlockK), args.t.splits = 1;
    args.t.units = (long long)args.t.groups * args.t.m_tiles * args.t.n_tiles;
    const int pairs = args.t.units < c.sms / 2 ? (int)args.t.units : c.sms / 2;
    // a row's tiles lie with at most this many pairs, each of which leaves kParts parts
    args.slots = kParts * ((int)((args.t.n_tiles - 1) / (args.t.units / pairs)) + 2);
    const long long rows = in->n_groups * in->rows;
    const size_t o_partial = ws.add(sizeof(float2) * args.slots * rows);
    const bool few = c.k <= kFewEntries;
    const long long lists = (long long)in->n_groups * ((in->rows + 31) / 32);
    const size_t o_keys = ws.add(few ? 0 : sizeof(unsigned int) * c.k * rows), o_starts = ws.add(few ? 0 : sizeof(int) * 5 * lists);
    const size_t o_entries = ws.add(out_stats ? 0 : sizeof(float) * c.k * rows);
    int rc = ws.allocate(c.device, c.stream);
    if (rc) return rc;
    cudaError_t e = lay_out<T>(ws, a, c.sms, c.stream);
    if (e == cudaSuccess) e = lay_out<T>(ws, b, c.sms, c.stream);
    if (e != cudaSuccess) return cuda_fail(e, "towers: layout launch");
    CUtensorMap map_a, map_b;
    if ((rc = make_map(&map_a, a.table, 128, in->dtype)) || (rc = make_map(&map_b, b.table, 128, in->dtype))) return rc;
    args.a_z = a.table.group_stride != 0, args.b_z = b.table.group_stride != 0;
    args.rows = (int)in->rows, args.hosts = in->n_hosts, args.width = in->width, args.col_end = in->n_hosts;
    args.asks = reinterpret_cast<const int4 *>(in->asks), args.room = reinterpret_cast<const int4 *>(in->room);
    args.c = kLog2e / c.T;
    args.partial = ws.at<float2>(o_partial);
    args.ids = c.ids, args.k = c.k;
    args.entries = out_stats ? out_stats + 2 : ws.at<float>(o_entries), args.entry_stride = out_stats ? 2 + c.k : c.k;
    if (!few) {
        args.keys = ws.at<unsigned int>(o_keys), args.key_starts = ws.at<int>(o_starts);
        const bool fine = in->n_hosts <= 32 * c.k;   // (64 rows x 256 hosts with 256 entries each: 139 -> 58 us)
        const int shared = 4 * args.t.n_tiles * (fine ? 64 : 1) * (int)sizeof(unsigned int);
        e = allow_shared(sort_entries_kernel, shared);
        if (e == cudaSuccess)
            e = launch_next(sort_entries_kernel, dim3((unsigned int)lists), 256, shared, c.stream, c.ids, (int)in->rows, (int)c.k, (int)in->n_hosts,
                            args.t.n_tiles, fine, ws.at<unsigned int>(o_keys), ws.at<int>(o_starts));
        if (e != cudaSuccess) return cuda_fail(e, "towers: entries launch");
    }
    e = in->asks ? launch_tower<STATS, kTileN, true, 1, T>(map_a, map_b, map_a, args, pairs, c.stream)
                 : launch_tower<STATS, kTileN, false, 1, T>(map_a, map_b, map_a, args, pairs, c.stream);
    if (e != cudaSuccess) return cuda_fail(e, "towers: scores launch");
    FinishArgs f = {};
    f.groups = in->n_groups, f.rows = (int)in->rows, f.hosts = in->n_hosts, f.k = c.k, f.slots = args.slots, f.pairs = pairs;
    f.m_tiles = args.t.m_tiles, f.n_tiles = args.t.n_tiles, f.units = args.t.units;
    f.ids = c.ids, f.teacher = c.teacher, f.teacher_stride = c.teacher_stride, f.asks = args.asks, f.room = args.room;
    f.T = c.T, f.c = args.c, f.partial = args.partial, f.loss = out_loss, f.stats = out_stats;
    f.entries = args.entries, f.entry_stride = args.entry_stride;
    // A warp a row where a row has many parts, or few rows have many entries each; else eight lanes. (65,536 x 256, eight lanes / a warp: one
    // entry 27 / 53 us, 32 entries 87 / 109; 4,099 x 10,007 with capacities, 32 entries 76 / 57; 48 x 65,536, 3 entries 18 / 15.)
    e = args.slots > 32 || (c.k > 8 && rows <= 8192) ? launch_next(finish_kernel<32>, dim3((unsigned int)((rows + 7) / 8)), 256, 0, c.stream, f)
                                   : launch_next(finish_kernel<8>, dim3((unsigned int)((rows + 31) / 32)), 256, 0, c.stream, f);
    return e == cudaSuccess ? NBOS_OK : cuda_fail(e, "towers: loss launch");
}

template <Kind KIND, typename T>
cudaError_t launch_gradient(const CUtensorMap &a, const CUtensorMap &b, const TowerArgs &args, bool narrow, int pairs, cudaStream_t stream)
{
    const int p = args.t.units < pairs ? (int)args.t.units : pairs;
    return narrow ? launch_tower<KIND, 128, false, 1, T>(a, b, a, args, p, stream) : launch_tower<KIND, 256, false, 1, T>(a, b, a, args, p, stream);
}

// Pieces of G: whole groups while they fit; of a group that does not, runs along its longer side, so that the gradient that has to be
// added up over the pieces is the smaller one.
struct Pieces {
    int groups, rows, hosts;          // of a piece
};
Pieces plan_pieces(int groups, int rows, int hosts, int planes)
{
    const size_t group_bytes = (size_t)rows * ((hosts + 63) & ~63) * 2 * planes;
    Pieces p = {1, rows, hosts};
    auto even = [&](int n, int tile) {   // whole tiles, pieces of much the same size
        const int pieces = (int)((group_bytes + kPieceBytes - 1) / kPieceBytes), size = ceil_div(ceil_div(n, pieces), tile) * tile;
        return size < n ? size : n;
    };
    if (group_bytes <= kPieceBytes) {
        p.groups = (int)(kPieceBytes / group_bytes);
        if (p.groups > groups) p.groups = groups;
    } else if (rows <= hosts) {
        p.hosts = even(hosts, kTileN);
    } else {
        p.rows = even(rows, kTileM);
    }
    return p;
}
// do_one(first group, first row, first host) for one piece after the other, until it returns an error. (Counted in 64 bits: a piece
// may end at 2^31.)
template <typename F>
int for_pieces(const Pieces &p, int groups, int rows, int hosts, F do_one)
{
    for (long long g0 = 0; g0 < groups; g0 += p.groups)
        for (long long r0 = 0; r0 < rows; r0 += p.rows)
            for (long long h0 = 0; h0 < hosts; h0 += p.hosts) {
                const int rc = do_one((int)g0, (int)r0, (int)h0);
                if (rc) return rc;
            }
    return NBOS_OK;
}

template <typename T>
int backward(const Call &c, const float *stats, const float *grad_loss, float grad_scale, T *grad_a, long long a_stride, long long a_group_stride,
             T *grad_b, long long b_stride, long long b_group_stride)
{
    const nbos_towers *in = c.in;
    const int groups = in->n_groups, rows = (int)in->rows, hosts = in->n_hosts, width = in->width, pairs = c.sms / 2;
    // An entry of G is held as two 16-bit values, the second what rounding took off the first, and the contractions go over both. With one,
    // gradients are a sum of rounded terms: their errors against 64 bits are 1.4 times the plain form's, 2.5 where a group has one row, and far
    // more where the terms cancel. A row's p - q add up to 0, so what all hosts' vectors have in common does: where that is as large as what
    // tells them apart the error is 1.7 times the plain form's, at ten times as large 9.4 (2,048 x 4,096 of width 128; two values: 1.0 in
    // all of these). The second value doubles two of four products: 65,536 x 4,096 of width 256, both calls 528 us with one, 881 with two.
    const int planes = in->gradient_values == 1 ? 1 : 2;
    const Pieces piece_of = plan_pieces(groups, rows, hosts, planes);
    const int piece_groups = piece_of.groups, piece_rows = piece_of.rows, piece_hosts = piece_of.hosts;
    const bool cut_rows = piece_rows < rows, cut_hosts = piece_hosts < hosts;
    const int g_stride = (piece_hosts + 63) & ~63;
    const bool narrow = width <= 128;
    const int n_tiles = ceil_div(width, narrow ? 128 : 256);

    auto tiles = [&](int gn, int m, int n, int kb) {
        Tiles t = {gn, ceil_div(m, kTileM), n, kb, 1, kb, 0};
        t.units = (long long)gn * t.m_tiles * n;
        return t;
    };
    Tiles ta = tiles(piece_groups, piece_rows, n_tiles, planes * ceil_div(piece_hosts, kBlockK));
    Tiles tb = tiles(piece_groups, piece_hosts, n_tiles, planes * ceil_div(piece_rows, kBlockK));
    plan_splits(ta, pairs);
    plan_splits(tb, pairs);
    const bool sums_a = ta.splits > 1 || cut_hosts, sums_b = tb.splits > 1 || cut_rows;

    Workspace ws;
    Operand a = plan_operand(ws, in->requests, rows, in->request_stride, groups, in->request_group_stride, width);
    Operand b = plan_operand(ws, in->hosts, hosts, in->host_stride, groups, in->host_group_stride, width);
    const size_t o_g = ws.add((size_t)planes * piece_groups * piece_rows * g_stride * 2);
    const size_t o_a = ws.add(grad_a && sums_a ? sizeof(float) * ta.splits * piece_groups * piece_rows * ((width + 3) & ~3) : 0);
    const size_t o_b = ws.add(grad_b && sums_b ? sizeof(float) * tb.splits * piece_groups * piece_hosts * ((width + 3) & ~3) : 0);
    const size_t o_largest = ws.add(16);
    int rc = ws.allocate(c.device, c.stream);
    if (rc) return rc;
    cudaError_t e = lay_out<T>(ws, a, c.sms, c.stream);
    if (e == cudaSuccess) e = lay_out<T>(ws, b, c.sms, c.stream);
    const float scale = grad_scale * c.T;
    Range range = {nullptr, scale, (1.0f - 0x1p-8f) * (in->dtype == NBOS_F16 ? 0x1p15f : 1.0f)};
    if (grad_loss && e == cudaSuccess) {
        unsigned int *largest = ws.at<unsigned int>(o_largest);
        range.largest = largest;
        e = cudaMemsetAsync(largest, 0, 4, c.stream);
        const long long n = (long long)groups * rows, blocks = (n + 1023) / 1024;
        if (e == cudaSuccess)
            e = launch_next(largest_kernel, dim3((unsigned int)(blocks < 2 * c.sms ? blocks : 2 * c.sms)), 256, 0, c.stream, grad_loss, stats, 2 + c.k, n, largest);
    }
    if (e != cudaSuccess) return cuda_fail(e, "towers: layout launch");

    CUtensorMap a_rows, b_rows, a_cols, b_cols;   // boxes along the vectors, and across them
    if ((rc = make_map(&a_rows, a.table, 128, in->dtype)) || (rc = make_map(&b_rows, b.table, 128, in->dtype)) ||
        (rc = make_map(&a_cols, a.table, kBlockK, in->dtype)) || (rc = make_map(&b_cols, b.table, kBlockK, in->dtype)))
        return rc;
    const int az = a.table.group_stride != 0, bz = b.table.group_stride != 0;
    T *g = ws.at<T>(o_g);

    return for_pieces(piece_of, groups, rows, hosts, [&](int g0, int r0, int h0) -> int {
        const int gn = groups - g0 < piece_groups ? groups - g0 : piece_groups;
        const int rn = rows - r0 < piece_rows ? rows - r0 : piece_rows, hn = hosts - h0 < piece_hosts ? hosts - h0 : piece_hosts;
        const Table piece{g, g_stride, (long long)piece_rows * g_stride, planes * gn, rn, hn};
        CUtensorMap g_out, g_rows, g_cols;   // written, and read along rows and across them
        if ((rc = make_map(&g_out, piece, 32, in->dtype, planes == 2 ? 32 : 64)) || (rc = make_map(&g_rows, piece, 128, in->dtype)) || (rc = make_map(&g_cols, piece, kBlockK, in->dtype)))
            return rc;

        TowerArgs p = {};
        p.t = tiles(gn, rn, ceil_div(hn, kTileN), ceil_div(width, kBlockK));
        p.a_z = az, p.a_z0 = g0 * az, p.b_z = bz, p.b_z0 = g0 * bz, p.a_m0 = r0, p.b_n0 = h0;
        p.group0 = g0, p.row0 = r0, p.rows = rows, p.hosts = hosts, p.width = width, p.col0 = h0, p.col_end = hn, p.m_rows = rn;
        p.asks = reinterpret_cast<const int4 *>(in->asks), p.room = reinterpret_cast<const int4 *>(in->room);
        p.c = kLog2e / c.T, p.stats = stats, p.stats_stride = 2 + c.k, p.grad_loss = grad_loss, p.range = range;
        const bool few = c.k <= kFewEntries;
        if (few) p.ids = c.ids, p.teacher = c.teacher, p.teacher_stride = c.teacher_stride, p.k = c.k;
        const int used = p.t.units < pairs ? (int)p.t.units : pairs;
        if (planes == 2)
            e = in->asks ? launch_tower<GRAD, kTileN, true, 2, T>(a_rows, b_rows, g_out, p, used, c.stream)
                         : launch_tower<GRAD, kTileN, false, 2, T>(a_rows, b_rows, g_out, p, used, c.stream);
        else
            e = in->asks ? launch_tower<GRAD, kTileN, true, 1, T>(a_rows, b_rows, g_out, p, used, c.stream)
                         : launch_tower<GRAD, kTileN, false, 1, T>(a_rows, b_rows, g_out, p, used, c.stream);
        if (e != cudaSuccess) return cuda_fail(e, "towers: scores launch");

        if (!few) {
            PatchArgs q = {};
            q.groups = gn, q.group0 = g0, q.row0 = r0, q.rows_here = rn, q.rows = rows, q.host0 = h0, q.hosts_here = hn, q.hosts = hosts, q.k = c.k;
            q.ids = c.ids, q.teacher = c.teacher, q.teacher_stride = c.teacher_stride, q.stats = stats, q.grad_loss = grad_loss, q.range = range;
            q.c = p.c, q.grad = g, q.grad_stride = g_stride, q.grad_group_stride = piece.group_stride;
            q.plane_stride = planes == 2 ? gn * piece.group_stride : 0;
            int lanes = 1;
            while (lanes < 32 && lanes < c.k) lanes *= 2;
            e = launch_next(patch_kernel<T>, dim3((unsigned int)(((long long)gn * rn * lanes + 255) / 256)), 256, 0, c.stream, q, lanes);
            if (e != cudaSuccess) return cuda_fail(e, "towers: teacher launch");
        }

        if (grad_a) {
            TowerArgs d = {};
            d.t = ta, d.t.groups = gn, d.t.m_tiles = ceil_div(rn, kTileM), d.k_shift = planes - 1, d.plane_z = gn, d.t.k_blocks = planes * ceil_div(hn, kBlockK);
            d.t.units = (long long)gn * d.t.m_tiles * d.t.n_tiles * d.t.splits;
            d.a_z = 1, d.b_z = bz, d.b_z0 = g0 * bz, d.b_k0 = h0;
            d.group0 = g0, d.width = width, d.range = range, d.m_rows = rn, d.out_row0 = r0;
            d.out = grad_a, d.out_stride = a_stride, d.out_group_stride = a_group_stride, d.out_wide = readable(grad_a, rows, a_stride, groups, a_group_stride);
            d.sums = sums_a ? ws.at<float>(o_a) : nullptr, d.add = h0 > 0;
            e = launch_gradient<GRAD_REQUESTS, T>(g_rows, b_cols, d, narrow, pairs, c.stream);
            if (e == cudaSuccess && sums_a && h0 + hn == hosts) {
                const long long n = (long long)gn * rn * width, blocks = (n + 1023) / 1024;
                e = launch_next(sums_kernel<T>, dim3((unsigned int)(blocks < 8 * c.sms ? blocks : 8 * c.sms)), 256, 0, c.stream,
                                d.sums, ta.splits, gn, rn, width, range, grad_a + g0 * a_group_stride + r0 * a_stride, a_stride, a_group_stride);
            }
            if (e != cudaSuccess) return cuda_fail(e, "towers: gradient launch");
        }
        if (grad_b) {
            TowerArgs d = {};
            d.t = tb, d.t.groups = gn, d.t.m_tiles = ceil_div(hn, kTileM), d.k_shift = planes - 1, d.plane_z = gn, d.t.k_blocks = planes * ceil_div(rn, kBlockK);
            d.t.units = (long long)gn * d.t.m_tiles * d.t.n_tiles * d.t.splits;
            d.a_z = 1, d.b_z = az, d.b_z0 = g0 * az, d.b_k0 = r0;
            d.group0 = g0, d.width = width, d.range = range, d.m_rows = hn, d.out_row0 = h0;
            d.out = grad_b, d.out_stride = b_stride, d.out_group_stride = b_group_stride, d.out_wide = readable(grad_b, hosts, b_stride, groups, b_group_stride);
            d.sums = sums_b ? ws.at<float>(o_b) : nullptr, d.add = r0 > 0;
            e = launch_gradient<GRAD_HOSTS, T>(g_cols, a_cols, d, narrow, pairs, c.stream);
            if (e == cudaSuccess && sums_b && r0 + rn == rows) {
                const long long n = (long long)gn * hn * width, blocks = (n + 1023) / 1024;
                e = launch_next(sums_kernel<T>, dim3((unsigned int)(blocks < 8 * c.sms ? blocks : 8 * c.sms)), 256, 0, c.stream,
                                d.sums, tb.splits, gn, hn, width, range, grad_b + g0 * b_group_stride + h0 * b_stride, b_stride, b_group_stride);
            }
            if (e != cudaSuccess) return cuda_fail(e, "towers: gradient launch");
        }
        return NBOS_OK;
    });
}

int check_gradient(const char *what, const void *data, int64_t rows, int64_t stride, int64_t groups, int64_t group_stride, int width)
{
    if (!data) return NBOS_OK;
    const int64_t far = (int64_t)1 << 38;
    if (!aligned_to(data, 2)) return fail(NBOS_ERR_INVALID_ARG, "%s is not aligned to its element type", what);
    if (rows > 1 && (stride < width || stride > far)) return fail(NBOS_ERR_INVALID_ARG, "%s: the row stride must be in width..2^38", what);
    if (groups > 1 && (group_stride < (rows > 0 ? (rows - 1) * (rows > 1 ? stride : 0) + width : 0) || group_stride > far))
        return fail(NBOS_ERR_INVALID_ARG, "%s: groups must not overlap", what);
    return NBOS_OK;
}

}  // namespace
}  // namespace nbos

using namespace nbos;
using namespace nbos::policy;

extern "C" int nbos_policy_towers(const nbos_towers *towers, const int32_t *hosts, const float *teacher_logits, int64_t teacher_stride,
                                  int32_t k, float temperature, float *out_loss, float *out_stats, void *cuda_stream)
{
    int rc = check(towers, hosts, teacher_logits, teacher_stride, k, temperature);
    if (rc || towers->rows == 0) return rc;
    if (!out_loss && !out_stats) return fail(NBOS_ERR_INVALID_ARG, "no output asked for");
    if (!aligned_to(out_loss, 4) || !aligned_to(out_stats, 4)) return fail(NBOS_ERR_INVALID_ARG, "an int32 / float array is not 4-byte aligned");
    Call c{towers, hosts, teacher_logits, teacher_stride, k, temperature, 0, 0, static_cast<cudaStream_t>(cuda_stream)};
    if ((rc = check_sm100(&c.sms, &c.device))) return rc;
    return towers->dtype == NBOS_BF16 ? forward<__nv_bfloat16>(c, out_loss, out_stats) : forward<__half>(c, out_loss, out_stats);
}

extern "C" int nbos_policy_towers_backward(const nbos_towers *towers, const int32_t *hosts, const float *teacher_logits,
                                           int64_t teacher_stride, int32_t k, float temperature, const float *stats,
                                           const float *grad_loss, float grad_scale, void *out_grad_requests,
                                           int64_t grad_request_stride, int64_t grad_request_group_stride, void *out_grad_hosts,
                                           int64_t grad_host_stride, int64_t grad_host_group_stride, void *cuda_stream)
{
    int rc = check(towers, hosts, teacher_logits, teacher_stride, k, temperature);
    if (rc) return rc;
    const int64_t rows = towers->rows, groups = towers->n_groups;
    if (rows > 0 && !stats) return fail(NBOS_ERR_INVALID_ARG, "stats is NULL");
    if (!out_grad_requests && !out_grad_hosts) return rows > 0 ? fail(NBOS_ERR_INVALID_ARG, "no output asked for") : NBOS_OK;
    if (!aligned_to(stats, 4) || !aligned_to(grad_loss, 4)) return fail(NBOS_ERR_INVALID_ARG, "an int32 / float array is not 4-byte aligned");
    if ((rc = check_gradient("out_grad_requests", out_grad_requests, rows, grad_request_stride, groups, grad_request_group_stride, towers->width)) ||
        (rc = check_gradient("out_grad_hosts", out_grad_hosts, towers->n_hosts, grad_host_stride, groups, grad_host_group_stride, towers->width)))
        return rc;
    Call c{towers, hosts, teacher_logits, teacher_stride, k, temperature, 0, 0, static_cast<cudaStream_t>(cuda_stream)};
    if ((rc = check_sm100(&c.sms, &c.device))) return rc;
    if (rows == 0) {   // no request pulls at a host
        for (int64_t g = 0; out_grad_hosts && g < groups; ++g) {
            zero_kernel<<<c.sms, 256, 0, c.stream>>>(static_cast<__half *>(out_grad_hosts) + g * grad_host_group_stride, towers->n_hosts,
                                                     towers->width, towers->n_hosts > 1 ? (long long)grad_host_stride : 0ll);
            NBOS_CUDA_TRY(cudaGetLastError());
        }
        return NBOS_OK;
    }
    auto run = [&](auto zero) {
        using T = decltype(zero);
        return backward<T>(c, stats, grad_loss, grad_scale, static_cast<T *>(out_grad_requests), grad_request_stride, grad_request_group_stride,
                           static_cast<T *>(out_grad_hosts), grad_host_stride, grad_host_group_stride);
    };
    return towers->dtype == NBOS_BF16 ? run(__nv_bfloat16()) : run(__half());
}

extern "C" int nbos_policy_towers_status(void *cuda_stream)
{
    int sms = 0, device = 0;
    const int rc = check_sm100(&sms, &device);
    if (rc) return rc;
    unsigned int word = 0, zero = 0;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    NBOS_CUDA_TRY(cudaMemcpyFromSymbolAsync(&word, tower_status, sizeof(word), 0, cudaMemcpyDeviceToHost, stream));
    NBOS_CUDA_TRY(cudaStreamSynchronize(stream));
    if (!word) return NBOS_OK;
    NBOS_CUDA_TRY(cudaMemcpyToSymbolAsync(tower_status, &zero, sizeof(zero), 0, cudaMemcpyHostToDevice, stream));
    NBOS_CUDA_TRY(cudaStreamSynchronize(stream));
    return fail(NBOS_ERR_DEVICE_TIMEOUT, "a two-tower kernel gave up on a bounded wait; its outputs are undefined");
}

extern "C" int nbos_probe_towers_stall(int kernel, uint64_t limit_ns)
{
    if (kernel < -1 || kernel > GRAD_HOSTS) return fail(NBOS_ERR_INVALID_ARG, "kernel must be in -1..%d (got %d)", (int)GRAD_HOSTS, kernel);
    const uint64_t least = 1000000ull, most = 5000000000ull;
    stall_next = {kernel, limit_ns < least ? least : limit_ns > most ? most : limit_ns};
    return NBOS_OK;
}

extern "C" int nbos_probe_towers_pieces(int32_t n_groups, int64_t rows, int32_t n_hosts, int32_t gradient_values, int64_t *out_pieces,
                                        int64_t *out_entries, int64_t *out_largest_bytes)
{
    if (!out_pieces || !out_entries || !out_largest_bytes) return fail(NBOS_ERR_INVALID_ARG, "NULL output");
    if (n_groups < 1 || n_groups > 65535 || rows < 1 || rows > NBOS_POLICY_MAX_ROWS / n_groups || n_hosts < 1 || n_hosts > NBOS_MAX_HOSTS ||
        gradient_values < 1 || gradient_values > 2)
        return fail(NBOS_ERR_INVALID_ARG, "probe arguments out of range");
    const int n = (int)rows;
    const Pieces p = plan_pieces(n_groups, n, n_hosts, gradient_values);
    int64_t pieces = 0, entries = 0;
    const int rc = for_pieces(p, n_groups, n, n_hosts, [&](int g0, int r0, int h0) -> int {
        if (g0 < 0 || r0 < 0 || h0 < 0) return fail(NBOS_ERR_RANGE, "a piece starts at group %d, row %d, host %d", g0, r0, h0);
        auto here = [](int all, int from, int size) { return (int64_t)(all - from < size ? all - from : size); };
        ++pieces, entries += here(n_groups, g0, p.groups) * here(n, r0, p.rows) * here(n_hosts, h0, p.hosts);
        return NBOS_OK;
    });
    *out_pieces = pieces, *out_entries = entries;
    *out_largest_bytes = (int64_t)p.groups * p.rows * ((p.hosts + 63) & ~63) * 2 * gradient_values;
    return rc;
}
