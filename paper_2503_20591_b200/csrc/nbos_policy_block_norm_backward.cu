// Backward kernels of the norms around a residual block; the mathematics stands in nbos_policy_block_norm.cuh.
#include "nbos_policy_block_norm.cuh"

namespace nbos {
namespace block_norm {
namespace {

template <typename T, int CH, bool BLOCK, bool WIDE, bool ANY, Gate GATE>
__global__ void __maxnreg__((kBackwardRegs<WIDE>)) backward_kernel(const __grid_constant__ BlockArgs a, int team, int ahead)
{
    constexpr int VEC = kPer16<T>, TABLES = ANY && GATE == ROW_GATE ? 5 : 4;   // branch, residual, dh, dr, and a gate that may start anywhere
    using Ring = Ahead<T, VEC, CH, BLOCK, WIDE, ANY>;
    __shared__ float4 warps[2][8];
    // the rows to come; the weights; teams of a warp or less: [teams][width] of one sum after the other; shared gates: [width], gate S of the
    // gates behind the block
    extern __shared__ uint4 staged_words[];
    char *const staged = reinterpret_cast<char *>(staged_words);
    int half = 0;
    const int teams = BLOCK ? 1 : blockDim.x / team, t = BLOCK ? threadIdx.x : threadIdx.x % team, mine = BLOCK ? 0 : threadIdx.x / team;
    const Columns c(team, t, a.width, VEC, mine, teams);
    const int staged_bytes = Ring::bytes(ahead, TABLES, team, teams);
    float *const post = reinterpret_cast<float *>(staged + staged_bytes), *const pre = post + team * CH * VEC;
    float *const columns = pre + team * CH * VEC;
    float *const sum_q = columns + (BLOCK ? 0 : teams * a.width);
    float sum_s[CH][VEC], sum_p[CH][VEC];
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int col = (k * team + t) * VEC + i;
            sum_s[k][i] = sum_p[k][i] = 0.0f;
            if (GATE == SHARED_GATE && mine == 0 && col < a.width) sum_q[col] = 0.0f;   // this thread's own
        }
    if (BLOCK) {
        if (threadIdx.x < 16) warps[threadIdx.x / 8][threadIdx.x % 8] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        __syncthreads();
    }

    // this thread's sums over the block's teams (they hold the same columns), in a fixed order
    auto over_teams = [&](float (&v)[CH][VEC]) {
        if (BLOCK) return;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int col = (k * team + t) * VEC + i;
                if (col < a.width) columns[mine * a.width + col] = v[k][i];
            }
        __syncthreads();
        if (mine != 0) return;
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int col = (k * team + t) * VEC + i;
                if (col >= a.width) continue;
                for (int m = 1; m < teams; ++m) v[k][i] += columns[m * a.width + col];
            }
    };

    Ring::clear(staged, staged_bytes);
    const Rows rows(a, GATE == SHARED_GATE);
    auto of = [&](const void *table, long long stride, unsigned int row) { return static_cast<const T *>(table) + row * stride; };
    const bool gate_staged = Ring::kStaged && TABLES == 5 && (sizeof(T) == 4 || !a.gate_f32);
    auto fetch = [&](long long first, long long end, int stage) {
        if (!Ring::kStaged) return;
        if (first < end) {
            const unsigned int row = (unsigned int)(first + mine < end ? first + mine : first);
            Ring::copy(staged, TABLES * stage, of(a.y, a.y_stride, row), row * a.y_stride, c);
            Ring::copy(staged, TABLES * stage + 1, of(a.x, a.x_stride, row), row * a.x_stride, c);
            if (a.dh) Ring::copy(staged, TABLES * stage + 2, of(a.dh, a.dh_stride, row), row * a.dh_stride, c);
            if (a.dr) Ring::copy(staged, TABLES * stage + 3, of(a.dr, a.dr_stride, row), row * a.dr_stride, c);
            if (gate_staged) Ring::copy(staged, TABLES * stage + 4, static_cast<const T *>(gate_at<T>(a, row)), row * a.gate_stride, c);
        }
        copies_commit();
    };
    if (BLOCK || mine == 0) fill_weights<T, VEC, CH>(pre, a.pre, a.weight_f32, nullptr, false, team, t, a.width);
    for (unsigned int gi = rows.gate_from; gi < rows.gate_to; ++gi) {
        const void *const gate = GATE == SHARED_GATE ? gate_at<T>(a, gi) : nullptr;
        const long long end = (long long)gi * rows.per_gate + rows.part_to;
        int stage = 0;
        if (ANY) team_sync<BLOCK>();   // the gate's rows before have left
        for (int i = 0; i < (ANY ? 1 : ahead); ++i) fetch((long long)gi * rows.per_gate + rows.part_from + i * teams, end, i);
        if (!BLOCK) __syncthreads();   // the gate before is done with
        if (BLOCK || mine == 0) fill_weights<T, VEC, CH>(post, a.post, a.weight_f32, gate, a.gate_f32, team, t, a.width);
        if (!BLOCK) __syncthreads();   // (a block's threads read their own columns)
        for (long long first = (long long)gi * rows.per_gate + rows.part_from; first < end; first += teams) {
            const bool inside = first + mine < end;
            const unsigned int row = (unsigned int)(inside ? first + mine : first);
            const T *x = of(a.x, a.x_stride, row), *y = of(a.y, a.y_stride, row);
            const float root_y = a.saved[2ll * row], root_r = a.saved[2ll * row + 1];
            float r[CH][VEC], d[CH][VEC];   // r^, then f;  e, then d
            float s[2] = {0.0f, 0.0f}, mean_r = 0.0f;
            if (Ring::kStaged && ANY) {
                copies_wait<0>();
                team_sync<BLOCK>();    // all of the row is there, and all of the row before has left
                if (ahead == 2) fetch(first + teams, end, stage ^ 1);
            } else if (Ring::kStaged) {
                if (ahead == 2)
                    copies_wait<1>();
                else
                    copies_wait<0>();
            }
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float w[VEC];
                Ring::read(r[k], staged, TABLES * stage, k, y, c);
                scale_all(r[k], root_y);
                weights(w, post, k, team, t);
                mul_all(r[k], w);
                if (GATE == ROW_GATE) {
                    if (gate_staged)
                        Ring::read(w, staged, TABLES * stage + 4, k, static_cast<const T *>(gate_at<T>(a, row)), c);
                    else
                        get_either<T, VEC, ANY>(w, gate_at<T>(a, row), a.gate_f32, k, c);
                    mul_all(r[k], w);
                }
                Ring::read(w, staged, TABLES * stage + 1, k, x, c);
                add_scaled(r[k], w, a.alpha);
                scale_all(r[k], root_r);
                if (a.dh) {
                    Ring::read(d[k], staged, TABLES * stage + 2, k, of(a.dh, a.dh_stride, row), c);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) w[i] = inside ? d[k][i] : 0.0f;
                    add_product(sum_p[k], w, r[k]);
                    weights(w, pre, k, team, t);
                    mul_all(d[k], w);
                    dot_all(s, d[k], r[k]);
                }
            }
            if (a.dh) mean_r = row_sum<BLOCK, WIDE>(s[0] + s[1], team, warps, half) * a.per_width;
            s[0] = s[1] = 0.0f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float w[VEC], y_hat[VEC];
                if (a.dh) {
                    add_scaled(d[k], r[k], -mean_r);
                    scale_all(d[k], root_r);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[k][i] = 0.0f;
                }
                if (a.dr) {
                    Ring::read(w, staged, TABLES * stage + 3, k, of(a.dr, a.dr_stride, row), c);
                    add_scaled(d[k], w, 1.0f);
                }
                Ring::read(y_hat, staged, TABLES * stage, k, y, c);
                scale_all(y_hat, root_y);
#pragma unroll
                for (int i = 0; i < VEC; ++i) r[k][i] = d[k][i];
                if (GATE == ROW_GATE) {
                    if (gate_staged)
                        Ring::read(w, staged, TABLES * stage + 4, k, static_cast<const T *>(gate_at<T>(a, row)), c);
                    else
                        get_either<T, VEC, ANY>(w, gate_at<T>(a, row), a.gate_f32, k, c);
                    mul_all(r[k], w);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) w[i] = inside ? r[k][i] : 0.0f;
                add_product(sum_s[k], w, y_hat);
                weights(w, post, k, team, t);
                mul_all(r[k], w);
                dot_all(s, r[k], y_hat);
            }
            const float mean_y = a.dy ? row_sum<BLOCK, WIDE>(s[0] + s[1], team, warps, half) * a.per_width : 0.0f;
            if (Ring::kStaged && ANY) team_sync<BLOCK>();   // results take the place of what has been read
            T *const dx = static_cast<T *>(a.dx) + row * a.dx_stride, *const dy = static_cast<T *>(a.dy) + row * a.dy_stride;
            char *const dgate = static_cast<char *>(a.dgate) + row * a.dgate_stride * (a.gate_f32 ? 4 : (int)sizeof(T));
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                if (!inside) continue;
                float v[VEC], y_hat[VEC];
                Ring::read(y_hat, staged, TABLES * stage, k, y, c);
                scale_all(y_hat, root_y);
                if (GATE == ROW_GATE && a.dgate) {
                    weights(v, post, k, team, t);
                    mul_all(v, d[k]);
                    mul_all(v, y_hat);
                    if (gate_staged)
                        Ring::write(reinterpret_cast<T *>(dgate), staged, TABLES * stage + 1, v, k, c);
                    else
                        put_either<T, VEC, ANY>(dgate, a.gate_f32, v, k, c);
                }
                if (a.dy) {
                    add_scaled(r[k], y_hat, -mean_y);
                    scale_all(r[k], root_y);
                }
                if (a.dx) {
                    scale_all(d[k], a.alpha);
                    Ring::write(dx, staged, TABLES * stage + 3, d[k], k, c);
                }
                if (a.dy) Ring::write(dy, staged, TABLES * stage + 2, r[k], k, c);
            }
            if (Ring::kStaged && ANY) {
                team_sync<BLOCK>();
                if (inside && a.dx) Ring::row_out(dx, staged, TABLES * stage + 3, c);
                if (inside && a.dy) Ring::row_out(dy, staged, TABLES * stage + 2, c);
                if (inside && GATE == ROW_GATE && a.dgate && gate_staged) Ring::row_out(reinterpret_cast<T *>(dgate), staged, TABLES * stage + 1, c);
                if (ahead == 1) {
                    team_sync<BLOCK>();
                    fetch(first + teams, end, 0);
                }
            } else if (Ring::kStaged) {
                fetch(first + (long long)ahead * teams, end, stage);
            }
            stage = stage + 1 == ahead ? 0 : stage + 1;
        }
        if (GATE == SHARED_GATE && a.blocks_per_gate == 1) {   // all of the gate's rows are this block's
            over_teams(sum_s);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int col = (k * team + t) * VEC;
                if (mine == 0 && col < a.width) {
                    float g[VEC], v[VEC];
                    get_either<T, VEC, ANY>(g, gate, a.gate_f32, k, c);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] = a.post && col + i < a.width ? one_value(a.post, col + i, a.weight_f32, T()) : 1.0f;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        if (col + i < a.width) sum_q[col + i] = fmaf(g[i], sum_s[k][i], sum_q[col + i]);
                        v[i] *= sum_s[k][i];
                    }
                    if (a.dgate)
                        put_either<T, VEC, ANY>(static_cast<char *>(a.dgate) + gi * a.dgate_stride * (a.gate_f32 ? 4 : (int)sizeof(T)), a.gate_f32, v, k, c);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum_s[k][i] = 0.0f;
            }
        }
    }
    if (!a.partial) return;
    const bool whole = GATE == SHARED_GATE && a.blocks_per_gate == 1;
    if (!whole) over_teams(sum_s);
    over_teams(sum_p);
    if (mine != 0) return;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int col = (k * team + t) * VEC + i;
            if (col >= a.width) continue;
            float *to = a.partial + (long long)blockIdx.x * 2 * a.width + col;
            if constexpr (GATE == SHARED_GATE)
                to[0] = whole ? sum_q[col] : sum_s[k][i];
            else
                to[0] = sum_s[k][i];
            to[a.width] = sum_p[k][i];
        }
}

// The blocks' column sums become the gradients of the weights (blockIdx.y = 0) and of gate blockIdx.y - 1: 32 columns a
// block, its warps take every 32nd of the partial sums, four at a time.
constexpr int kColumnWarps = 32;
template <typename T>
__global__ void __launch_bounds__(32 * kColumnWarps) columns_kernel(const __grid_constant__ ColumnArgs c)
{
    __shared__ float sums[2][kColumnWarps][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
    const bool there = col < c.width;
    const int gate = (int)blockIdx.y - 1;
    const int from = gate < 0 ? 0 : gate * c.blocks_per_gate, to = gate < 0 ? c.blocks : from + c.blocks_per_gate;
    float s = 0.0f, p = 0.0f;
    for (int b0 = from + warp; b0 < to; b0 += 4 * kColumnWarps) {
        float v[4], w[4], q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int b = b0 + u * kColumnWarps;
            const bool take = there && b < to;
            const float *at = c.partial + (long long)b * 2 * c.width + col;
            v[u] = take ? at[0] : 0.0f;
            q[u] = take && gate < 0 ? at[c.width] : 0.0f;
            w[u] = take && gate < 0 && c.weigh ? one_value(c.gate, b / c.blocks_per_gate * c.gate_stride + col, c.gate_f32, T()) : 1.0f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) s = fmaf(v[u], w[u], s), p += q[u];
    }
    sums[0][warp][lane] = s, sums[1][warp][lane] = p;
    __syncthreads();
    if (warp != 0 || !there) return;
    for (int w = 1; w < kColumnWarps; ++w) s += sums[0][w][lane], p += sums[1][w][lane];
    auto write = [&](void *to, long long i, bool f32, float v) {
        if (f32 || sizeof(T) == 4)
            static_cast<float *>(to)[i] = v;
        else
            static_cast<T *>(to)[i] = from_float<T>(v);
    };
    if (gate >= 0) {
        write(c.dgate, gate * c.dgate_stride + col, c.gate_f32, s * (c.post ? one_value(c.post, col, c.weight_f32, T()) : 1.0f));
        return;
    }
    if (c.dpost) write(c.dpost, col, c.weight_f32, s);
    if (c.dpre) write(c.dpre, col, c.weight_f32, p);
}

template <typename T, Gate GATE>
cudaError_t run_backward(const BlockArgs &args, Shape s, int sms, ColumnArgs &c, cudaMemPool_t pool, cudaStream_t stream)
{
    const int tables = s.any && GATE == ROW_GATE ? 5 : 4;
    // 32-bit rows of nearly 8,192 values: staged rows, weights and a shared gate's sums are too much for shared memory, so they are not staged
    if (s.block && tables * (s.chunks * s.team + 2) * 16 + 2 * s.team * 16 * 4 + args.width * 4 > kMostShared) s.wide = true;
    return by_shape<T>(s, [&](auto chunks, auto block, auto wide, auto any) -> cudaError_t {
        auto *kernel = backward_kernel<T, chunks(), block(), wide(), any(), GATE>;
        static const int regs = kernel_registers(kernel);
        BlockArgs a = args;
        const int teams = s.threads / s.team;
        using Ring = Ahead<T, kPer16<T>, chunks(), block(), wide(), any()>;
        const int ahead = Ring::rows(tables, s.team, teams);
        const int shared = Ring::bytes(ahead, tables, s.team, teams) + (2 * s.team * kPer16<T> * chunks() + (s.block ? 0 : teams * a.width) +
                           (GATE == SHARED_GATE ? a.width : 0)) * (int)sizeof(float);
        cudaError_t e = allow_shared(kernel, shared);
        if (e != cudaSuccess) return e;
        const Split split = split_rows(a.rows, a.rows_per_gate, GATE == SHARED_GATE, teams, (long long)sms * resident_blocks(regs, s.threads, shared + 512));
        const long long share = split.share, blocks = split.blocks, gates = GATE == SHARED_GATE ? a.rows / a.rows_per_gate : 1;
        a.blocks_per_gate = split.share;
        float *partial = nullptr;
        const bool sums = c.dpost || c.dpre || (GATE == SHARED_GATE && a.dgate && share > 1);
        if (sums) {
            e = cudaMallocFromPoolAsync(reinterpret_cast<void **>(&partial), sizeof(float) * 2 * a.width * blocks, pool, stream);
            if (e != cudaSuccess) return e;
        }
        a.partial = partial;
        kernel<<<(unsigned int)blocks, s.threads, shared, stream>>>(a, s.team, ahead);
        e = cudaGetLastError();
        if (e == cudaSuccess && sums) {
            c.partial = partial, c.blocks = (int)blocks, c.blocks_per_gate = (int)share;
            c.weigh = GATE == SHARED_GATE && share > 1;
            const int dgates = GATE == SHARED_GATE && a.dgate && share > 1 ? (int)gates : 0;
            columns_kernel<T><<<dim3((a.width + 31) / 32, 1 + dgates), 32 * kColumnWarps, 0, stream>>>(c);
            e = cudaGetLastError();
        }
        if (partial) cudaFreeAsync(partial, stream);
        return e;
    });
}


template <typename T>
cudaError_t by_gate(const BlockArgs &a, const Shape &s, int sms, ColumnArgs &c, cudaMemPool_t pool, cudaStream_t stream)
{
    if (!a.gate) return run_backward<T, NO_GATE>(a, s, sms, c, pool, stream);
    if (a.rows_per_gate == 1) return run_backward<T, ROW_GATE>(a, s, sms, c, pool, stream);
    return run_backward<T, SHARED_GATE>(a, s, sms, c, pool, stream);
}

}  // namespace

cudaError_t launch_backward(int dtype, const BlockArgs &a, const Shape &s, int sms, ColumnArgs &c, cudaMemPool_t pool, cudaStream_t stream)
{
    if (dtype == NBOS_F32) return by_gate<float>(a, s, sms, c, pool, stream);
    return dtype == NBOS_BF16 ? by_gate<__nv_bfloat16>(a, s, sms, c, pool, stream) : by_gate<__half>(a, s, sms, c, pool, stream);
}

}  // namespace block_norm
}  // namespace nbos
