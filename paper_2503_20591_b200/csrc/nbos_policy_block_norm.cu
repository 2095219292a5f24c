// The norms around a residual block: forward kernels and entry points; the mathematics stands in nbos_policy_block_norm.cuh.
#include "nbos_policy_block_norm.cuh"

namespace nbos {
namespace block_norm {
namespace {

template <typename T, int CH, bool BLOCK, bool WIDE, bool ANY, Gate GATE>
__global__ void __maxnreg__((kForwardRegs<WIDE>)) forward_kernel(const __grid_constant__ BlockArgs a, int team, int ahead)
{
    constexpr int VEC = kPer16<T>, TABLES = ANY && GATE == ROW_GATE ? 3 : 2;   // branch, residual, and a gate that may start anywhere
    using Ring = Ahead<T, VEC, CH, BLOCK, WIDE, ANY>;
    __shared__ float4 warps[2][8];
    extern __shared__ uint4 staged_words[];
    char *const staged = reinterpret_cast<char *>(staged_words);
    int half = 0;
    const int teams = BLOCK ? 1 : blockDim.x / team, t = BLOCK ? threadIdx.x : threadIdx.x % team, mine = BLOCK ? 0 : threadIdx.x / team;
    const Columns c(team, t, a.width, VEC, mine, teams);
    const int staged_bytes = Ring::bytes(ahead, TABLES, team, teams);
    float *const post = reinterpret_cast<float *>(staged + staged_bytes), *const pre = post + team * CH * VEC;
    if (BLOCK) {
        if (threadIdx.x < 16) warps[threadIdx.x / 8][threadIdx.x % 8] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        __syncthreads();
    }
    const bool gate_staged = Ring::kStaged && TABLES == 3 && (sizeof(T) == 4 || !a.gate_f32);
    auto of = [&](const void *table, long long stride, unsigned int row) { return static_cast<const T *>(table) + row * stride; };
    auto fetch = [&](long long first, long long end, int stage) {
        if (!Ring::kStaged) return;
        if (first < end) {
            const unsigned int row = (unsigned int)(first + mine < end ? first + mine : first);
            Ring::copy(staged, TABLES * stage, of(a.y, a.y_stride, row), row * a.y_stride, c);
            Ring::copy(staged, TABLES * stage + 1, of(a.x, a.x_stride, row), row * a.x_stride, c);
            if (gate_staged) Ring::copy(staged, TABLES * stage + 2, static_cast<const T *>(gate_at<T>(a, row)), row * a.gate_stride, c);
        }
        copies_commit();
    };
    Ring::clear(staged, staged_bytes);
    const Rows rows(a, GATE == SHARED_GATE);
    if (BLOCK || mine == 0) fill_weights<T, VEC, CH>(pre, a.pre, a.weight_f32, nullptr, false, team, t, a.width);
    for (unsigned int gi = rows.gate_from; gi < rows.gate_to; ++gi) {
        const long long end = (long long)gi * rows.per_gate + rows.part_to;
        long long first = (long long)gi * rows.per_gate + rows.part_from;
        if (ANY) team_sync<BLOCK>();   // the gate's rows before have left
        for (int i = 0; i < (ANY ? 1 : ahead); ++i) fetch(first + i * teams, end, i);
        if (!BLOCK) __syncthreads();   // the gate before is done with
        if (BLOCK || mine == 0)
            fill_weights<T, VEC, CH>(post, a.post, a.weight_f32, GATE == SHARED_GATE ? gate_at<T>(a, gi) : nullptr, a.gate_f32, team, t, a.width);
        if (!BLOCK) __syncthreads();   // (a block's threads read their own columns)
        int stage = 0;
        for (; first < end; first += teams) {
            const bool inside = first + mine < end;
            const unsigned int row = (unsigned int)(inside ? first + mine : first);
            const T *x = of(a.x, a.x_stride, row), *y = of(a.y, a.y_stride, row);
            float r[CH][VEC], s[2] = {0.0f, 0.0f};
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
                Ring::read(r[k], staged, TABLES * stage, k, y, c);
                dot_all(s, r[k], r[k]);
            }
            const float root_y = rsqrtf(fmaf(row_sum<BLOCK, WIDE>(s[0] + s[1], team, warps, half), a.per_width, a.eps));
            s[0] = s[1] = 0.0f;
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float w[VEC];
                scale_all(r[k], root_y);
                weights(w, post, k, team, t);
                mul_all(r[k], w);
                if (GATE == ROW_GATE) {
                    if (gate_staged)
                        Ring::read(w, staged, TABLES * stage + 2, k, static_cast<const T *>(gate_at<T>(a, row)), c);
                    else
                        get_either<T, VEC, ANY>(w, gate_at<T>(a, row), a.gate_f32, k, c);
                    mul_all(r[k], w);
                }
                Ring::read(w, staged, TABLES * stage + 1, k, x, c);
                add_scaled(r[k], w, a.alpha);
                dot_all(s, r[k], r[k]);
            }
            if (Ring::kStaged && !ANY) fetch(first + (long long)ahead * teams, end, stage);
            const float root_r = rsqrtf(fmaf(row_sum<BLOCK, WIDE>(s[0] + s[1], team, warps, half), a.per_width, a.eps));
            if (Ring::kStaged && ANY) team_sync<BLOCK>();   // results take the place of what has been read
            T *const out = static_cast<T *>(a.out) + row * a.out_stride, *const normed = static_cast<T *>(a.normed) + row * a.normed_stride;
            if (inside) {
                if (a.stats && t == 0) a.stats[2ll * row] = root_y, a.stats[2ll * row + 1] = root_r;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    if (a.out) Ring::write(out, staged, TABLES * stage, r[k], k, c);
                    if (a.normed) {
                        float w[VEC];
                        weights(w, pre, k, team, t);
                        scale_all(r[k], root_r);
                        mul_all(r[k], w);
                        Ring::write(normed, staged, TABLES * stage + 1, r[k], k, c);
                    }
                }
            }
            if (Ring::kStaged && ANY) {
                team_sync<BLOCK>();
                if (inside && a.out) Ring::row_out(out, staged, TABLES * stage, c);
                if (inside && a.normed) Ring::row_out(normed, staged, TABLES * stage + 1, c);
                if (ahead == 1) {
                    team_sync<BLOCK>();
                    fetch(first + teams, end, 0);
                }
            }
            stage = stage + 1 == ahead ? 0 : stage + 1;
        }
    }
}

template <typename T, Gate GATE>
cudaError_t run_forward(const BlockArgs &args, const Shape &s, int sms, cudaStream_t stream)
{
    return by_shape<T>(s, [&](auto chunks, auto block, auto wide, auto any) -> cudaError_t {
        auto *kernel = forward_kernel<T, chunks(), block(), wide(), any(), GATE>;
        static const int regs = kernel_registers(kernel);
        using Ring = Ahead<T, kPer16<T>, chunks(), block(), wide(), any()>;
        const int tables = any() && GATE == ROW_GATE ? 3 : 2, teams = s.threads / s.team, ahead = Ring::rows(tables, s.team, teams);
        const int shared = Ring::bytes(ahead, tables, s.team, teams) + 2 * s.team * kPer16<T> * chunks() * (int)sizeof(float);
        const cudaError_t e = allow_shared(kernel, shared);
        if (e != cudaSuccess) return e;
        BlockArgs a = args;
        const Split split = split_rows(a.rows, a.rows_per_gate, GATE == SHARED_GATE, teams, (long long)sms * resident_blocks(regs, s.threads, shared + 512));
        a.blocks_per_gate = split.share;
        kernel<<<(unsigned int)split.blocks, s.threads, shared, stream>>>(a, s.team, ahead);
        return cudaGetLastError();
    });
}
int check_table(const char *what, const void *p, int64_t rows, int64_t stride, int width, size_t elem, bool needed)
{
    if (!p) return needed && rows > 0 ? fail(NBOS_ERR_INVALID_ARG, "%s is NULL", what) : NBOS_OK;
    if (!aligned_to(p, elem)) return fail(NBOS_ERR_INVALID_ARG, "%s is not aligned to its element type", what);
    if (rows > 1 && (stride < width || stride > ((int64_t)1 << 40)))
        return fail(NBOS_ERR_INVALID_ARG, "%s: the row stride must be in width..2^40 (got %lld)", what, (long long)stride);
    return NBOS_OK;
}
bool known(int dtype) { return dtype == NBOS_F32 || dtype == NBOS_BF16 || dtype == NBOS_F16; }

int check(const nbos_block *b)
{
    if (!b) return fail(NBOS_ERR_INVALID_ARG, "block is NULL");
    if (!known(b->dtype)) return fail(NBOS_ERR_INVALID_ARG, "unknown dtype %d", b->dtype);
    if (b->gate_dtype != b->dtype && b->gate_dtype != NBOS_F32) return fail(NBOS_ERR_INVALID_ARG, "gate_dtype must be dtype or NBOS_F32 (got %d)", b->gate_dtype);
    if (b->weight_dtype != b->dtype && b->weight_dtype != NBOS_F32)
        return fail(NBOS_ERR_INVALID_ARG, "weight_dtype must be dtype or NBOS_F32 (got %d)", b->weight_dtype);
    if (b->width < 1 || b->width > NBOS_BLOCK_MAX_WIDTH) return fail(NBOS_ERR_INVALID_ARG, "width must be in 1..%d (got %d)", NBOS_BLOCK_MAX_WIDTH, b->width);
    if (b->rows < 0 || b->rows > NBOS_POLICY_MAX_ROWS) return fail(NBOS_ERR_INVALID_ARG, "rows must be in 0..2^31 - 1 (got %lld)", (long long)b->rows);
    if (!isfinite(b->residual_scale)) return fail(NBOS_ERR_INVALID_ARG, "residual_scale must be finite");
    if (!(b->eps >= 0.0f) || !isfinite(b->eps)) return fail(NBOS_ERR_INVALID_ARG, "eps must be finite and >= 0");
    const size_t elem = dtype_bytes(b->dtype);
    int rc;
    if ((rc = check_table("residual", b->residual, b->rows, b->residual_stride, b->width, elem, true)) ||
        (rc = check_table("branch", b->branch, b->rows, b->branch_stride, b->width, elem, true)))
        return rc;
    if (b->gate) {
        if (b->rows_per_gate < 1 || (b->rows > 0 && b->rows % b->rows_per_gate))
            return fail(NBOS_ERR_INVALID_ARG, "rows must be a multiple of rows_per_gate (got %lld)", (long long)b->rows_per_gate);
        if ((rc = check_table("gate", b->gate, b->rows / b->rows_per_gate, b->gate_stride, b->width, dtype_bytes(b->gate_dtype), true))) return rc;
    }
    if (!aligned_to(b->post_weight, dtype_bytes(b->weight_dtype)) || !aligned_to(b->pre_weight, dtype_bytes(b->weight_dtype)))
        return fail(NBOS_ERR_INVALID_ARG, "post_weight / pre_weight is not aligned to its element type");
    return NBOS_OK;
}

BlockArgs arguments(const nbos_block *b)
{
    BlockArgs a = {};
    a.x = b->residual, a.y = b->branch, a.gate = b->gate, a.post = b->post_weight, a.pre = b->pre_weight;
    a.x_stride = b->residual_stride, a.y_stride = b->branch_stride;
    a.rows = b->rows, a.rows_per_gate = b->gate ? b->rows_per_gate : 1, a.gate_stride = b->gate && b->rows > b->rows_per_gate ? b->gate_stride : 0;
    a.width = b->width, a.gate_f32 = b->gate_dtype == NBOS_F32, a.weight_f32 = b->weight_dtype == NBOS_F32;
    a.alpha = b->residual_scale, a.eps = b->eps, a.per_width = 1.0f / (float)b->width;
    return a;
}
bool gate_anywhere(const nbos_block *b, const void *gate, int64_t stride)
{
    return rows_anywhere(gate, gate && b->rows > b->rows_per_gate ? 2 : 1, stride, (int)dtype_bytes(b->gate_dtype));
}

int launched(cudaError_t e)
{
    if (e == cudaErrorMemoryAllocation) {
        cudaGetLastError();
        return fail(NBOS_ERR_NO_MEMORY, "device allocation failed: %s", cudaGetErrorString(e));
    }
    return e == cudaSuccess ? NBOS_OK : cuda_fail(e, "block norm launch");
}
template <typename T>
cudaError_t launch_forward(const BlockArgs &a, const Shape &s, int sms, cudaStream_t stream)
{
    if (!a.gate) return run_forward<T, NO_GATE>(a, s, sms, stream);
    if (a.rows_per_gate == 1) return run_forward<T, ROW_GATE>(a, s, sms, stream);
    return run_forward<T, SHARED_GATE>(a, s, sms, stream);
}

}  // namespace
}  // namespace block_norm
}  // namespace nbos

using namespace nbos;
using namespace nbos::policy;
using namespace nbos::block_norm;

extern "C" int nbos_policy_block_norm(const nbos_block *block, void *out_residual, int64_t out_residual_stride, void *out_normed,
                                      int64_t out_normed_stride, float *out_stats, void *cuda_stream)
{
    int rc = check(block);
    if (rc) return rc;
    const size_t elem = dtype_bytes(block->dtype);
    if ((rc = check_table("out_residual", out_residual, block->rows, out_residual_stride, block->width, elem, false)) ||
        (rc = check_table("out_normed", out_normed, block->rows, out_normed_stride, block->width, elem, false)))
        return rc;
    if (!aligned_to(out_stats, 4)) return fail(NBOS_ERR_INVALID_ARG, "out_stats is not 4-byte aligned");
    if (block->rows == 0) return NBOS_OK;
    if (!out_residual && !out_normed && !out_stats) return fail(NBOS_ERR_INVALID_ARG, "no output asked for");
    int sms = 0, device = 0;
    if ((rc = check_sm100(&sms, &device))) return rc;
    BlockArgs a = arguments(block);
    a.out = out_residual, a.normed = out_normed, a.out_stride = out_residual_stride, a.normed_stride = out_normed_stride, a.stats = out_stats;
    bool any = gate_anywhere(block, block->gate, block->gate_stride) || rows_anywhere(a.post, 1, 0, 4) || rows_anywhere(a.pre, 1, 0, 4);
    const struct { const void *p; int64_t stride; } tables[] = {{a.x, a.x_stride}, {a.y, a.y_stride}, {a.out, a.out_stride}, {a.normed, a.normed_stride}};
    for (const auto &t : tables) any |= rows_anywhere(t.p, a.rows, t.stride, (int)elem);
    const Shape s = plan(a.width, (int)elem, any);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return launched(block->dtype == NBOS_F32    ? launch_forward<float>(a, s, sms, stream)
                    : block->dtype == NBOS_BF16 ? launch_forward<__nv_bfloat16>(a, s, sms, stream)
                                                : launch_forward<__half>(a, s, sms, stream));
}

extern "C" int nbos_policy_block_norm_backward(const nbos_block *block, const float *stats, const void *grad_residual,
                                               int64_t grad_residual_stride, const void *grad_normed, int64_t grad_normed_stride,
                                               void *out_grad_residual, int64_t out_grad_residual_stride, void *out_grad_branch,
                                               int64_t out_grad_branch_stride, void *out_grad_gate, int64_t out_grad_gate_stride,
                                               void *out_grad_post, void *out_grad_pre, void *cuda_stream)
{
    int rc = check(block);
    if (rc) return rc;
    const size_t elem = dtype_bytes(block->dtype), gate_elem = dtype_bytes(block->gate_dtype), weight_elem = dtype_bytes(block->weight_dtype);
    const int64_t gates = block->gate ? block->rows / block->rows_per_gate : 0;
    if ((rc = check_table("grad_residual", grad_residual, block->rows, grad_residual_stride, block->width, elem, false)) ||
        (rc = check_table("grad_normed", grad_normed, block->rows, grad_normed_stride, block->width, elem, false)) ||
        (rc = check_table("out_grad_residual", out_grad_residual, block->rows, out_grad_residual_stride, block->width, elem, false)) ||
        (rc = check_table("out_grad_branch", out_grad_branch, block->rows, out_grad_branch_stride, block->width, elem, false)) ||
        (rc = check_table("out_grad_gate", out_grad_gate, gates, out_grad_gate_stride, block->width, gate_elem, false)))
        return rc;
    if (out_grad_gate && !block->gate) return fail(NBOS_ERR_INVALID_ARG, "out_grad_gate without a gate");
    if ((out_grad_post && !block->post_weight) || (out_grad_pre && !block->pre_weight)) return fail(NBOS_ERR_INVALID_ARG, "the gradient of a weight that is NULL");
    if (!aligned_to(out_grad_post, weight_elem) || !aligned_to(out_grad_pre, weight_elem))
        return fail(NBOS_ERR_INVALID_ARG, "out_grad_post / out_grad_pre is not aligned to its element type");
    if (!aligned_to(stats, 4)) return fail(NBOS_ERR_INVALID_ARG, "stats is not 4-byte aligned");
    if (!out_grad_residual && !out_grad_branch && !out_grad_gate && !out_grad_post && !out_grad_pre)
        return block->rows > 0 ? fail(NBOS_ERR_INVALID_ARG, "no output asked for") : NBOS_OK;
    if (block->rows > 0 && !stats) return fail(NBOS_ERR_INVALID_ARG, "stats is NULL");
    if (block->rows > 0 && !grad_residual && !grad_normed) return fail(NBOS_ERR_INVALID_ARG, "grad_residual and grad_normed are both NULL");
    int sms = 0, device = 0;
    if ((rc = check_sm100(&sms, &device))) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (block->rows == 0) {   // sums of nothing (a gate of no rows has no gradient to write)
        void *const weights[2] = {out_grad_post, out_grad_pre};
        for (void *w : weights)
            if (w) NBOS_CUDA_TRY(cudaMemsetAsync(w, 0, weight_elem * block->width, stream));
        return NBOS_OK;
    }
    cudaMemPool_t pool = nullptr;
    if ((rc = library_pool(device, &pool))) return rc;
    BlockArgs a = arguments(block);
    a.saved = stats, a.dr = grad_residual, a.dh = grad_normed, a.dr_stride = grad_residual_stride, a.dh_stride = grad_normed_stride;
    a.dx = out_grad_residual, a.dy = out_grad_branch, a.dx_stride = out_grad_residual_stride, a.dy_stride = out_grad_branch_stride;
    a.dgate = out_grad_gate, a.dgate_stride = gates > 1 ? out_grad_gate_stride : 0;
    bool any = gate_anywhere(block, block->gate, block->gate_stride) || gate_anywhere(block, out_grad_gate, out_grad_gate_stride) ||
               rows_anywhere(a.post, 1, 0, 4) || rows_anywhere(a.pre, 1, 0, 4);
    const struct { const void *p; int64_t stride; } tables[] = {{a.x, a.x_stride}, {a.y, a.y_stride}, {a.dr, a.dr_stride}, {a.dh, a.dh_stride},
                                                               {a.dx, a.dx_stride}, {a.dy, a.dy_stride}};
    for (const auto &t : tables) any |= rows_anywhere(t.p, a.rows, t.stride, (int)elem);
    const Shape s = plan(a.width, (int)elem, any);
    ColumnArgs c = {};
    c.width = a.width, c.gate = a.gate, c.post = a.post, c.gate_stride = a.gate_stride, c.gate_f32 = a.gate_f32, c.weight_f32 = a.weight_f32;
    c.dpost = out_grad_post, c.dpre = out_grad_pre, c.dgate = a.dgate, c.dgate_stride = a.dgate_stride;
    return launched(launch_backward(block->dtype, a, s, sms, c, pool, stream));
}
