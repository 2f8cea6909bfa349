// C ABI of strata_layer.h: argument validation and kernel launches.  Host-side only; the kernels live in route.cu,
// norm.cu and matmul.cu.
#include <cmath>

#include "ctx.cuh"
#include "layer.cuh"

namespace {

using namespace strata;

constexpr int kMaxCols = 32768;          // longest row the norm and the quantiser hold in registers
constexpr int kMaxInner = 131056;        // 2^31 / 128^2, less one: int8 sums cannot overflow int32

WorkQueue matmul_queue(const strata_ctx* c) { return WorkQueue{reinterpret_cast<unsigned int*>(c->ws) + 8}; }

bool on(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

strata_status check_route(const strata_ctx* ctx, const strata_route_params* r, int type, int64_t stride)
{
    const strata_moe_shape& s = ctx->shape;
    if (r->score != STRATA_SCORE_SOFTMAX && r->score != STRATA_SCORE_SIGMOID) return STRATA_ERR_INVALID_ARG;
    if (r->group_score != STRATA_GROUP_MAX && r->group_score != STRATA_GROUP_TOP2) return STRATA_ERR_INVALID_ARG;
    if (r->renormalise != 0 && r->renormalise != 1) return STRATA_ERR_INVALID_ARG;
    if (!std::isfinite(r->scale)) return STRATA_ERR_INVALID_ARG;
    if (type != STRATA_T_BF16 && type != STRATA_T_F32) return STRATA_ERR_INVALID_ARG;
    if (r->n_group < 1 || r->n_group > 32 || s.E % r->n_group != 0) return STRATA_ERR_SHAPE;
    if (r->topk_group < 1 || r->topk_group > r->n_group) return STRATA_ERR_SHAPE;
    if ((int64_t)r->topk_group * (s.E / r->n_group) < s.K) return STRATA_ERR_SHAPE;
    if (stride < s.E || (int64_t)s.R * s.T >= (1ll << 31)) return STRATA_ERR_SHAPE;
    return STRATA_OK;
}

// bf16 rows: 16-byte aligned, a stride that keeps every row so and does not overlap rows
strata_status check_rows16(const void* p, int64_t stride, int32_t cols)
{
    if (stride < cols || stride % 8 != 0) return STRATA_ERR_SHAPE;
    return on(p, 16) ? STRATA_OK : STRATA_ERR_ALIGNMENT;
}
strata_status check_codes(const void* q, int64_t q_stride, const float* q_scale, int64_t scale_stride, int32_t type,
                          int32_t cols)
{
    if (!q_scale) return STRATA_ERR_INVALID_ARG;
    if (type != STRATA_T_INT8 && type != STRATA_T_E4M3) return STRATA_ERR_INVALID_ARG;
    if (q_stride < cols || q_stride % 8 != 0 || scale_stride < 1) return STRATA_ERR_SHAPE;
    return on(q, 8) && on(q_scale, 4) ? STRATA_OK : STRATA_ERR_ALIGNMENT;
}
bool bad_extent(int64_t rows, int32_t cols)
{
    return rows < 0 || rows >= (1ll << 31) || cols < 8 || cols % 8 != 0 || cols > kMaxCols;
}

#define STRATA_CHECK(call)                          \
    do {                                            \
        const strata_status st_ = (call);           \
        if (st_ != STRATA_OK) return st_;           \
    } while (0)

}  // namespace

extern "C" {

strata_status strata_moe_route(strata_ctx* ctx, const strata_route_params* params, const void* logits,
                               int32_t logits_type, int64_t logits_stride, const float* bias, int32_t* topk_ids,
                               float* topk_w, void* stream)
{
    if (!ctx || !params || !logits || !topk_ids || !topk_w) return STRATA_ERR_INVALID_ARG;
    STRATA_CHECK(check_route(ctx, params, logits_type, logits_stride));
    if (!on(logits, logits_type == STRATA_T_F32 ? 4 : 2) || !on(bias, 4) || !on(topk_ids, 4) || !on(topk_w, 4))
        return STRATA_ERR_ALIGNMENT;
    if (ctx->device < 0) return STRATA_ERR_CUDA;
    DeviceGuard g(ctx->device);
    if (!g.ok) return STRATA_ERR_CUDA;
    return launched(ctx, launch_route(ctx->shape, *params, logits, logits_type, logits_stride, bias, topk_ids, topk_w,
                                      ctx->n_sm_device, static_cast<cudaStream_t>(stream)));
}

strata_status strata_moe_route_grad(strata_ctx* ctx, const strata_route_params* params, const void* logits,
                                    int32_t logits_type, int64_t logits_stride, const int32_t* topk_ids,
                                    const float* dtopk_w, void* dlogits, int64_t dlogits_stride, void* stream)
{
    if (!ctx || !params || !logits || !topk_ids || !dtopk_w || !dlogits) return STRATA_ERR_INVALID_ARG;
    STRATA_CHECK(check_route(ctx, params, logits_type, logits_stride));
    if (dlogits_stride < ctx->shape.E) return STRATA_ERR_SHAPE;
    const uintptr_t size = logits_type == STRATA_T_F32 ? 4 : 2;
    if (!on(logits, size) || !on(dlogits, size) || !on(topk_ids, 4) || !on(dtopk_w, 4)) return STRATA_ERR_ALIGNMENT;
    if (!ctx->ws) return STRATA_ERR_WORKSPACE;
    if (ctx->device < 0) return STRATA_ERR_CUDA;
    DeviceGuard g(ctx->device);
    if (!g.ok) return STRATA_ERR_CUDA;
    return launched(ctx, launch_route_grad(ctx->shape, *params, logits, logits_type, logits_stride, topk_ids, dtopk_w,
                                           dlogits, dlogits_stride, ctx->ws, static_cast<cudaStream_t>(stream)));
}

strata_status strata_norm(strata_ctx* ctx, const strata_norm_args* a, void* stream)
{
    if (!ctx || !a) return STRATA_ERR_INVALID_ARG;
    if (a->rows == 0) return bad_extent(0, a->cols) ? STRATA_ERR_SHAPE : STRATA_OK;    // row tensors may be NULL then
    if (!a->x || !a->weight || (!a->out && !a->q)) return STRATA_ERR_INVALID_ARG;
    if ((a->residual == nullptr) != (a->residual_out == nullptr)) return STRATA_ERR_INVALID_ARG;
    if (a->weight_type != STRATA_T_BF16 && a->weight_type != STRATA_T_F32) return STRATA_ERR_INVALID_ARG;
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return STRATA_ERR_INVALID_ARG;
    if (bad_extent(a->rows, a->cols)) return STRATA_ERR_SHAPE;
    STRATA_CHECK(check_rows16(a->x, a->x_stride, a->cols));
    if (a->residual) {
        STRATA_CHECK(check_rows16(a->residual, a->residual_stride, a->cols));
        STRATA_CHECK(check_rows16(a->residual_out, a->residual_out_stride, a->cols));
    }
    if (a->out) STRATA_CHECK(check_rows16(a->out, a->out_stride, a->cols));
    if (a->q) STRATA_CHECK(check_codes(a->q, a->q_stride, a->q_scale, a->q_scale_stride, a->q_type, a->cols));
    if (!on(a->weight, 16)) return STRATA_ERR_ALIGNMENT;
    if (ctx->device < 0) return STRATA_ERR_CUDA;
    DeviceGuard g(ctx->device);
    if (!g.ok) return STRATA_ERR_CUDA;
    return launched(ctx, launch_norm(*a, static_cast<cudaStream_t>(stream)));
}

strata_status strata_norm_grad_scratch_bytes(strata_ctx* ctx, int64_t rows, int32_t cols, size_t* bytes)
{
    if (!ctx || !bytes) return STRATA_ERR_INVALID_ARG;
    if (bad_extent(rows, cols)) return STRATA_ERR_SHAPE;
    *bytes = norm_grad_scratch_bytes(rows, cols, ctx->n_sm_device);
    return STRATA_OK;
}

strata_status strata_norm_grad(strata_ctx* ctx, const strata_norm_grad_args* a, void* stream)
{
    if (!ctx || !a || !a->weight || !a->dweight) return STRATA_ERR_INVALID_ARG;
    if (a->rows != 0 && (!a->dy || !a->h || !a->dx)) return STRATA_ERR_INVALID_ARG;
    if (a->weight_type != STRATA_T_BF16 && a->weight_type != STRATA_T_F32) return STRATA_ERR_INVALID_ARG;
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return STRATA_ERR_INVALID_ARG;
    if (bad_extent(a->rows, a->cols)) return STRATA_ERR_SHAPE;
    STRATA_CHECK(check_rows16(a->dy, a->dy_stride, a->cols));
    STRATA_CHECK(check_rows16(a->h, a->h_stride, a->cols));
    if (a->dresidual) STRATA_CHECK(check_rows16(a->dresidual, a->dresidual_stride, a->cols));
    STRATA_CHECK(check_rows16(a->dx, a->dx_stride, a->cols));
    if (!on(a->weight, 16) || !on(a->dweight, 4) || !on(a->scratch, 16)) return STRATA_ERR_ALIGNMENT;
    const size_t need = norm_grad_scratch_bytes(a->rows, a->cols, ctx->n_sm_device);
    if (a->scratch_bytes < need) return STRATA_ERR_CAPACITY;
    if (need > 0 && !a->scratch) return STRATA_ERR_INVALID_ARG;
    if (!ctx->ws) return STRATA_ERR_WORKSPACE;
    if (ctx->device < 0) return STRATA_ERR_CUDA;
    DeviceGuard g(ctx->device);
    if (!g.ok) return STRATA_ERR_CUDA;
    int n = 0;
    const cudaError_t err = launch_norm_grad(*a, ctx->ws, ctx->n_sm_device, static_cast<cudaStream_t>(stream), &n);
    return launched(ctx, err, (uint64_t)n);
}

strata_status strata_quantize_rows(strata_ctx* ctx, const void* x, int64_t x_stride, int64_t rows, int32_t cols,
                                   int32_t q_type, void* q, int64_t q_stride, float* q_scale, int64_t q_scale_stride,
                                   const int32_t* n_valid, void* stream)
{
    if (!ctx) return STRATA_ERR_INVALID_ARG;
    if (bad_extent(rows, cols)) return STRATA_ERR_SHAPE;
    if (rows == 0) return STRATA_OK;
    if (!x || !q) return STRATA_ERR_INVALID_ARG;
    STRATA_CHECK(check_rows16(x, x_stride, cols));
    STRATA_CHECK(check_codes(q, q_stride, q_scale, q_scale_stride, q_type, cols));
    if (!on(n_valid, 4)) return STRATA_ERR_ALIGNMENT;
    if (ctx->device < 0) return STRATA_ERR_CUDA;
    DeviceGuard g(ctx->device);
    if (!g.ok) return STRATA_ERR_CUDA;
    return launched(ctx, launch_quantize(x, x_stride, rows, cols, q_type, q, q_stride, q_scale, q_scale_stride, n_valid,
                                         static_cast<cudaStream_t>(stream)));
}

strata_status strata_moe_expert_matmul(strata_ctx* ctx, const strata_moe_layout_t* layout, const strata_matmul_args* a,
                                       void* stream)
{
    if (!ctx || !layout || !a || !a->a || !a->a_scale || !a->w || !a->w_scale || !a->out) return STRATA_ERR_INVALID_ARG;
    if (!layout->expert_offset || !layout->expert_count) return STRATA_ERR_INVALID_ARG;
    if (a->type != STRATA_T_INT8 && a->type != STRATA_T_E4M3) return STRATA_ERR_INVALID_ARG;
    if (a->gated != 0 && a->gated != 1) return STRATA_ERR_INVALID_ARG;
    const strata_moe_shape& s = ctx->shape;
    if (a->inner < 16 || a->inner % 16 != 0 || a->inner > kMaxInner) return STRATA_ERR_SHAPE;
    if (a->channels < 1 || (a->gated && a->channels % 2 != 0) || a->channels > (1 << 24)) return STRATA_ERR_SHAPE;
    if ((int64_t)a->channels * s.E >= (1ll << 31)) return STRATA_ERR_SHAPE;
    if (a->a_stride < a->inner || a->a_stride % 16 != 0 || a->a_stride >= (1ll << 40)) return STRATA_ERR_SHAPE;
    if (a->a_scale_stride < 1 || a->a_rows >= (1ll << 31)) return STRATA_ERR_SHAPE;
    if (a->out_stride < a->channels / (a->gated ? 2 : 1)) return STRATA_ERR_SHAPE;
    if (!on(a->a, 16) || !on(a->w, 16) || !on(a->a_scale, 4) || !on(a->w_scale, 4) || !on(a->out, 2))
        return STRATA_ERR_ALIGNMENT;
    if (!ctx->ws) return STRATA_ERR_WORKSPACE;
    if (a->a_rows < (int64_t)recv_rows(s)) return STRATA_ERR_CAPACITY;
    if (ctx->device < 0) return STRATA_ERR_CUDA;
    DeviceGuard g(ctx->device);
    if (!g.ok) return STRATA_ERR_CUDA;
    return launched(ctx, launch_expert_matmul(s, *layout, *a, ctx->ws, matmul_queue(ctx), ctx->n_sm, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
