// Entry points of the training-step operators: every argument is checked here, on the host, before anything is
// launched; scratch comes from the context and grows on demand.

#include <cmath>

#include "train_common.cuh"

using namespace rubick;

#define CUDA_TRY(ctx, call, what) do { cudaError_t e_ = (call); if (e_ != cudaSuccess) return cuda_fail(ctx, e_, what); } while (0)

namespace {

int esize(int32_t dtype) { return dtype == RUBICK_F32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == RUBICK_BF16 || dtype == RUBICK_F16 || dtype == RUBICK_F32; }
bool on(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(size - 1)) == 0; }

int set_device(rubick_ctx *ctx)
{
    CUDA_TRY(ctx, cudaSetDevice(ctx->device), "cudaSetDevice");
    return RUBICK_OK;
}

// A new buffer for one that has become too small, twice as large at least, so that there are few of them: the old one is kept
// until the context goes, since earlier work of the stream and captured graphs may still use it.  In a capture nothing
// grows (an allocation would end it, and the clearing of counters would become part of the graph).
int grow(rubick_ctx *ctx, void **ptr, size_t *cap, size_t need, const char *what)
{
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    CUDA_TRY(ctx, cudaStreamIsCapturing(ctx->stream, &capture), "cudaStreamIsCapturing");
    if (capture != cudaStreamCaptureStatusNone) return fail(ctx, RUBICK_ESTATE, "training-step operators: scratch would have to grow during a stream capture; make the call once before it");
    if (*ptr && ctx->n_retired == int(sizeof(ctx->retired) / sizeof(ctx->retired[0]))) return fail(ctx, RUBICK_ENOMEM, "training-step operators: scratch has grown too often");
    const size_t least = 1 << 16;
    size_t bytes = need > 2 * *cap ? need : 2 * *cap;
    if (bytes < least) bytes = least;
    void *fresh = nullptr;
    if (cudaMalloc(&fresh, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        bytes = need;
        CUDA_TRY(ctx, cudaMalloc(&fresh, bytes), what);
    }
    if (*ptr) ctx->retired[ctx->n_retired++] = *ptr;
    *ptr = fresh;
    *cap = bytes;
    return RUBICK_OK;
}

// scratch of at least `bytes` bytes
int scratch(rubick_ctx *ctx, size_t bytes)
{
    return bytes <= ctx->cap_train ? RUBICK_OK : grow(ctx, &ctx->d_train, &ctx->cap_train, bytes, "cudaMalloc (training scratch)");
}

// arrival counters: zero when they are made, and every launch leaves them zero
int tickets(rubick_ctx *ctx, size_t n)
{
    if (n <= ctx->cap_tickets) return RUBICK_OK;
    void *fresh = ctx->d_tickets;
    size_t bytes = ctx->cap_tickets * sizeof(uint32_t);
    const int rc = grow(ctx, &fresh, &bytes, n * sizeof(uint32_t), "cudaMalloc (arrival counters)");
    if (rc) return rc;
    ctx->d_tickets = static_cast<uint32_t *>(fresh);
    ctx->cap_tickets = 0;                         // (none of them until they are cleared)
    CUDA_TRY(ctx, cudaMemsetAsync(fresh, 0, bytes, ctx->stream), "cudaMemsetAsync (arrival counters)");
    ctx->cap_tickets = bytes / sizeof(uint32_t);
    return RUBICK_OK;
}

int check_norm(rubick_ctx *ctx, const rubick_block_norm_desc *d, bool y, bool gate, const void *w_after, const void *w_before)
{
    if (!d) return fail(ctx, RUBICK_EINVAL, "block norm: null descriptor");
    if (d->rows < 0 || d->rows > 0x7fffffff) return fail(ctx, RUBICK_EINVAL, "block norm: rows must be 0 .. 2^31 - 1");
    if (d->cols < 1 || d->cols > RUBICK_MAX_NORM_COLS) return fail(ctx, RUBICK_EINVAL, "block norm: cols out of range");
    if (!known(d->dtype) || (d->wtype != d->dtype && d->wtype != RUBICK_F32)) return fail(ctx, RUBICK_EINVAL, "block norm: unknown type, or weights of another 16-bit type");
    if (d->flags & ~(RUBICK_NORM_AFTER | RUBICK_NORM_BEFORE | RUBICK_NORM_UNIT_OFFSET | RUBICK_NORM_TANH_GATE)) return fail(ctx, RUBICK_EINVAL, "block norm: unknown flag");
    if (!(d->eps > 0.f) || std::isinf(d->eps) || !std::isfinite(d->alpha)) return fail(ctx, RUBICK_EINVAL, "block norm: eps must be positive, eps and alpha finite");
    const bool after = d->flags & RUBICK_NORM_AFTER, before = d->flags & RUBICK_NORM_BEFORE;
    if (!y && (after || gate || !before)) return fail(ctx, RUBICK_EINVAL, "block norm: without y there is only the norm before the block");
    if ((w_after && !after) || (w_before && !before)) return fail(ctx, RUBICK_EINVAL, "block norm: weights of a norm that is not taken");
    if (!gate && (d->flags & RUBICK_NORM_TANH_GATE)) return fail(ctx, RUBICK_EINVAL, "block norm: tanh of no gate");
    if (gate && (d->group_rows < 1 || d->ld_gate < d->cols)) return fail(ctx, RUBICK_EINVAL, "block norm: group_rows or ld_gate too small");
    if (d->ld_x < d->cols || (y && d->ld_y < d->cols) || (before && d->ld_h < d->cols)) return fail(ctx, RUBICK_EINVAL, "block norm: a row distance is smaller than cols");
    const int ws = esize(d->wtype);
    if (!on(w_after, ws) || !on(w_before, ws)) return fail(ctx, RUBICK_EINVAL, "block norm: weights not aligned to their type");
    return RUBICK_OK;
}

int check_router(rubick_ctx *ctx, const rubick_router_desc *d)
{
    if (!d) return fail(ctx, RUBICK_EINVAL, "router: null descriptor");
    if (d->rows < 0 || d->rows > 0x7fffffff) return fail(ctx, RUBICK_EINVAL, "router: rows must be 0 .. 2^31 - 1");
    if (d->experts < 1 || d->experts > RUBICK_MAX_EXPERTS) return fail(ctx, RUBICK_EINVAL, "router: experts out of range");
    if (d->k < 1 || d->k > d->experts || d->k > RUBICK_MAX_CHOSEN) return fail(ctx, RUBICK_EINVAL, "router: k out of range");
    if (!known(d->dtype)) return fail(ctx, RUBICK_EINVAL, "router: unknown type");
    if (d->flags & ~RUBICK_ROUTER_RENORM) return fail(ctx, RUBICK_EINVAL, "router: unknown flag");
    if (d->group_rows < 1 || d->ld < d->experts) return fail(ctx, RUBICK_EINVAL, "router: group_rows or ld too small");
    if (!std::isfinite(d->coef)) return fail(ctx, RUBICK_EINVAL, "router: coef must be finite");
    if (d->reserved) return fail(ctx, RUBICK_EINVAL, "router: reserved must be 0");
    return RUBICK_OK;
}

int check_distill(rubick_ctx *ctx, const rubick_distill_desc *d)
{
    if (!d) return fail(ctx, RUBICK_EINVAL, "distill: null descriptor");
    if (d->rows < 0 || d->rows > 0x7fffffff) return fail(ctx, RUBICK_EINVAL, "distill: rows must be 0 .. 2^31 - 1");
    if (d->vocab < 1 || d->vocab > (1 << 30)) return fail(ctx, RUBICK_EINVAL, "distill: vocab out of range");
    if (d->k < 1 || d->k > RUBICK_MAX_TEACHER_LOGITS) return fail(ctx, RUBICK_EINVAL, "distill: k out of range");
    if (!known(d->dtype) || !known(d->ttype)) return fail(ctx, RUBICK_EINVAL, "distill: unknown type");
    if (d->ld < d->vocab) return fail(ctx, RUBICK_EINVAL, "distill: ld smaller than vocab");
    if (!(d->temperature > 0.f) || std::isinf(d->temperature)) return fail(ctx, RUBICK_EINVAL, "distill: the temperature must be positive and finite");
    if (d->reserved) return fail(ctx, RUBICK_EINVAL, "distill: reserved must be 0");
    return RUBICK_OK;
}

}  // namespace

extern "C" {

int rubick_block_norm_forward(rubick_ctx *ctx, const rubick_block_norm_desc *h_desc, const void *d_x, const void *d_y,
                              const void *d_w_after, const void *d_gate, const void *d_w_before, void *d_x_out,
                              void *d_h, float *d_rstd)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_norm(ctx, h_desc, d_y != nullptr, d_gate != nullptr, d_w_after, d_w_before);
    if (rc) return rc;
    if (h_desc->rows == 0) return RUBICK_OK;
    const bool before = h_desc->flags & RUBICK_NORM_BEFORE;
    if (!d_x || !d_y != !d_x_out || before != (d_h != nullptr)) return fail(ctx, RUBICK_EINVAL, "block norm: x is null, x_out does not go with y, or h with the norm before the block");
    const int es = esize(h_desc->dtype);
    if (!on(d_x, es) || !on(d_y, es) || !on(d_gate, es) || !on(d_x_out, es) || !on(d_h, es) || !on(d_rstd, 8)) return fail(ctx, RUBICK_EINVAL, "block norm: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    NormArgs a = {};
    a.d = *h_desc;
    a.x = d_x; a.y = d_y; a.w_after = d_w_after; a.gate = d_gate; a.w_before = d_w_before;
    a.x_out = d_x_out; a.h = d_h; a.rstd = d_rstd; a.status = ctx->d_status;
    if (!d_gate || a.d.group_rows > a.d.rows) a.d.group_rows = a.d.rows;
    CUDA_TRY(ctx, launch_norm_forward(a, ctx->num_sms, ctx->stream), "launch block_norm_forward");
    return RUBICK_OK;
}

int rubick_block_norm_backward(rubick_ctx *ctx, const rubick_block_norm_desc *h_desc, const void *d_x_out, const void *d_y,
                               const void *d_w_after, const void *d_gate, const void *d_w_before, const float *d_rstd,
                               const void *d_dx_out, const void *d_dh, void *d_dx, void *d_dy, float *d_dw_after,
                               void *d_dgate, float *d_dw_before)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_norm(ctx, h_desc, d_y != nullptr, d_gate != nullptr, d_w_after, d_w_before);
    if (rc) return rc;
    const bool after = h_desc->flags & RUBICK_NORM_AFTER, before = h_desc->flags & RUBICK_NORM_BEFORE;
    if ((d_dw_after && !after) || (d_dw_before && !before) || (d_dgate && !d_gate)) return fail(ctx, RUBICK_EINVAL, "block norm: gradient of something that is not there");
    const int es = esize(h_desc->dtype);
    if (!on(d_dw_after, 4) || !on(d_dw_before, 4)) return fail(ctx, RUBICK_EINVAL, "block norm: a tensor is not aligned to its type");
    if (h_desc->rows == 0) {
        if ((rc = set_device(ctx))) return rc;
        if (d_dw_after) CUDA_TRY(ctx, cudaMemsetAsync(d_dw_after, 0, size_t(h_desc->cols) * 4, ctx->stream), "clear dw_after");
        if (d_dw_before) CUDA_TRY(ctx, cudaMemsetAsync(d_dw_before, 0, size_t(h_desc->cols) * 4, ctx->stream), "clear dw_before");
        return RUBICK_OK;
    }
    if (!d_dx || !d_y != !d_dy || (before && (!d_x_out || !d_dh)) || (!before && d_dh)) return fail(ctx, RUBICK_EINVAL, "block norm: dx is null, dy does not go with y, or x_out and dh with the norm before the block");
    if ((after || before) && !d_rstd) return fail(ctx, RUBICK_EINVAL, "block norm: rstd is null");
    if (!on(d_x_out, es) || !on(d_y, es) || !on(d_gate, es) || !on(d_dx_out, es) || !on(d_dh, es) || !on(d_dx, es) || !on(d_dy, es) || !on(d_dgate, es) || !on(d_rstd, 8))
        return fail(ctx, RUBICK_EINVAL, "block norm: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    NormArgs a = {};
    a.d = *h_desc;
    if (!d_gate || a.d.group_rows > a.d.rows) a.d.group_rows = a.d.rows;
    a.x = before ? d_x_out : nullptr; a.y = d_y; a.w_after = d_w_after; a.gate = d_gate; a.w_before = d_w_before;
    a.status = ctx->d_status;
    a.rstd_in = d_rstd; a.dx_out = d_dx_out; a.dh = d_dh;
    a.dx = d_dx; a.dy = d_dy; a.dw_after = d_dw_after; a.dgate = d_dgate; a.dw_before = d_dw_before;
    const size_t need = norm_backward_scratch(a, ctx->num_sms, &a.chunk_rows, &a.n_chunks);
    if ((rc = scratch(ctx, need * sizeof(float)))) return rc;
    a.part = static_cast<float *>(ctx->d_train);
    CUDA_TRY(ctx, launch_norm_backward(a, ctx->num_sms, ctx->stream), "launch block_norm_backward");
    return RUBICK_OK;
}

int rubick_router_forward(rubick_ctx *ctx, const rubick_router_desc *h_desc, const void *d_logits, const uint8_t *d_mask,
                          int32_t *d_index, float *d_weight, int32_t *d_counts, float *d_prob_sum, int32_t *d_valid,
                          float *d_loss)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_router(ctx, h_desc);
    if (rc) return rc;
    if (!d_loss || !on(d_loss, 4)) return fail(ctx, RUBICK_EINVAL, "router: loss is null or not aligned");
    if (h_desc->rows == 0) {
        if ((rc = set_device(ctx))) return rc;
        CUDA_TRY(ctx, cudaMemsetAsync(d_loss, 0, 4, ctx->stream), "clear loss");
        return RUBICK_OK;
    }
    if (!d_logits || !d_index || !d_weight || !d_counts || !d_prob_sum || !d_valid) return fail(ctx, RUBICK_EINVAL, "router: null pointer");
    if (!on(d_logits, esize(h_desc->dtype)) || !on(d_index, 4) || !on(d_weight, 4) || !on(d_counts, 4) || !on(d_prob_sum, 4) || !on(d_valid, 4))
        return fail(ctx, RUBICK_EINVAL, "router: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    RouterArgs a = {};
    a.d = *h_desc;
    if (a.d.group_rows > a.d.rows) a.d.group_rows = a.d.rows;
    a.groups = (a.d.rows + a.d.group_rows - 1) / a.d.group_rows;
    a.logits = d_logits; a.mask = d_mask; a.index = d_index; a.weight = d_weight;
    a.counts = d_counts; a.prob_sum = d_prob_sum; a.valid = d_valid; a.loss = d_loss;
    a.chunks = router_chunks(a, ctx->num_sms);
    const size_t slots = a.chunks > 1 ? size_t(a.groups) * a.chunks : 0, E = size_t(a.d.experts);
    if ((rc = scratch(ctx, (slots * (2 * E + 1) + size_t(a.groups)) * 4))) return rc;
    if ((rc = tickets(ctx, size_t(a.groups) + 1))) return rc;
    a.group_loss = static_cast<float *>(ctx->d_train);
    a.part = a.group_loss + a.groups;
    a.part_counts = reinterpret_cast<int32_t *>(a.part + slots * E);
    a.tickets = ctx->d_tickets;
    CUDA_TRY(ctx, launch_router_forward(a, ctx->num_sms, ctx->stream), "launch router_forward");
    return RUBICK_OK;
}

int rubick_router_backward(rubick_ctx *ctx, const rubick_router_desc *h_desc, const void *d_logits, const int32_t *d_index,
                           const float *d_weight, const int32_t *d_counts, const int32_t *d_valid, const float *d_dloss,
                           const float *d_dweight, void *d_dlogits)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_router(ctx, h_desc);
    if (rc) return rc;
    if (h_desc->rows == 0) return RUBICK_OK;
    if (!d_logits || !d_index || !d_weight || !d_counts || !d_valid || !d_dlogits) return fail(ctx, RUBICK_EINVAL, "router: null pointer");
    const int es = esize(h_desc->dtype);
    if (!on(d_logits, es) || !on(d_dlogits, es) || !on(d_index, 4) || !on(d_weight, 4) || !on(d_counts, 4) || !on(d_valid, 4) || !on(d_dloss, 4) || !on(d_dweight, 4))
        return fail(ctx, RUBICK_EINVAL, "router: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    RouterArgs a = {};
    a.d = *h_desc;
    if (a.d.group_rows > a.d.rows) a.d.group_rows = a.d.rows;
    a.groups = (a.d.rows + a.d.group_rows - 1) / a.d.group_rows;
    a.logits = d_logits; a.index_in = d_index; a.weight_in = d_weight; a.counts_in = d_counts; a.valid_in = d_valid;
    a.dloss = d_dloss; a.dweight = d_dweight; a.dlogits = d_dlogits;
    // counted beforehand where every block's own count of the groups would take longer than one more launch (one row a group,
    // 64 experts: 32,000 groups 16.9 us counted by every block, 17.9 beforehand; 131,000: 42.4 and 35.3)
    if (a.groups > 32768) {
        if ((rc = scratch(ctx, sizeof(float)))) return rc;
        a.some = static_cast<const float *>(ctx->d_train);
    }
    CUDA_TRY(ctx, launch_router_backward(a, ctx->num_sms, ctx->stream), "launch router_backward");
    return RUBICK_OK;
}

int rubick_distill_forward(rubick_ctx *ctx, const rubick_distill_desc *h_desc, const void *d_z, const int32_t *d_index,
                           const void *d_teacher, float *d_loss, float *d_lse)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_distill(ctx, h_desc);
    if (rc) return rc;
    if (h_desc->rows == 0) return RUBICK_OK;
    if (!d_z || !d_index || !d_teacher || !d_loss) return fail(ctx, RUBICK_EINVAL, "distill: null pointer");
    if (!on(d_z, esize(h_desc->dtype)) || !on(d_teacher, esize(h_desc->ttype)) || !on(d_index, 4) || !on(d_loss, 4) || !on(d_lse, 4))
        return fail(ctx, RUBICK_EINVAL, "distill: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    DistillArgs a = {};
    a.d = *h_desc;
    a.status = ctx->d_status;
    a.z = d_z; a.index = d_index; a.teacher = d_teacher; a.loss = d_loss; a.lse = d_lse;
    CUDA_TRY(ctx, launch_distill_forward(a, ctx->num_sms, ctx->stream), "launch distill_forward");
    return RUBICK_OK;
}

int rubick_distill_backward(rubick_ctx *ctx, const rubick_distill_desc *h_desc, const void *d_z, const int32_t *d_index,
                            const void *d_teacher, const float *d_lse, const float *d_dloss, void *d_dz)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_distill(ctx, h_desc);
    if (rc) return rc;
    if (h_desc->rows == 0) return RUBICK_OK;
    if (!d_z || !d_index || !d_teacher || !d_lse || !d_dz) return fail(ctx, RUBICK_EINVAL, "distill: null pointer");
    const int es = esize(h_desc->dtype);
    if (!on(d_z, es) || !on(d_dz, es) || !on(d_teacher, esize(h_desc->ttype)) || !on(d_index, 4) || !on(d_lse, 4) || !on(d_dloss, 4))
        return fail(ctx, RUBICK_EINVAL, "distill: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    DistillArgs a = {};
    a.d = *h_desc;
    a.status = ctx->d_status;
    a.z = d_z; a.index = d_index; a.teacher = d_teacher; a.lse_in = d_lse; a.dloss = d_dloss; a.dz = d_dz;
    CUDA_TRY(ctx, launch_distill_backward(a, ctx->num_sms, ctx->stream), "launch distill_backward");
    return RUBICK_OK;
}

int rubick_distill_step(rubick_ctx *ctx, const rubick_distill_desc *h_desc, const void *d_z, const int32_t *d_index,
                        const void *d_teacher, const float *d_dloss, float *d_loss, float *d_lse, void *d_dz)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_distill(ctx, h_desc);
    if (rc) return rc;
    if (h_desc->rows == 0) return RUBICK_OK;
    if (!d_z || !d_index || !d_teacher || !d_loss || !d_lse || !d_dz) return fail(ctx, RUBICK_EINVAL, "distill: null pointer");
    const int es = esize(h_desc->dtype);
    if (!on(d_z, es) || !on(d_dz, es) || !on(d_teacher, esize(h_desc->ttype)) || !on(d_index, 4) || !on(d_lse, 4) || !on(d_loss, 4) || !on(d_dloss, 4))
        return fail(ctx, RUBICK_EINVAL, "distill: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    DistillArgs a = {};
    a.d = *h_desc;
    a.status = ctx->d_status;
    a.z = d_z; a.index = d_index; a.teacher = d_teacher; a.dloss = d_dloss; a.loss = d_loss; a.lse = d_lse; a.dz = d_dz;
    if (const size_t need = distill_step_scratch(a)) {
        if ((rc = scratch(ctx, need * sizeof(float)))) return rc;
        a.lse_low = static_cast<float *>(ctx->d_train);
    }
    CUDA_TRY(ctx, launch_distill_step(a, ctx->num_sms, ctx->stream), "launch distill_step");
    return RUBICK_OK;
}

}  // extern "C"
