// Entry points of the training-step operators: every argument is checked here, on the host, before anything is
// launched; scratch comes from the context and grows on demand.

#include <cmath>

#include "product.cuh"

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

bool is16(int32_t dtype) { return dtype == RUBICK_BF16 || dtype == RUBICK_F16; }
bool features(int32_t n) { return n >= 1 && n <= RUBICK_MAX_FEATURES; }
bool probability(float p) { return p >= 0.f && p < 1.f; }

DropArgs drop_args(float p, const uint64_t *seed)
{
    if (p == 0.f) return DropArgs{nullptr, 0, 1.f};
    return DropArgs{seed, uint32_t(double(p) * 4294967296.0), float(1.0 / (1.0 - double(p)))};
}

int check_linear(rubick_ctx *ctx, const rubick_linear_desc *d, const void *seed)
{
    if (!d) return fail(ctx, RUBICK_EINVAL, "linear: null descriptor");
    if (d->rows < 0 || d->rows > 0x7fffffff) return fail(ctx, RUBICK_EINVAL, "linear: rows must be 0 .. 2^31 - 1");
    if (!features(d->inputs) || !features(d->outputs)) return fail(ctx, RUBICK_EINVAL, "linear: inputs or outputs out of range");
    if (!is16(d->dtype) || (d->btype != d->dtype && d->btype != RUBICK_F32)) return fail(ctx, RUBICK_EINVAL, "linear: the operands are RUBICK_BF16 or RUBICK_F16, the bias of their type or RUBICK_F32");
    if (d->flags & ~RUBICK_WEIGHT_BY_OUTPUT) return fail(ctx, RUBICK_EINVAL, "linear: unknown flag");
    if (d->activation < RUBICK_ACT_NONE || d->activation > RUBICK_ACT_SILU) return fail(ctx, RUBICK_EINVAL, "linear: unknown activation");
    if (!probability(d->p)) return fail(ctx, RUBICK_EINVAL, "linear: p must be in [0, 1)");
    if (d->reserved) return fail(ctx, RUBICK_EINVAL, "linear: reserved must be 0");
    if (d->p > 0.f && (!seed || !on(seed, 8))) return fail(ctx, RUBICK_EINVAL, "linear: the seed is null or not aligned");
    return RUBICK_OK;
}
// distance between the rows of a weight against its width
bool weight_distance(int64_t ld, bool by_output, int32_t inputs, int32_t outputs) { return ld >= (by_output ? inputs : outputs); }

int check_dropout(rubick_ctx *ctx, const rubick_dropout_desc *d, const void *seed)
{
    if (!d) return fail(ctx, RUBICK_EINVAL, "dropout: null descriptor");
    if (d->rows < 0 || d->rows > 0x7fffffff) return fail(ctx, RUBICK_EINVAL, "dropout: rows must be 0 .. 2^31 - 1");
    if (!features(d->cols)) return fail(ctx, RUBICK_EINVAL, "dropout: cols out of range");
    if (!known(d->dtype)) return fail(ctx, RUBICK_EINVAL, "dropout: unknown type");
    if (!probability(d->p)) return fail(ctx, RUBICK_EINVAL, "dropout: p must be in [0, 1)");
    if (d->ld_x < d->cols || d->ld_out < d->cols) return fail(ctx, RUBICK_EINVAL, "dropout: a row distance is smaller than cols");
    if (d->reserved) return fail(ctx, RUBICK_EINVAL, "dropout: reserved must be 0");
    if (d->p > 0.f && (!seed || !on(seed, 8))) return fail(ctx, RUBICK_EINVAL, "dropout: the seed is null or not aligned");
    return RUBICK_OK;
}

int check_head(rubick_ctx *ctx, const rubick_head_loss_desc *d)
{
    if (!d) return fail(ctx, RUBICK_EINVAL, "head loss: null descriptor");
    if (d->rows < 0 || d->rows > 0x7fffffff) return fail(ctx, RUBICK_EINVAL, "head loss: rows must be 0 .. 2^31 - 1");
    if (!features(d->hidden)) return fail(ctx, RUBICK_EINVAL, "head loss: hidden out of range");
    if (d->vocab < 1 || d->vocab > (1 << 30)) return fail(ctx, RUBICK_EINVAL, "head loss: vocab out of range");
    if (!is16(d->dtype)) return fail(ctx, RUBICK_EINVAL, "head loss: the type is RUBICK_BF16 or RUBICK_F16");
    if (d->flags & ~RUBICK_WEIGHT_BY_OUTPUT) return fail(ctx, RUBICK_EINVAL, "head loss: unknown flag");
    if (d->ld_h < d->hidden || !weight_distance(d->ld_w, d->flags & RUBICK_WEIGHT_BY_OUTPUT, d->hidden, d->vocab)) return fail(ctx, RUBICK_EINVAL, "head loss: a row distance is too small");
    return RUBICK_OK;
}

// Parts of the scratch buffer: taken first, which adds them up, and addressed once the buffer is there.
struct Parts {
    size_t used = 0;
    size_t take(size_t bytes) { const size_t at = used; used += (bytes + 255) & ~size_t(255); return at; }
};
template <typename T> T *part(rubick_ctx *ctx, size_t at) { return reinterpret_cast<T *>(static_cast<char *>(ctx->d_train) + at); }
int64_t up8(int64_t n) { return (n + 7) & ~int64_t(7); }
bool wide16(const void *p, int64_t ld) { return train::aligned16(p) && (ld & 7) == 0; }

// An operand that the products cannot read as it lies gets a place in scratch and is laid out anew there.
struct Laid { bool copy; size_t at; int64_t rows, cols; };
Laid plan_operand(Parts &parts, const Operand &o, int64_t rows, int64_t cols)
{
    if (product_takes(o)) return Laid{false, 0, rows, cols};
    return Laid{true, parts.take(size_t(rows) * up8(cols) * 2), rows, cols};
}
void lay_out(rubick_ctx *ctx, LayOutArgs &all, const Laid &l, Operand &o)
{
    if (!l.copy) return;
    const Operand to = {part<void>(ctx, l.at), up8(l.cols), o.along_k};
    all.one[all.n++] = LayOutArgs::One{o.p, o.ld, const_cast<void *>(to.p), to.ld, l.rows, l.cols};
    o = to;
}

// The head's loss, its gradient, or both.
int head_loss(rubick_ctx *ctx, const rubick_head_loss_desc *h_desc, const void *d_h, const void *d_w, const int32_t *d_label,
              const float *d_lse_in, const float *d_dloss, float *d_loss, float *d_lse, void *d_dh, void *d_dw, bool forward, bool backward)
{
    const rubick_head_loss_desc &d = *h_desc;
    const bool by_output = d.flags & RUBICK_WEIGHT_BY_OUTPUT;
    int rc;
    if ((rc = set_device(ctx))) return rc;
    if (d.rows == 0) {
        if (d_dw) CUDA_TRY(ctx, cudaMemset2DAsync(d_dw, size_t(d.ld_w) * 2, 0, size_t(by_output ? d.hidden : d.vocab) * 2, by_output ? d.vocab : d.hidden, ctx->stream), "clear dw");
        return RUBICK_OK;
    }
    const int64_t ld_copy = up8(d.hidden);
    Parts parts;
    ProductArgs z = {};
    z.m = d.rows; z.n = d.vocab; z.k = d.hidden; z.dtype = d.dtype; z.status = ctx->d_status;
    z.label = d_label; z.vocab = d.vocab;
    Operand weight = {d_w, d.ld_w, by_output};
    const Laid laid = plan_operand(parts, weight, by_output ? d.vocab : d.hidden, by_output ? d.hidden : d.vocab);
    z.a.along_k = 1; z.b.along_k = by_output;
    const int64_t tiles = forward ? product_stats_pairs(z, ctx->num_sms) : 0;
    // the gradient of w sums over the rows, so that those without a label have to be zeros; elsewhere h is read as it lies
    const bool copied = backward && d_dw;
    Operand hidden = {d_h, d.ld_h, 1};
    const Laid laid_h = copied ? Laid{} : plan_operand(parts, hidden, d.rows, d.hidden);
    // Few rows: dz is kept in two numbers of 16 bits, the second one in rows of its own, which cost the products next to nothing.
    // (A row's gradient is mostly its label's entry, so with a handful of rows one rounding decides how far it is off.)
    const bool in_two = backward && product_few(d.rows);
    const int64_t dz_rows = in_two ? 2 * d.rows : d.rows;
    const size_t at_copy = copied ? parts.take(size_t(dz_rows) * ld_copy * 2) : 0;
    const size_t at_stats = forward ? parts.take(size_t(tiles) * d.rows * sizeof(float2)) : 0, at_label = forward ? parts.take(size_t(d.rows) * 4) : 0;
    const size_t at_base = forward && backward ? parts.take(size_t(d.rows) * 4) : 0, at_rest = forward && backward ? parts.take(size_t(d.rows) * 4) : 0;
    const size_t at_scale = backward ? parts.take(8) : 0;
    // the vocabulary of a piece: as much as 512 MB of dz take, in whole tiles, and no longer than sums in tensor memory should be
    int64_t piece = (int64_t(512) << 20) / (2 * dz_rows) / 256 * 256;
    if (piece < 256) piece = 256;
    if (piece > 1 << 19) piece = 1 << 19;
    if (piece > d.vocab) piece = d.vocab;
    const int64_t ld_dz = up8(piece);
    const bool several = piece < d.vocab;
    // Where dz is one piece, a step writes the exponentials that it sums up to dz's place and makes dz of them there, instead of
    // working the logits out again: three products, not four (2,048 x 4,096 x 128,000 bf16 5.3 ms, 7.0 with four).  It pays
    // where a product costs more than reading and writing dz once: from 640 features on (4,096 x 32,000: 768 features 642 us,
    // 664 with four; 512: 490 and 471), or where dz stays in L2 (1,024 x 256 x 16,000 89 us, 98; 512 x 256 x 50,000 151, 147).
    const bool kept = forward && backward && !several && !in_two && (d.hidden >= 640 || d.rows * ld_dz * 2 <= 40 << 20) && product_keeps(z, ctx->num_sms);
    const size_t at_dz = backward ? parts.take(size_t(dz_rows) * ld_dz * 2) : 0;
    const size_t at_acc = backward && several && d_dh ? parts.take(size_t(d.rows) * ld_copy * 4) : 0;
    size_t sums = 0;
    auto gradient_products = [&](int64_t first, int64_t n, ProductArgs &h, ProductArgs &w) {
        h = ProductArgs{}; w = ProductArgs{};
        h.dtype = w.dtype = d.dtype;
        h.status = w.status = ctx->d_status;
        h.m = dz_rows; h.n = d.hidden; h.k = n;
        h.fold = in_two ? int(d.rows) : 0;
        h.a.along_k = 1;
        h.beside = w.beside = true;
        h.ld_out = d.ld_h; h.ld_acc = ld_copy;
        h.b = Operand{static_cast<const char *>(weight.p) + (by_output ? first * weight.ld : first) * 2, weight.ld, !by_output};
        h.out = d_dh;
        h.wide = wide16(d_dh, d.ld_h) ? WIDE_OUT : 0;
        w.k = dz_rows;
        w.ld_out = d.ld_w;
        w.wide = wide16(d_dw, d.ld_w) ? WIDE_OUT : 0;
        if (by_output) { w.m = n; w.n = d.hidden; w.out = static_cast<char *>(d_dw) + first * d.ld_w * 2; }
        else { w.m = d.hidden; w.n = n; w.out = static_cast<char *>(d_dw) + first * 2; }
    };
    if (backward) {
        for (const int64_t n : {piece, (d.vocab - 1) % piece + 1}) {
            ProductArgs g[2];
            gradient_products(0, n, g[0], g[1]);
            const size_t need = d_dh && d_dw ? plan_products(PRODUCT_OUT, g, 2, ctx->num_sms) : plan_products(PRODUCT_OUT, d_dh ? g : g + 1, 1, ctx->num_sms);
            sums = need > sums ? need : sums;
        }
    }
    const size_t at_sums = parts.take(sums * sizeof(float));
    if ((rc = scratch(ctx, parts.used))) return rc;

    HeadPrepArgs pre = {};
    pre.rows = d.rows; pre.ld_h = d.ld_h; pre.ld_copy = ld_copy; pre.hidden = d.hidden; pre.vocab = d.vocab; pre.dtype = d.dtype;
    pre.h = d_h; pre.label = d_label; pre.dloss = d_dloss; pre.twice = in_two;
    if (copied) { pre.copy = part<void>(ctx, at_copy); hidden = Operand{pre.copy, ld_copy, 1}; }
    if (backward) {
        pre.scale = part<float>(ctx, at_scale);
        CUDA_TRY(ctx, launch_head_prep(pre, ctx->num_sms, ctx->stream), "launch head_prep");
    }
    LayOutArgs lay = {};
    lay_out(ctx, lay, laid, weight);
    if (!copied) lay_out(ctx, lay, laid_h, hidden);
    CUDA_TRY(ctx, launch_lay_out(lay, ctx->num_sms, ctx->stream), "launch lay_out");
    z.a = hidden;
    if (forward) {
        z.b = weight;
        z.stats = part<float2>(ctx, at_stats); z.at_label = part<float>(ctx, at_label);
        if (kept) { z.out = part<void>(ctx, at_dz); z.ld_out = ld_dz; }
        plan_products(PRODUCT_STATS, &z, 1, ctx->num_sms);
        CUDA_TRY(ctx, launch_products(PRODUCT_STATS, &z, 1, nullptr, ctx->num_sms, ctx->stream), "launch product (logits)");
        HeadFinishArgs f = {};
        f.rows = d.rows; f.vocab = d.vocab; f.tiles = int(tiles);
        f.label = d_label; f.stats = z.stats; f.at_label = z.at_label; f.loss = d_loss; f.lse = d_lse;
        if (backward) { f.base = part<float>(ctx, at_base); f.rest = part<float>(ctx, at_rest); }
        CUDA_TRY(ctx, launch_head_finish(f, ctx->num_sms, ctx->stream), "launch head_finish");
    }
    if (!backward) return RUBICK_OK;
    z.base = forward ? part<float>(ctx, at_base) : d_lse_in;
    z.rest = forward ? part<float>(ctx, at_rest) : nullptr;
    z.dloss = d_dloss; z.up = pre.scale + 1; z.in_two = in_two;
    for (int64_t first = 0; first < d.vocab; first += piece) {
        const int64_t n = first + piece < d.vocab ? piece : d.vocab - first;
        ProductArgs g[2], &h = g[0], &w = g[1];
        gradient_products(first, n, h, w);
        z.n = n; z.first = int32_t(first);
        z.b = Operand{h.b.p, weight.ld, by_output};
        z.out = part<void>(ctx, at_dz); z.ld_out = ld_dz;
        if (kept) {
            HeadScaleArgs k = {};
            k.rows = d.rows; k.ld = ld_dz; k.vocab = d.vocab; k.dtype = d.dtype; k.unit = z.way.cols / 2;
            k.label = d_label; k.stats = z.stats; k.at_label = z.at_label; k.base = z.base; k.rest = z.rest; k.dloss = d_dloss; k.up = z.up; k.dz = z.out;
            CUDA_TRY(ctx, launch_head_scale(k, ctx->num_sms, ctx->stream), "launch head_scale");
        } else {
            plan_products(PRODUCT_GRAD, &z, 1, ctx->num_sms);
            CUDA_TRY(ctx, launch_products(PRODUCT_GRAD, &z, 1, nullptr, ctx->num_sms, ctx->stream), "launch product (logits' gradient)");
        }
        h.scale = w.scale = pre.scale;
        h.a = Operand{z.out, ld_dz, 1};
        const Operand dz = {z.out, ld_dz, 0}, copy = {pre.copy, ld_copy, 0};
        w.a = by_output ? dz : copy;
        w.b = by_output ? copy : dz;
        if (several && d_dh) {
            if (first) h.acc_in = part<float>(ctx, at_acc);
            if (first + n < d.vocab) h.acc_out = part<float>(ctx, at_acc);
        }
        ProductArgs *const which = d_dh ? g : g + 1;
        const int products = d_dh && d_dw ? 2 : 1;
        plan_products(PRODUCT_OUT, which, products, ctx->num_sms);
        CUDA_TRY(ctx, launch_products(PRODUCT_OUT, which, products, part<float>(ctx, at_sums), ctx->num_sms, ctx->stream), "launch products (gradients)");
    }
    return RUBICK_OK;
}

int check_head_call(rubick_ctx *ctx, const void *h, const void *w, const int32_t *label)
{
    if (!h || !w || !label) return fail(ctx, RUBICK_EINVAL, "head loss: null pointer");
    if (!on(h, 2) || !on(w, 2) || !on(label, 4)) return fail(ctx, RUBICK_EINVAL, "head loss: a tensor is not aligned to its type");
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

int rubick_linear_forward(rubick_ctx *ctx, const rubick_linear_desc *h_desc, const void *d_x, const void *d_w,
                          const void *d_bias, const void *d_residual, const uint64_t *d_seed, void *d_pre, void *d_out)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_linear(ctx, h_desc, d_seed);
    if (rc) return rc;
    const rubick_linear_desc &d = *h_desc;
    const bool by_output = d.flags & RUBICK_WEIGHT_BY_OUTPUT;
    if (d.ld_x < d.inputs || !weight_distance(d.ld_w, by_output, d.inputs, d.outputs) || d.ld_out < d.outputs || (d_residual && d.ld_res < d.outputs) || (d_pre && d.ld_pre < d.outputs))
        return fail(ctx, RUBICK_EINVAL, "linear: a row distance is too small");
    if (d.rows == 0) return RUBICK_OK;
    if (!d_x || !d_w || !d_out) return fail(ctx, RUBICK_EINVAL, "linear: null pointer");
    if (!on(d_x, 2) || !on(d_w, 2) || !on(d_bias, esize(d.btype)) || !on(d_residual, 2) || !on(d_pre, 2) || !on(d_out, 2))
        return fail(ctx, RUBICK_EINVAL, "linear: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    ProductArgs a = {};
    a.m = d.rows; a.n = d.outputs; a.k = d.inputs; a.dtype = d.dtype; a.status = ctx->d_status;
    a.a = Operand{d_x, d.ld_x, 1};
    a.b = Operand{d_w, d.ld_w, by_output};
    a.out = d_out; a.ld_out = d.ld_out; a.pre = d_pre; a.ld_pre = d.ld_pre; a.residual = d_residual; a.ld_res = d.ld_res;
    a.bias = d_bias; a.bias_f32 = d.btype == RUBICK_F32; a.act = d.activation;
    a.wide = (wide16(d_out, d.ld_out) ? WIDE_OUT : 0) | (wide16(d_pre, d.ld_pre) ? WIDE_PRE : 0) | (wide16(d_residual, d.ld_res) ? WIDE_RES : 0) |
             (train::aligned16(d_bias) ? WIDE_BIAS : 0);
    a.drop = drop_args(d.p, d_seed);
    Parts parts;
    const Laid x = plan_operand(parts, a.a, d.rows, d.inputs), w = plan_operand(parts, a.b, by_output ? d.outputs : d.inputs, by_output ? d.inputs : d.outputs);
    const size_t at_sums = parts.take(plan_products(PRODUCT_OUT, &a, 1, ctx->num_sms) * sizeof(float));
    if ((rc = scratch(ctx, parts.used))) return rc;
    LayOutArgs lay = {};
    lay_out(ctx, lay, x, a.a);
    lay_out(ctx, lay, w, a.b);
    CUDA_TRY(ctx, launch_lay_out(lay, ctx->num_sms, ctx->stream), "launch lay_out");
    CUDA_TRY(ctx, launch_products(PRODUCT_OUT, &a, 1, part<float>(ctx, at_sums), ctx->num_sms, ctx->stream), "launch linear_forward");
    return RUBICK_OK;
}

int rubick_linear_backward(rubick_ctx *ctx, const rubick_linear_desc *h_desc, const void *d_x, const void *d_w,
                           const void *d_pre, const uint64_t *d_seed, const void *d_dout, void *d_dx, void *d_dw,
                           float *d_dbias)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_linear(ctx, h_desc, d_seed);
    if (rc) return rc;
    const rubick_linear_desc &d = *h_desc;
    const bool by_output = d.flags & RUBICK_WEIGHT_BY_OUTPUT, act = d.activation != RUBICK_ACT_NONE;
    if (((d_dx || d_dw) && (d.ld_x < d.inputs || !weight_distance(d.ld_w, by_output, d.inputs, d.outputs))) || d.ld_out < d.outputs || (act && d.ld_pre < d.outputs))
        return fail(ctx, RUBICK_EINVAL, "linear: a row distance is too small");
    if (!on(d_dw, 2) || !on(d_dbias, 4)) return fail(ctx, RUBICK_EINVAL, "linear: a tensor is not aligned to its type");
    if (d.rows == 0) {
        if ((rc = set_device(ctx))) return rc;
        const int32_t wide = by_output ? d.inputs : d.outputs, high = by_output ? d.outputs : d.inputs;
        if (d_dw) CUDA_TRY(ctx, cudaMemset2DAsync(d_dw, size_t(d.ld_w) * 2, 0, size_t(wide) * 2, high, ctx->stream), "clear dw");
        if (d_dbias) CUDA_TRY(ctx, cudaMemsetAsync(d_dbias, 0, size_t(d.outputs) * 4, ctx->stream), "clear dbias");
        return RUBICK_OK;
    }
    if (!d_dout || (act && !d_pre) || (d_dx && !d_w) || (d_dw && !d_x)) return fail(ctx, RUBICK_EINVAL, "linear: null pointer");
    if (!on(d_x, 2) || !on(d_w, 2) || !on(d_pre, 2) || !on(d_dout, 2) || !on(d_dx, 2)) return fail(ctx, RUBICK_EINVAL, "linear: a tensor is not aligned to its type");
    if (!d_dx && !d_dw && !d_dbias) return RUBICK_OK;
    if ((rc = set_device(ctx))) return rc;
    // dz is dout itself where nothing lies between them and the products can read it as it lies
    const bool products = d_dx || d_dw, plain = !act && d.p == 0.f && wide16(d_dout, d.ld_out);
    LinearGradArgs g = {};
    g.rows = d.rows; g.ld_dout = d.ld_out; g.ld_pre = d.ld_pre; g.ld_dz = up8(d.outputs); g.cols = d.outputs; g.dtype = d.dtype; g.act = d.activation;
    g.dout = d_dout; g.pre = d_pre; g.drop = drop_args(d.p, d_seed); g.dbias = d_dbias;
    plan_linear_grad(g, ctx->num_sms);
    Parts parts;
    const bool keep = products && !plain;
    const size_t at_dz = keep ? parts.take(size_t(d.rows) * g.ld_dz * 2) : 0;
    const size_t at_columns = d_dbias ? parts.take(size_t(g.chunks) * d.outputs * 4) : 0;
    ProductArgs both[2] = {}, &dx = both[0], &dw = both[1];
    dx.dtype = dw.dtype = d.dtype;
    dx.status = dw.status = ctx->d_status;
    dx.m = d.rows; dx.n = d.inputs; dx.k = d.outputs;
    dx.a.along_k = 1;
    dx.beside = dw.beside = true;
    dx.out = d_dx; dx.ld_out = d.ld_x; dx.wide = wide16(d_dx, d.ld_x) ? WIDE_OUT : 0;
    dx.b = Operand{d_w, d.ld_w, !by_output};
    dw.m = by_output ? d.outputs : d.inputs; dw.n = by_output ? d.inputs : d.outputs; dw.k = d.rows;
    dw.out = d_dw; dw.ld_out = d.ld_w; dw.wide = wide16(d_dw, d.ld_w) ? WIDE_OUT : 0;
    Operand x = {d_x, d.ld_x, 0};
    const Laid laid_x = d_dw ? plan_operand(parts, x, d.rows, d.inputs) : Laid{}, laid_w = d_dx ? plan_operand(parts, dx.b, by_output ? d.outputs : d.inputs, by_output ? d.inputs : d.outputs) : Laid{};
    ProductArgs *const which = d_dx ? both : both + 1;
    const int n_products = d_dx && d_dw ? 2 : 1;
    const size_t at_sums = products ? parts.take(plan_products(PRODUCT_OUT, which, n_products, ctx->num_sms) * sizeof(float)) : 0;
    if ((rc = scratch(ctx, parts.used))) return rc;
    if (keep) g.dz = part<void>(ctx, at_dz);
    if (d_dbias) g.part = part<float>(ctx, at_columns);
    if (d_dbias && g.chunks > 1) {
        if ((rc = tickets(ctx, size_t(g.strips)))) return rc;
        g.tickets = ctx->d_tickets;
    }
    if (keep || d_dbias) CUDA_TRY(ctx, launch_linear_grad(g, ctx->num_sms, ctx->stream), "launch linear_grad");
    LayOutArgs lay = {};
    if (d_dw) lay_out(ctx, lay, laid_x, x);
    if (d_dx) lay_out(ctx, lay, laid_w, dx.b);
    CUDA_TRY(ctx, launch_lay_out(lay, ctx->num_sms, ctx->stream), "launch lay_out");
    const void *dz = keep ? g.dz : d_dout;
    const int64_t ld_dz = keep ? g.ld_dz : d.ld_out;
    dx.a = Operand{dz, ld_dz, 1};
    const Operand z = {dz, ld_dz, 0};
    dw.a = by_output ? z : x;
    dw.b = by_output ? x : z;
    if (products) CUDA_TRY(ctx, launch_products(PRODUCT_OUT, which, n_products, part<float>(ctx, at_sums), ctx->num_sms, ctx->stream), "launch products (gradients)");
    return RUBICK_OK;
}

static int dropout(rubick_ctx *ctx, const rubick_dropout_desc *h_desc, const uint64_t *d_seed, const void *d_x, const void *d_residual, void *d_out, bool back)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_dropout(ctx, h_desc, d_seed);
    if (rc) return rc;
    if (d_residual && h_desc->ld_res < h_desc->cols) return fail(ctx, RUBICK_EINVAL, "dropout: a row distance is smaller than cols");
    if (h_desc->rows == 0) return RUBICK_OK;
    if (!d_x || !d_out) return fail(ctx, RUBICK_EINVAL, "dropout: null pointer");
    const int es = esize(h_desc->dtype);
    if (!on(d_x, es) || !on(d_residual, es) || !on(d_out, es)) return fail(ctx, RUBICK_EINVAL, "dropout: a tensor is not aligned to its type");
    if ((rc = set_device(ctx))) return rc;
    DropoutArgs a = {};
    a.d = *h_desc;
    if (back) { a.d.ld_x = h_desc->ld_out; a.d.ld_out = h_desc->ld_x; }      // dout lies as out, dx as x
    a.x = d_x; a.residual = d_residual; a.out = d_out;
    a.drop = drop_args(h_desc->p, d_seed);
    CUDA_TRY(ctx, launch_dropout(a, ctx->num_sms, ctx->stream), "launch dropout");
    return RUBICK_OK;
}

int rubick_dropout_forward(rubick_ctx *ctx, const rubick_dropout_desc *h_desc, const uint64_t *d_seed, const void *d_x,
                           const void *d_residual, void *d_out)
{
    return dropout(ctx, h_desc, d_seed, d_x, d_residual, d_out, false);
}

int rubick_dropout_backward(rubick_ctx *ctx, const rubick_dropout_desc *h_desc, const uint64_t *d_seed, const void *d_dout,
                            void *d_dx)
{
    return dropout(ctx, h_desc, d_seed, d_dout, nullptr, d_dx, true);
}

int rubick_head_loss_forward(rubick_ctx *ctx, const rubick_head_loss_desc *h_desc, const void *d_h, const void *d_w,
                             const int32_t *d_label, float *d_loss, float *d_lse)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_head(ctx, h_desc);
    if (rc) return rc;
    if (h_desc->rows == 0) return RUBICK_OK;
    if ((rc = check_head_call(ctx, d_h, d_w, d_label))) return rc;
    if (!d_loss) return fail(ctx, RUBICK_EINVAL, "head loss: null pointer");
    if (!on(d_loss, 4) || !on(d_lse, 4)) return fail(ctx, RUBICK_EINVAL, "head loss: a tensor is not aligned to its type");
    return head_loss(ctx, h_desc, d_h, d_w, d_label, nullptr, nullptr, d_loss, d_lse, nullptr, nullptr, true, false);
}

int rubick_head_loss_backward(rubick_ctx *ctx, const rubick_head_loss_desc *h_desc, const void *d_h, const void *d_w,
                              const int32_t *d_label, const float *d_lse, const float *d_dloss, void *d_dh, void *d_dw)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_head(ctx, h_desc);
    if (rc) return rc;
    if (!on(d_dh, 2) || !on(d_dw, 2) || !on(d_lse, 4) || !on(d_dloss, 4)) return fail(ctx, RUBICK_EINVAL, "head loss: a tensor is not aligned to its type");
    if (h_desc->rows) {
        if ((rc = check_head_call(ctx, d_h, d_w, d_label))) return rc;
        if (!d_lse) return fail(ctx, RUBICK_EINVAL, "head loss: null pointer");
    }
    if (!d_dh && !d_dw) return RUBICK_OK;
    return head_loss(ctx, h_desc, d_h, d_w, d_label, d_lse, d_dloss, nullptr, nullptr, d_dh, d_dw, false, true);
}

int rubick_head_loss_step(rubick_ctx *ctx, const rubick_head_loss_desc *h_desc, const void *d_h, const void *d_w,
                          const int32_t *d_label, const float *d_dloss, float *d_loss, float *d_lse, void *d_dh, void *d_dw)
{
    if (!ctx) return RUBICK_EINVAL;
    int rc = check_head(ctx, h_desc);
    if (rc) return rc;
    if (!on(d_dh, 2) || !on(d_dw, 2) || !on(d_loss, 4) || !on(d_lse, 4) || !on(d_dloss, 4)) return fail(ctx, RUBICK_EINVAL, "head loss: a tensor is not aligned to its type");
    if (h_desc->rows) {
        if ((rc = check_head_call(ctx, d_h, d_w, d_label))) return rc;
        if (!d_loss) return fail(ctx, RUBICK_EINVAL, "head loss: null pointer");
    }
    return head_loss(ctx, h_desc, d_h, d_w, d_label, nullptr, d_dloss, d_loss, d_lse, d_dh, d_dw, true, d_dh || d_dw);
}

}  // extern "C"
