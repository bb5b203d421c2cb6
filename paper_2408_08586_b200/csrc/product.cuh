// What the matrix products of a training step share: operands, the counter-based generator, activations, and what is done
// with eight neighbouring sums of a row.
#pragma once

#include "train_common.cuh"

namespace rubick {

// One operand of D[m][n] = sum_k A[m][k] B[n][k]: [dim][k] with the k next to each other (along_k), or [k][dim].
struct Operand { const void *p; int64_t ld; int along_k; };

struct DropArgs { const uint64_t *seed; uint32_t below; float scale; };     // kept: word >= below, times scale; seed NULL: no dropout

enum ProductKind { PRODUCT_OUT, PRODUCT_PART, PRODUCT_STATS, PRODUCT_GRAD };

struct ProductArgs {
    int64_t m, n, k;
    Operand a, b;
    int dtype;
    // PRODUCT_OUT: out = residual + drop(act(sum * scale + acc_in + bias)); with acc_out the sum goes there instead
    void *out, *pre;
    const void *bias, *residual;
    int64_t ld_out, ld_pre, ld_res, ld_acc;
    int bias_f32, act;
    int wide;                            // bit i: out / pre / residual / bias may be accessed 16 bytes at a time
    DropArgs drop;
    const float *scale;                  // one float in device memory, or NULL
    const float *acc_in; float *acc_out; // single-precision sums of earlier pieces, and of this and the earlier ones
    // PRODUCT_PART: the k are dealt out to `splits`, which write their sums to part[split][m][ld_acc]
    float *part;
    int splits;
    // PRODUCT_STATS, PRODUCT_GRAD: the logits of vocabulary first .. first + n - 1
    const int32_t *label;
    int32_t first, vocab;
    float2 *stats;                       // [ceil(n / product_stats_cols)][m]
    float *at_label;                     // [m] logit of the label
    const float *base, *rest;            // log of the row's sum of exponentials, in two parts (rest may be NULL)
    const float *weight;                 // [m] weight of a row times the common power of two
    uint32_t *status;
};
enum { WIDE_OUT = 1, WIDE_PRE = 2, WIDE_RES = 4, WIDE_BIAS = 8 };

struct DropoutArgs {
    rubick_dropout_desc d;
    const void *x, *residual;
    void *out;
    DropArgs drop;
};
// dz = act'(pre) drop(dout) with its column sums
struct LinearGradArgs {
    int64_t rows, ld_dout, ld_pre, ld_dz;
    int cols, dtype, act;
    const void *dout, *pre;
    DropArgs drop;
    void *dz;                            // NULL: only the column sums are wanted
    float *dbias;                        // or NULL
    float *part;                         // [chunks][cols] sums of row chunks
    int chunks;
};
// rows of h whose label takes part (zeros for the others), next to each other; the largest weight of a row
struct HeadPrepArgs {
    int64_t rows, ld_h, ld_copy;
    int hidden, vocab, dtype;
    const void *h;
    const int32_t *label;
    const float *dloss;
    void *copy;
    float *weight;                       // [rows] weight times 2^s
    float *scale;                        // 2^-s
    uint32_t *largest;                   // bits of the largest finite |weight|
};
struct HeadFinishArgs {
    int64_t rows;
    int vocab, tiles;
    const int32_t *label;
    const float2 *stats;
    const float *at_label;
    float *loss, *lse;                   // lse may be NULL
    float *base, *rest;                  // the row's maximum and the log of its sum behind it, or NULL
};

int product_splits(const ProductArgs &a, int num_sms);           // into how many parts the k are dealt out
int product_stats_cols(const ProductArgs &a, int num_sms);       // columns of the logits that one pair (maximum, sum) covers
bool product_takes(const Operand &o);                            // as it lies, that is
cudaError_t launch_lay_out(const void *from, int64_t ld_from, void *to, int64_t ld_to, int64_t rows, int64_t cols, cudaStream_t st);
cudaError_t launch_product(ProductKind kind, const ProductArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_dropout(const DropoutArgs &a, int num_sms, cudaStream_t st);
int linear_grad_chunks(int64_t rows, int cols, int num_sms);
cudaError_t launch_linear_grad(const LinearGradArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_head_prep(const HeadPrepArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_head_finish(const HeadFinishArgs &a, int num_sms, cudaStream_t st);

namespace train {

// ---- Philox4x32-10 (Salmon et al., SC 2011): four words of a counter under a key -------------------------------------
__device__ __forceinline__ uint4 philox(uint32_t quad, uint32_t row, uint64_t seed, uint64_t offset)
{
    uint32_t c0 = quad, c1 = row, c2 = uint32_t(offset), c3 = uint32_t(offset >> 32);
    uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = uint64_t(0xD2511F53u) * c0, b = uint64_t(0xCD9E8D57u) * c2;
        c0 = uint32_t(b >> 32) ^ c1 ^ k0; c1 = uint32_t(b);
        c2 = uint32_t(a >> 32) ^ c3 ^ k1; c3 = uint32_t(a);
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
struct Drop {
    uint64_t seed, offset;
    uint32_t below;
    float scale;
    bool on;
    __device__ __forceinline__ explicit Drop(const DropArgs &a) : seed(0), offset(0), below(a.below), scale(a.scale), on(a.seed != nullptr)
    {
        if (on) { seed = a.seed[0]; offset = a.seed[1]; }
    }
    // VE elements of a row from column c (a multiple of four)
    template <int VE> __device__ __forceinline__ void apply(int64_t row, int c, float (&v)[VE]) const
    {
        static_assert(VE % 4 == 0, "a counter serves four columns");
#pragma unroll
        for (int q = 0; q < VE; q += 4) {
            const uint4 w = philox(uint32_t(c + q) >> 2, uint32_t(row), seed, offset);
            v[q] = w.x >= below ? v[q] * scale : 0.f; v[q + 1] = w.y >= below ? v[q + 1] * scale : 0.f;
            v[q + 2] = w.z >= below ? v[q + 2] * scale : 0.f; v[q + 3] = w.w >= below ? v[q + 3] * scale : 0.f;
        }
    }
};

// ---- activations -------------------------------------------------------------------------------------------------
// v / (1 + exp(-u)): where the exponential overflows the quick division gives the right 0
__device__ __forceinline__ float over_one_plus_exp(float v, float u) { return __fdividef(v, 1.f + __expf(-u)); }
__device__ __forceinline__ float tanh_arg2(float v) { return 1.5957691216057308f * (v + 0.044715f * v * v * v); }   // 2 sqrt(2 / pi) ..
__device__ __forceinline__ float act_value(int act, float v)
{
    switch (act) {
    case RUBICK_ACT_RELU: return v > 0.f ? v : (v != v ? v : 0.f);
    case RUBICK_ACT_GELU: return 0.5f * v * erfcf(-0.70710678118654752f * v);     // (1 + erf would cancel on the far left)
    case RUBICK_ACT_GELU_TANH: return over_one_plus_exp(v, tanh_arg2(v));          // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
    case RUBICK_ACT_SILU: return over_one_plus_exp(v, v);
    }
    return v;
}
__device__ __forceinline__ float act_slope(int act, float v)
{
    switch (act) {
    case RUBICK_ACT_RELU: return v > 0.f ? 1.f : (v != v ? v : 0.f);
    case RUBICK_ACT_GELU: return 0.5f * erfcf(-0.70710678118654752f * v) + v * 0.3989422804014327f * __expf(-0.5f * v * v);
    case RUBICK_ACT_GELU_TANH: {
        const float s = over_one_plus_exp(1.f, tanh_arg2(v)), r = over_one_plus_exp(1.f, -tanh_arg2(v));   // r = 1 - s
        return s + s * r * v * 1.5957691216057308f * (1.f + 0.134145f * v * v);
    }
    case RUBICK_ACT_SILU: {
        const float s = over_one_plus_exp(1.f, v), r = over_one_plus_exp(1.f, -v);
        return s * (1.f + v * r);
    }
    }
    return 1.f;
}

// Eight elements of a row from column c on (a multiple of eight), 16 bytes at a time where the tensor allows it; columns
// from n on are not touched.
template <typename T> __device__ __forceinline__ void load8(const T *row, int64_t c, int64_t n, bool wide, float (&v)[8])
{
    if (wide && c + 8 <= n) {
#pragma unroll
        for (int i = 0; i < 8; i += Lanes<T>::N) {
            float part[Lanes<T>::N];
            unpack16<T>(ld_stream(row + c + i), part);
#pragma unroll
            for (int e = 0; e < Lanes<T>::N; ++e) v[i + e] = part[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < n ? to_f(row[c + e]) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T *row, int64_t c, int64_t n, bool wide, const float (&v)[8])
{
    if (wide && c + 8 <= n) {
#pragma unroll
        for (int i = 0; i < 8; i += Lanes<T>::N) {
            float part[Lanes<T>::N];
#pragma unroll
            for (int e = 0; e < Lanes<T>::N; ++e) part[e] = v[i + e];
            *reinterpret_cast<uint4 *>(row + c + i) = pack16<T>(part);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (c + e < n) row[c + e] = from_f<T>(v[e]);
    }
}

// PRODUCT_OUT's epilogue for eight sums of a row.
template <typename T, int ACT> struct Finish {
    T *out, *pre;
    const T *residual;
    const void *bias;
    const float *acc_in;
    float *acc_out;
    int64_t ld_out, ld_pre, ld_res, ld_acc, n;
    float scale;
    int wide;
    bool bias_f32;
    Drop drop;
    __device__ __forceinline__ explicit Finish(const ProductArgs &a)
        : out(static_cast<T *>(a.out)), pre(static_cast<T *>(a.pre)), residual(static_cast<const T *>(a.residual)), bias(a.bias), acc_in(a.acc_in), acc_out(a.acc_out),
          ld_out(a.ld_out), ld_pre(a.ld_pre), ld_res(a.ld_res), ld_acc(a.ld_acc), n(a.n), scale(a.scale ? *a.scale : 1.f), wide(a.wide), bias_f32(a.bias_f32), drop(a.drop)
    {
    }
    // what every row of columns c .. c + 7 gets
    __device__ __forceinline__ void load_bias(int64_t c, float (&b)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = 0.f;
        if (!bias || acc_out) return;
        if (bias_f32) load8<float>(static_cast<const float *>(bias), c, n, wide & WIDE_BIAS, b);
        else load8<T>(static_cast<const T *>(bias), c, n, wide & WIDE_BIAS, b);
    }
    __device__ __forceinline__ void operator()(int64_t row, int64_t c, float (&v)[8], const float (&b)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        if (acc_in) {
            float s[8];
            load8<float>(acc_in + row * ld_acc, c, ld_acc, true, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += s[e];
        }
        if (acc_out) { store8<float>(acc_out + row * ld_acc, c, ld_acc, true, v); return; }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += b[e];
        if (pre) store8<T>(pre + row * ld_pre, c, n, wide & WIDE_PRE, v);
        if constexpr (ACT != RUBICK_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = act_value(ACT, v[e]);
        }
        if (drop.on) drop.apply<8>(row, int(c), v);
        if (residual) {
            float r[8];
            load8<T>(residual + row * ld_res, c, n, wide & WIDE_RES, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += r[e];
        }
        store8<T>(out + row * ld_out, c, n, wide & WIDE_OUT, v);
    }
    // The same for eight sums of four rows each, 8 rows apart, all of them within the matrix and every tensor read and written
    // 16 bytes at a time: one branch for what there is instead of one each for every eight sums (a branch costs some 20
    // cycles, and a warp has little else to do meanwhile: 550 cycles for eight sums one by one).
    __device__ __forceinline__ void four(int64_t row, int64_t c, float (&v)[4][8], const float (&b)[8]) const
    {
        uint4 res[4];
        if (residual) {
#pragma unroll
            for (int r = 0; r < 4; ++r) res[r] = ld_stream(residual + (row + 8 * r) * ld_res + c);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[r][e] = fmaf(v[r][e], scale, b[e]);
        if (pre) {
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<uint4 *>(pre + (row + 8 * r) * ld_pre + c) = pack16<T>(v[r]);
        }
        if constexpr (ACT != RUBICK_ACT_NONE) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[r][e] = act_value(ACT, v[r][e]);
        }
        if (drop.on) {
#pragma unroll
            for (int r = 0; r < 4; ++r) drop.apply<8>(row + 8 * r, int(c), v[r]);
        }
        if (residual) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float x[8];
                unpack16<T>(res[r], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[r][e] += x[e];
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) *reinterpret_cast<uint4 *>(out + (row + 8 * r) * ld_out + c) = pack16<T>(v[r]);
    }
    // whether a whole block of 32 rows x 32 columns may go that way
    __device__ __forceinline__ bool takes_four() const
    {
        return !acc_in && !acc_out && (wide & WIDE_OUT) && (!pre || (wide & WIDE_PRE)) && (!residual || (wide & WIDE_RES));
    }
};

constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float ex2(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

}  // namespace train
}  // namespace rubick
