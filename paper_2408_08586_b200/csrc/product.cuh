// What the matrix products of a training step share: operands, the counter-based generator, activations, and what is done
// with eight neighbouring sums of a row.
#pragma once

#include "train_common.cuh"

namespace rubick {

// One operand of D[m][n] = sum_k A[m][k] B[n][k]: [dim][k] with the k next to each other (along_k), or [k][dim].
struct Operand { const void *p; int64_t ld; int along_k; };

struct DropArgs { const uint64_t *seed; uint32_t below; float scale; };     // kept: word >= below, times scale; seed NULL: no dropout

enum ProductKind { PRODUCT_OUT, PRODUCT_STATS, PRODUCT_GRAD };

// How a product is cut: into which tiles, how many blocks of a cluster share one's k, into how many parts the k are dealt out
// besides.
struct ProductWay { int shape, cols, share, splits; float cost; int64_t blocks; };

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
    // with way.splits > 1 the sums of each part of the k lie in part[split][m][ld_acc] until they are joined
    float *part;
    size_t part_at;                      // where they begin in the launch's scratch, in floats
    ProductWay way;
    bool beside;                         // one of the two gradients of a product
    int fold;                            // rows fold .. 2 fold - 1 are added to the first ones (0: they are rows like others)
    // PRODUCT_STATS, PRODUCT_GRAD: the logits of vocabulary first .. first + n - 1; with `out`, PRODUCT_STATS keeps there the
    // exponentials of their distances to their pair's maximum, times KEPT
    const int32_t *label;
    int32_t first, vocab;
    float2 *stats;                       // [product_stats_pairs][m]: maximum, sum of exponentials
    float *at_label;                     // [m] logit of the label
    const float *base, *rest;            // log of the row's sum of exponentials, in two parts (rest may be NULL)
    const float *dloss, *up;             // [m] weight of a row (NULL: 1), and the weights' common factor
    bool in_two;                         // PRODUCT_GRAD writes m more rows: what the first ones lack by their rounding
    uint32_t *status;
};
enum { WIDE_OUT = 1, WIDE_PRE = 2, WIDE_RES = 4, WIDE_BIAS = 8 };

constexpr float KEPT = 16384.f;          // (so that half precision holds those of 2^-28 and more to 11 bits)

struct DropoutArgs {
    rubick_dropout_desc d;
    const void *x, *residual;
    void *out;
    DropArgs drop;
    int chunks;                          // runs of rows
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
    uint32_t *tickets;                   // [strips] arrivals, zero between calls
    int chunks, strips;                  // of rows, of columns
    int lanes;                           // lanes of a warp that share a row (a power of two); the others take further rows
};
// rows of h whose label takes part (zeros for the others), next to each other; the weights' common factor
struct HeadPrepArgs {
    int64_t rows, ld_h, ld_copy;
    int hidden, vocab, dtype;
    const void *h;
    const int32_t *label;
    const float *dloss;
    void *copy;
    bool twice;                          // the copy's rows once more behind them
    float *scale;                        // the factor's reciprocal, the factor
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

struct LayOutArgs {
    struct One { const void *from; int64_t ld_from; void *to; int64_t ld_to, rows, cols; } one[2];
    int n;
};

// Up to two products of one launch (two only for PRODUCT_OUT without activations): how they are cut, which goes by their sizes
// and by how their operands lie (along_k has to be there already), and the floats of scratch that this takes.
size_t plan_products(ProductKind kind, ProductArgs *a, int n, int num_sms);
cudaError_t launch_products(ProductKind kind, ProductArgs *a, int n, float *part, int num_sms, cudaStream_t st);
bool product_few(int64_t rows);                                      // whether PRODUCT_GRAD can write that many rows in two
bool product_keeps(const ProductArgs &a, int num_sms);               // whether PRODUCT_STATS can keep the exponentials
int64_t product_stats_pairs(const ProductArgs &a, int num_sms);      // pairs (maximum, sum) of a row that the logits come in
bool product_takes(const Operand &o);                            // as it lies, that is
cudaError_t launch_lay_out(const LayOutArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_dropout(const DropoutArgs &a, int num_sms, cudaStream_t st);
void plan_linear_grad(LinearGradArgs &a, int num_sms);
cudaError_t launch_linear_grad(const LinearGradArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_head_prep(const HeadPrepArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_head_finish(const HeadFinishArgs &a, int num_sms, cudaStream_t st);
// kept exponentials become dz where they lie
struct HeadScaleArgs {
    int64_t rows, ld;
    int vocab, dtype, unit;              // columns of a pair
    const int32_t *label;
    const float2 *stats;
    const float *at_label, *base, *rest, *dloss, *up;
    void *dz;
};
cudaError_t launch_head_scale(const HeadScaleArgs &a, int num_sms, cudaStream_t st);

// A launch that may begin while the one before it in the stream ends: its kernel waits (chain_wait) before it touches memory.
template <typename... P, typename... A> cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    count_launch();
    return e;
}

namespace train {

// The next launch may begin; everything before this one is over.
__device__ __forceinline__ void chain_go() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- dropout: Philox4x32-10 (Salmon et al., SC 2011), the four words of a counter under a key -------------------------
// A round takes (c0, c1, c2, c3) to (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)).  The counter is (column / 4,
// row, offset), so what of its first three rounds does not depend on the row is worked out once for a thread's columns:
// of the 20 products of a counter 15 are left to each row, and one for all of a row's counters.
struct Drop {
    uint64_t seed, offset;
    uint32_t below;
    float scale;
    bool on;
    __device__ __forceinline__ explicit Drop(const DropArgs &a) : seed(0), offset(0), below(a.below), scale(a.scale), on(a.seed != nullptr)
    {
        if (on) { seed = a.seed[0]; offset = a.seed[1]; }
    }
};
template <int VE> struct DropColumns {
    static_assert(VE % 4 == 0, "a counter serves four columns");
    static constexpr uint32_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u, W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
    uint32_t k0, k1, row_key, below;
    uint32_t second[VE / 4], third[VE / 4], fourth[VE / 4], fifth[VE / 4];
    __device__ __forceinline__ static uint32_t hi(uint64_t v) { return uint32_t(v >> 32); }
    __device__ __forceinline__ static uint32_t lo(uint64_t v) { return uint32_t(v); }
    // from column c on (a multiple of four)
    __device__ __forceinline__ DropColumns(const Drop &d, int c) : k0(uint32_t(d.seed)), k1(uint32_t(d.seed >> 32)), below(d.below)
    {
        const uint64_t b1 = uint64_t(M1) * uint32_t(d.offset);
        row_key = hi(b1) ^ k0;                                         // round 1: c0 = row ^ row_key
#pragma unroll
        for (int q = 0; q < VE / 4; ++q) {
            const uint64_t a1 = uint64_t(M0) * (uint32_t(c) / 4 + q);
            const uint32_t c2 = hi(a1) ^ uint32_t(d.offset >> 32) ^ k1, c3 = lo(a1);
            second[q] = c3 ^ (k1 + W1);                                // round 2: c2 = hi(M0 c0) ^ second, c3 = lo(M0 c0)
            const uint64_t b2 = uint64_t(M1) * c2;
            const uint32_t c0 = hi(b2) ^ lo(b1) ^ (k0 + W0);
            third[q] = lo(b2) ^ (k0 + 2 * W0);                         // round 3: c0 = hi(M1 c2) ^ third, c1 = lo(M1 c2)
            const uint64_t a3 = uint64_t(M0) * c0;
            fourth[q] = hi(a3) ^ (k1 + 2 * W1);                        //          c2 = c3 ^ fourth
            fifth[q] = lo(a3);                                         //          c3
        }
    }
    // 0 where an element of the row is dropped; the others still lack their factor
    __device__ __forceinline__ void choose(uint32_t row, float (&v)[VE]) const
    {
        const uint64_t a2 = uint64_t(M0) * (row ^ row_key);
#pragma unroll
        for (int q = 0; q < VE / 4; ++q) {
            const uint64_t b3 = uint64_t(M1) * (hi(a2) ^ second[q]);
            uint32_t c0 = hi(b3) ^ third[q], c1 = lo(b3), c2 = lo(a2) ^ fourth[q], c3 = fifth[q];
#pragma unroll
            for (uint32_t i = 3; i < 10; ++i) {
                const uint64_t a = uint64_t(M0) * c0, b = uint64_t(M1) * c2;
                c0 = hi(b) ^ c1 ^ (k0 + i * W0); c1 = lo(b);
                c2 = hi(a) ^ c3 ^ (k1 + i * W1); c3 = lo(a);
            }
            v[4 * q] = c0 >= below ? v[4 * q] : 0.f; v[4 * q + 1] = c1 >= below ? v[4 * q + 1] : 0.f;
            v[4 * q + 2] = c2 >= below ? v[4 * q + 2] : 0.f; v[4 * q + 3] = c3 >= below ? v[4 * q + 3] : 0.f;
        }
    }
};

// ---- activations -------------------------------------------------------------------------------------------------
// The hardware's exponential and reciprocal, subnormal numbers taken as zero (with them kept, each costs three instructions
// more, for results that are rounded to 16 bits or summed with larger ones).
constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float ex2(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float rcp(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
// v / (1 + exp(-u)): where the exponential overflows the reciprocal is the right 0
__device__ __forceinline__ float over_one_plus_exp(float v, float u) { return v * rcp(1.f + ex2(-LOG2E * u)); }
__device__ __forceinline__ float tanh_arg2(float v) { return 1.5957691216057308f * (v + 0.044715f * v * v * v); }   // 2 sqrt(2 / pi) ..
// Phi(v), the normal distribution's integral, and exp(-v^2 / 2): erfc(x) = (a1 t + .. + a5 t^5) exp(-x^2), t = 1 / (1 + p x),
// x = |v| / sqrt(2) (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26: off by 1.5e-7 at most).  The
// exponential is the one that the slope needs as well, and on the far left nothing cancels, as in 1 + erf.
__device__ __forceinline__ float normal_integral(float v, float &bell)
{
    const float x = fabsf(v) * 0.70710678118654752f, t = rcp(fmaf(0.3275911f, x, 1.f));
    bell = ex2(-0.5f * LOG2E * v * v);
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float tail = 0.5f * p * bell;
    return v > 0.f ? 1.f - tail : tail;
}
__device__ __forceinline__ float act_value(int act, float v)
{
    float bell;
    switch (act) {
    case RUBICK_ACT_RELU: return v > 0.f ? v : (v != v ? v : 0.f);
    case RUBICK_ACT_GELU: return v * normal_integral(v, bell);
    case RUBICK_ACT_GELU_TANH: return over_one_plus_exp(v, tanh_arg2(v));          // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
    case RUBICK_ACT_SILU: return over_one_plus_exp(v, v);
    }
    return v;
}
__device__ __forceinline__ float act_slope(int act, float v)
{
    float bell;
    switch (act) {
    case RUBICK_ACT_RELU: return v > 0.f ? 1.f : (v != v ? v : 0.f);
    case RUBICK_ACT_GELU: {
        const float phi = normal_integral(v, bell);
        return fmaf(v * 0.3989422804014327f, bell, phi);
    }
    // with s = 1 / (1 + exp(-u)), 1 - s (off by half a step of one, in products with what stays below one)
    case RUBICK_ACT_GELU_TANH: {
        const float s = over_one_plus_exp(1.f, tanh_arg2(v));
        return s + s * (1.f - s) * v * 1.5957691216057308f * (1.f + 0.134145f * v * v);
    }
    case RUBICK_ACT_SILU: {
        const float s = over_one_plus_exp(1.f, v);
        return s * (1.f + v * (1.f - s));
    }
    }
    return 1.f;
}

// 16 bytes of a row from column c on, whatever its alignment: the two aligned pieces that hold them, asked for in one step and
// shifted in another, where both lie within the row; else element by element (0 past the end).  WIDE: every row begins on a
// 16-byte boundary, and one piece is all.
template <bool WIDE> struct Pieces { uint4 a, b; };
template <> struct Pieces<true> { uint4 a; };
template <typename T, typename I> __device__ __forceinline__ bool two_pieces(const T *at, I c, I n, uint32_t &off)
{
    off = uint32_t(reinterpret_cast<uintptr_t>(at)) & 15;
    const I before = I(off / uint32_t(sizeof(T)));
    return c >= before && c - before + 2 * Lanes<T>::N <= n;
}
template <bool WIDE, typename T, typename I> __device__ __forceinline__ Pieces<WIDE> ask(const T *row, I c, I n)
{
    constexpr int N = Lanes<T>::N;
    const T *const at = row + c;
    Pieces<WIDE> p;
    if constexpr (WIDE) {
        if (c + N <= n) { p.a = ld_stream(at); return p; }
    } else {
        uint32_t off;
        if (two_pieces(at, c, n, off)) {
            const uint8_t *const from = reinterpret_cast<const uint8_t *>(at) - off;
            p.a = ld_cached(from);
            p.b = ld_cached(from + 16);
            return p;
        }
        p.b = uint4{};
    }
    uint32_t w[4] = {};
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (c + e < n) {
            if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(at[e]);
            else w[e >> 1] |= uint32_t(reinterpret_cast<const uint16_t *>(at)[e]) << (16 * (e & 1));
        }
    }
    p.a = make_uint4(w[0], w[1], w[2], w[3]);
    return p;
}
template <bool WIDE, typename T, typename I> __device__ __forceinline__ uint4 take(const T *row, I c, I n, const Pieces<WIDE> &p)
{
    if constexpr (WIDE) return p.a;
    else {
        uint32_t off;
        if (!two_pieces(row + c, c, n, off)) return p.a;
        const uint4 &a = p.a, &b = p.b;
        const bool four = off & 4, eight = off & 8;
        // 32 bytes moved down by eight, then four, then what is left below four
        const uint32_t u0 = eight ? a.z : a.x, u1 = eight ? a.w : a.y, u2 = eight ? b.x : a.z, u3 = eight ? b.y : a.w, u4 = eight ? b.z : b.x, u5 = eight ? b.w : b.y;
        const uint32_t w0 = four ? u1 : u0, w1 = four ? u2 : u1, w2 = four ? u3 : u2, w3 = four ? u4 : u3, w4 = four ? u5 : u4;
        if constexpr (sizeof(T) == 4) return make_uint4(w0, w1, w2, w3);
        const uint32_t bits = (off & 2) * 8;
        return make_uint4(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits), __funnelshift_r(w2, w3, bits), __funnelshift_r(w3, w4, bits));
    }
}
template <typename T, typename I> __device__ __forceinline__ uint4 load_any(const T *row, I c, I n) { return take<false>(row, c, n, ask<false>(row, c, n)); }

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
    // the sum so far; true: that is all there is to do
    __device__ __forceinline__ bool accumulate(int64_t row, int64_t c, float (&v)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        if (acc_in) {
            float s[8];
            load8<float>(acc_in + row * ld_acc, c, ld_acc, true, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += s[e];
        }
        if (acc_out) store8<float>(acc_out + row * ld_acc, c, ld_acc, true, v);
        return acc_out != nullptr;
    }
    __device__ __forceinline__ void activate(int64_t row, int64_t c, float (&v)[8]) const
    {
        if constexpr (ACT != RUBICK_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = act_value(ACT, v[e]);
        }
        if (drop.on) {
            DropColumns<8>(drop, int(c)).choose(uint32_t(row), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= drop.scale;
        }
    }
    // the residual of eight columns, 0 without one
    __device__ __forceinline__ void load_residual(int64_t row, int64_t c, float (&r)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = 0.f;
        if (residual && !acc_out) load8<T>(residual + row * ld_res, c, n, wide & WIDE_RES, r);
    }
    __device__ __forceinline__ void operator()(int64_t row, int64_t c, float (&v)[8], const float (&b)[8], const float (&r)[8]) const
    {
        if (accumulate(row, c, v)) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += b[e];
        if (pre) store8<T>(pre + row * ld_pre, c, n, wide & WIDE_PRE, v);
        activate(row, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r[e];
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
            const DropColumns<8> columns(drop, int(c));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                columns.choose(uint32_t(row + 8 * r), v[r]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[r][e] *= drop.scale;
            }
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
    // whether there is nothing to fetch or keep for a row's sums: a thread may then finish a whole row of 64
    __device__ __forceinline__ bool takes_rows() const { return !acc_in && !acc_out && !pre && !residual && !drop.on && (wide & WIDE_OUT); }
    // whether a whole block of 32 rows x 32 columns may go that way
    __device__ __forceinline__ bool takes_four() const
    {
        return !acc_in && !acc_out && (wide & WIDE_OUT) && (!pre || (wide & WIDE_PRE)) && (!residual || (wide & WIDE_RES));
    }
};


}  // namespace train
}  // namespace rubick
