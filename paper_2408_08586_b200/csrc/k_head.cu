// The head's cross entropy: what runs before and after the products of its logits.
//
// All of it is bound by memory or by one trip to it: head_prep copies h (2,048 x 4,096 9 us), head_finish reads 8 bytes per
// row and 64 or 128 tokens (5 to 9 us), head_scale reads and writes dz once (2,048 x 128,000 bf16 177 us, 5.9 TB/s).
#include "product.cuh"

namespace rubick {
namespace {

using namespace train;

__device__ __forceinline__ bool takes_part(int label, int vocab) { return label >= 0 && label < vocab; }

constexpr int PREP_THREADS = 1024;

// A copy of h with rows next to each other, zeros in the rows that take no part (whatever they hold must not reach the
// sums over the rows).  The first block works out the factor that makes the largest weight 2^14; it is taken out again, in
// single precision, behind the products.  In half precision the probabilities of a large vocabulary, times a weight of one
// over the rows, would mostly fall below its normal range; and the label's entry w (p - 1), the largest of most rows, comes
// to lie just below a power of two, where rounding takes least of it (gradients' distance from 64 bits: 1.46 times that of
// single-precision products with a power of two, 1.33 so).
template <typename T> __global__ void __launch_bounds__(PREP_THREADS) head_prep_kernel(const __grid_constant__ HeadPrepArgs a)
{
    chain_go();
    chain_wait();
    if (blockIdx.x == 0) {
        __shared__ float tops[PREP_THREADS / 32];
        float top = 0.f;
#pragma unroll 8
        for (int64_t row = threadIdx.x; row < a.rows; row += PREP_THREADS) {
            const float w = a.dloss ? fabsf(a.dloss[row]) : 1.f;
            if (takes_part(a.label[row], a.vocab) && w < __uint_as_float(0x7f800000u)) top = fmaxf(top, w);
        }
        top = warp_max(top);
        if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < PREP_THREADS / 32; ++w) top = fmaxf(top, tops[w]);
            const float up = top > 0.f ? fminf(16384.f / top, 0x1p126f) : 1.f;
            a.scale[0] = 1.f / up;
            a.scale[1] = up;
        }
        return;
    }
    if (!a.copy) return;
    const int units = int(a.ld_copy / 8);
    const int64_t all = a.rows * units, step = int64_t(gridDim.x - 1) * PREP_THREADS, down = step / units;
    const int along = int(step - down * units);
    const int64_t first = int64_t(blockIdx.x - 1) * PREP_THREADS + threadIdx.x;
    int64_t row = first / units;
    int u = int(first - row * units);
    for (int64_t i = first; i < all; i += step) {
        const uint4 v = takes_part(a.label[row], a.vocab) ? load_any(static_cast<const T *>(a.h) + row * a.ld_h, int64_t(u) * 8, int64_t(a.hidden)) : uint4{};
        *reinterpret_cast<uint4 *>(static_cast<T *>(a.copy) + row * a.ld_copy + u * 8) = v;
        if (a.twice) *reinterpret_cast<uint4 *>(static_cast<T *>(a.copy) + (a.rows + row) * a.ld_copy + u * 8) = v;
        row += down; u += along;
        if (u >= units) { u -= units; ++row; }
    }
}

// The pairs (maximum, sum of exponentials of the distances to it) of a row's pieces joined: a lane has a row, so that
// neighbouring lanes read neighbouring pairs; the block's warps share the pieces.
constexpr int FINISH_WARPS = 32;
__global__ void __launch_bounds__(32 * FINISH_WARPS) head_finish_kernel(const __grid_constant__ HeadFinishArgs a)
{
    chain_go();
    chain_wait();
    __shared__ float2 joined[FINISH_WARPS][32];
    const float ninf = __uint_as_float(0xff800000u);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = int64_t(blockIdx.x) * 32 + lane;
    const bool live = row < a.rows && takes_part(a.label[row], a.vocab);
    float top = ninf, sum = 0.f;
    // eight at a time: their maximum first, then terms that do not wait for one another
    constexpr int AHEAD = 8;
    auto join = [&](const float2 (&p)[AHEAD]) {
        float m = top;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) m = fmaxf(m, p[j].x);
        const float at = m == ninf ? 0.f : m;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) s += p[j].y * ex2((p[j].x - at) * LOG2E);
        sum = fmaf(sum, ex2((top - at) * LOG2E), s);
        top = m;
    };
    if (live) {
        for (int i = warp; i < a.tiles; i += FINISH_WARPS * AHEAD) {
            float2 p[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) p[j] = i + j * FINISH_WARPS < a.tiles ? a.stats[int64_t(i + j * FINISH_WARPS) * a.rows + row] : make_float2(ninf, 0.f);
            join(p);
        }
    }
    joined[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp || row >= a.rows) return;
    top = ninf; sum = 0.f;
#pragma unroll 1
    for (int w = 0; w < FINISH_WARPS; w += AHEAD) {
        float2 p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) p[j] = joined[w + j][lane];
        join(p);
    }
    const float rest = logf(sum), lse = top + rest;
    a.loss[row] = live ? (top - a.at_label[row]) + rest : 0.f;
    if (a.lse) a.lse[row] = live ? lse : 0.f;
    if (a.base) { a.base[row] = live ? top : 0.f; a.rest[row] = live ? rest : 0.f; }
}

// dz = w (exp(z - lse) - onehot) from exp(z - top) of the row's pieces, 16 bytes a lane and four at a time: every piece has one
// factor.  The label's entry is taken from its logit instead, which leaves 1 - p as exact as the logit is.
template <typename T> __global__ void __launch_bounds__(256) head_scale_kernel(const __grid_constant__ HeadScaleArgs a)
{
    chain_go();
    chain_wait();
    constexpr int AHEAD = 4, SEGMENT = 32 * 8 * AHEAD;
    const int lane = threadIdx.x & 31;
    const int64_t segments = (a.ld + SEGMENT - 1) / SEGMENT, all = a.rows * segments, step = int64_t(gridDim.x) * 8;
    const float up = *a.up;
    for (int64_t i = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5); i < all; i += step) {
        const int64_t row = i / segments, c = (i - row * segments) * SEGMENT + lane * 8;
        const int label = a.label[row];
        const bool live = takes_part(label, a.vocab);
        T *const at = static_cast<T *>(a.dz) + row * a.ld + c;
        uint4 p[AHEAD];
        float2 pair[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (live && c + j * 256 < a.ld) {
                p[j] = *reinterpret_cast<const uint4 *>(at + j * 256);
                const int64_t unit = (c + j * 256) / a.unit;
                pair[j] = c + j * 256 < a.vocab ? a.stats[unit * a.rows + row] : make_float2(0.f, 0.f);
            }
        const float base = live ? a.base[row] : 0.f, rest = live ? a.rest[row] : 0.f, w = live ? (a.dloss ? a.dloss[row] : 1.f) * up : 0.f;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (c + j * 256 >= a.ld) continue;
            uint4 out = {};
            if (live) {
                float v[8];
                unpack16<T>(p[j], v);
                // (a pair without logits above -inf has kept zeros)
                const float f = pair[j].x == __uint_as_float(0xff800000u) ? 0.f : w * ex2(((pair[j].x - base) - rest) * LOG2E) * (1.f / KEPT);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= f;
                const int64_t l = label - (c + j * 256);
                if (l >= 0 && l < 8) {
                    const float y = w * ex2(((a.at_label[row] - base) - rest) * LOG2E) - w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (e == l) v[e] = y;
                }
                out = pack16<T>(v);
            }
            *reinterpret_cast<uint4 *>(at + j * 256) = out;
        }
    }
}

}  // namespace

cudaError_t launch_head_scale(const HeadScaleArgs &a, int num_sms, cudaStream_t st)
{
    const int64_t warps = a.rows * ((a.ld + 1023) / 1024), blocks = (warps + 7) / 8, most = int64_t(num_sms) * 8;
    return launch_chained(a.dtype == RUBICK_BF16 ? head_scale_kernel<train::bf16> : head_scale_kernel<train::f16>, dim3(unsigned(blocks < most ? blocks : most)), dim3(256), 0, 1, st, a);
}

cudaError_t launch_head_prep(const HeadPrepArgs &a, int num_sms, cudaStream_t st)
{
    const int64_t blocks = a.copy ? (a.rows * (a.ld_copy / 8) + PREP_THREADS - 1) / PREP_THREADS : 0, most = int64_t(num_sms) * 2;
    return launch_chained(a.dtype == RUBICK_BF16 ? head_prep_kernel<train::bf16> : head_prep_kernel<train::f16>, dim3(unsigned(1 + (blocks < most ? blocks : most))), dim3(PREP_THREADS), 0, 1, st, a);
}

cudaError_t launch_head_finish(const HeadFinishArgs &a, int num_sms, cudaStream_t st)
{
    (void)num_sms;
    return launch_chained(head_finish_kernel, dim3(unsigned((a.rows + 31) / 32)), dim3(32 * FINISH_WARPS), 0, 1, st, a);
}

}  // namespace rubick
