// The head's cross entropy: what runs before and after the products of its logits.
#include "product.cuh"

namespace rubick {
namespace {

using namespace train;

__device__ __forceinline__ bool takes_part(int label, int vocab) { return label >= 0 && label < vocab; }

// A copy of h with rows next to each other, zeros in the rows that take no part (whatever they hold must not reach the
// sums over the rows), and the largest weight.
template <typename T> __global__ void __launch_bounds__(256) head_prep_kernel(const __grid_constant__ HeadPrepArgs a)
{
    const int units = int(a.ld_copy / 8);
    const bool wide = (a.ld_h & 7) == 0 && (reinterpret_cast<uintptr_t>(a.h) & 15) == 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const bool live = takes_part(a.label[row], a.vocab);
        if (a.largest && threadIdx.x == 0 && live) {
            const float w = a.dloss ? fabsf(a.dloss[row]) : 1.f;
            if (w < __uint_as_float(0x7f800000u)) atomicMax(a.largest, __float_as_uint(w));
        }
        const T *src = static_cast<const T *>(a.h) + row * a.ld_h;
        T *dst = static_cast<T *>(a.copy) + row * a.ld_copy;
        for (int u = threadIdx.x; u < units; u += blockDim.x) {
            float v[8] = {};
            if (live) load8<T>(src, u * 8, a.hidden, wide, v);
            store8<T>(dst, u * 8, a.ld_copy, true, v);
        }
    }
}
// Weights under a common power of two that brings the largest into [2^13, 2^14): in half precision the probabilities of a
// large vocabulary, times a weight of one over the rows, would mostly fall below its normal range.  The power is exact
// and taken out again, in single precision, behind the products.
__global__ void __launch_bounds__(256) head_weight_kernel(const __grid_constant__ HeadPrepArgs a)
{
    const float top = __uint_as_float(*a.largest);
    int e = 0;
    if (top > 0.f) frexpf(top, &e);
    e = 14 - e;
    e = e < -100 ? -100 : e > 100 ? 100 : e;
    const float up = ldexpf(1.f, e);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.scale = ldexpf(1.f, -e);
    for (int64_t row = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; row < a.rows; row += int64_t(gridDim.x) * blockDim.x)
        a.weight[row] = takes_part(a.label[row], a.vocab) ? (a.dloss ? a.dloss[row] : 1.f) * up : 0.f;
}

// The pairs (maximum, sum of exponentials of the distances to it) of a row's pieces joined: one thread a row, so that
// neighbouring threads read neighbouring pairs; the block's warps share the pieces.
__global__ void __launch_bounds__(256) head_finish_kernel(const __grid_constant__ HeadFinishArgs a)
{
    __shared__ float2 joined[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = int64_t(blockIdx.x) * 32 + lane;
    const bool live = row < a.rows && takes_part(a.label[row], a.vocab);
    float top = __uint_as_float(0xff800000u), sum = 0.f;
    auto join = [&](float2 p) {
        const float m = fmaxf(top, p.x), at = m == __uint_as_float(0xff800000u) ? 0.f : m;
        sum = sum * ex2((top - at) * LOG2E) + p.y * ex2((p.x - at) * LOG2E);
        top = m;
    };
    if (live) for (int i = warp; i < a.tiles; i += 8) join(a.stats[int64_t(i) * a.rows + row]);
    joined[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp || row >= a.rows) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) join(joined[w][lane]);
    const float rest = logf(sum), lse = top + rest;
    a.loss[row] = live ? (top - a.at_label[row]) + rest : 0.f;
    if (a.lse) a.lse[row] = live ? lse : 0.f;
    if (a.base) { a.base[row] = live ? top : 0.f; a.rest[row] = live ? rest : 0.f; }
}

}  // namespace

cudaError_t launch_head_prep(const HeadPrepArgs &a, int num_sms, cudaStream_t st)
{
    if (a.largest) {
        const cudaError_t e = cudaMemsetAsync(a.largest, 0, 4, st);
        if (e != cudaSuccess) return e;
    }
    const int grid = int(a.rows < int64_t(num_sms) * 8 ? a.rows : int64_t(num_sms) * 8);
    if (a.dtype == RUBICK_BF16) head_prep_kernel<train::bf16><<<grid, 256, 0, st>>>(a);
    else head_prep_kernel<train::f16><<<grid, 256, 0, st>>>(a);
    count_launch();
    if (a.largest) {
        const int64_t blocks = (a.rows + 255) / 256;
        head_weight_kernel<<<int(blocks < num_sms ? blocks : num_sms), 256, 0, st>>>(a);
        count_launch();
    }
    return cudaGetLastError();
}

cudaError_t launch_head_finish(const HeadFinishArgs &a, int num_sms, cudaStream_t st)
{
    (void)num_sms;
    head_finish_kernel<<<int((a.rows + 31) / 32), 256, 0, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace rubick
