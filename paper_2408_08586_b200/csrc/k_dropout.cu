// Dropout from a counter-based generator, and the elementwise part of a linear layer's backward pass with its column sums.
#include "product.cuh"

namespace rubick {
namespace {

using namespace train;

// Columns c .. c + VE - 1 of a row: 16 bytes at once where every row begins on such a boundary (WIDE), else one by one.
template <typename T, int VE, bool WIDE> __device__ __forceinline__ void read(const T *row, int c, int cols, float (&v)[VE])
{
    if constexpr (WIDE) load_cols<T, VE>(row, c, cols, v);
    else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = c + e < cols ? to_f(row[c + e]) : 0.f;
    }
}
template <typename T, int VE, bool WIDE> __device__ __forceinline__ void write(T *row, int c, int cols, const float (&v)[VE])
{
    if constexpr (WIDE) store_cols<T, VE>(row, c, cols, v);
    else {
#pragma unroll
        for (int e = 0; e < VE; ++e) if (c + e < cols) row[c + e] = from_f<T>(v[e]);
    }
}

// out = residual + drop(x), VE neighbouring columns a thread (VE is a multiple of four: a counter serves four columns).
template <typename T, int VE, bool WIDE> __global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    const Drop drop(a.drop);
    const int units = (a.d.cols + VE - 1) / VE;
    const int64_t all = a.d.rows * units, step = int64_t(gridDim.x) * blockDim.x;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += step) {
        const int64_t row = i / units;
        const int c = int(i - row * units) * VE;
        float v[VE], r[VE];
        read<T, VE, WIDE>(static_cast<const T *>(a.x) + row * a.d.ld_x, c, a.d.cols, v);
        if (a.residual) read<T, VE, WIDE>(static_cast<const T *>(a.residual) + row * a.d.ld_res, c, a.d.cols, r);
        if (drop.on) drop.apply<VE>(row, c, v);
        if (a.residual) {
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] += r[e];
        }
        write<T, VE, WIDE>(static_cast<T *>(a.out) + row * a.d.ld_out, c, a.d.cols, v);
    }
}

// dz = act'(pre) drop(dout); a block takes 8 columns x 32 lanes of a run of rows, and leaves the sums of its columns.
template <typename T> __global__ void __launch_bounds__(256) linear_grad_kernel(const __grid_constant__ LinearGradArgs a)
{
    __shared__ float sums[8][32][9];
    const Drop drop(a.drop);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = (blockIdx.x * 32 + lane) * 8;
    const int64_t per = (a.rows + a.chunks - 1) / a.chunks, from = per * blockIdx.y, to = from + per < a.rows ? from + per : a.rows;
    const bool w_dout = (a.ld_dout & 7) == 0 && (reinterpret_cast<uintptr_t>(a.dout) & 15) == 0;
    const bool w_pre = (a.ld_pre & 7) == 0 && (reinterpret_cast<uintptr_t>(a.pre) & 15) == 0;
    float total[8] = {};
    if (c < a.cols) {
        for (int64_t row = from + warp; row < to; row += 8) {
            float v[8], z[8];
            load8<T>(static_cast<const T *>(a.dout) + row * a.ld_dout, c, a.cols, w_dout, v);
            if (a.act != RUBICK_ACT_NONE) load8<T>(static_cast<const T *>(a.pre) + row * a.ld_pre, c, a.cols, w_pre, z);
            if (drop.on) drop.apply<8>(row, c, v);
            if (a.act != RUBICK_ACT_NONE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= act_slope(a.act, z[e]);
            }
            if (a.dz) store8<T>(static_cast<T *>(a.dz) + row * a.ld_dz, c, a.ld_dz, true, v);     // (its padding too)
#pragma unroll
            for (int e = 0; e < 8; ++e) total[e] += v[e];
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][lane][e] = total[e];
    __syncthreads();
    const int at = threadIdx.x >> 3, e = threadIdx.x & 7, col = (blockIdx.x * 32 + at) * 8 + e;
    if (col < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += sums[w][at][e];
        a.part[int64_t(blockIdx.y) * a.cols + col] = s;
    }
}
__global__ void __launch_bounds__(256) column_sum_kernel(const float *part, float *out, int cols, int chunks)
{
    __shared__ float sums[8][32];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
    float s = 0.f;
    if (col < cols) for (int i = warp; i < chunks; i += 8) s += part[int64_t(i) * cols + col];
    sums[warp][threadIdx.x & 31] = s;
    __syncthreads();
    if (warp == 0 && col < cols) {
#pragma unroll
        for (int w = 1; w < 8; ++w) s += sums[w][threadIdx.x];
        out[col] = s;
    }
}

template <typename T> cudaError_t dropout(const DropoutArgs &a, int num_sms, cudaStream_t st)
{
    const int es = int(sizeof(T));
    const bool wide = aligned16(a.x) && aligned16(a.out) && aligned16(a.residual) && (a.d.ld_x * es) % 16 == 0 && (a.d.ld_out * es) % 16 == 0 &&
                      (!a.residual || (a.d.ld_res * es) % 16 == 0);
    const int ve = wide ? Lanes<T>::N : 4;
    const int64_t units = (a.d.cols + ve - 1) / ve * a.d.rows, blocks = (units + 255) / 256, most = int64_t(num_sms) * 8;
    const int grid = int(blocks < most ? blocks : most);
    if (wide) dropout_kernel<T, Lanes<T>::N, true><<<grid, 256, 0, st>>>(a);
    else dropout_kernel<T, 4, false><<<grid, 256, 0, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs &a, int num_sms, cudaStream_t st)
{
    switch (a.d.dtype) {
    case RUBICK_BF16: return dropout<train::bf16>(a, num_sms, st);
    case RUBICK_F16: return dropout<train::f16>(a, num_sms, st);
    default: return dropout<float>(a, num_sms, st);
    }
}

// chunks of rows: enough blocks for four a multiprocessor, 32 rows each at least
int linear_grad_chunks(int64_t rows, int cols, int num_sms)
{
    const int64_t across = (cols + 255) / 256, want = (int64_t(num_sms) * 4 + across - 1) / across, most = (rows + 31) / 32;
    const int64_t n = want < most ? want : most;
    return int(n < 1 ? 1 : n > 65535 ? 65535 : n);
}

cudaError_t launch_linear_grad(const LinearGradArgs &a, int num_sms, cudaStream_t st)
{
    (void)num_sms;
    const dim3 grid((a.cols + 255) / 256, a.chunks);
    if (a.dtype == RUBICK_BF16) linear_grad_kernel<train::bf16><<<grid, 256, 0, st>>>(a);
    else linear_grad_kernel<train::f16><<<grid, 256, 0, st>>>(a);
    count_launch();
    if (a.dbias) {
        column_sum_kernel<<<(a.cols + 31) / 32, 256, 0, st>>>(a.part, a.dbias, a.cols, a.chunks);
        count_launch();
    }
    return cudaGetLastError();
}

}  // namespace rubick
