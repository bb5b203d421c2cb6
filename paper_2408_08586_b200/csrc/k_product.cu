// Matrix products of a training step with their epilogues.
#include "product.cuh"

namespace rubick {
namespace {

using namespace train;

constexpr int BM = 64, BN = STATS_COLS, BK = 16;

// 64 x 128 sums a block, 4 x 8 a thread, through shared memory in single precision.
template <typename T, ProductKind KIND> __global__ void __launch_bounds__(256) product_kernel(const __grid_constant__ ProductArgs a)
{
    __shared__ float sa[BK][BM + 1], sb[BK][BN + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t m0 = int64_t(blockIdx.y) * BM, n0 = int64_t(blockIdx.x) * BN;
    const int split = blockIdx.z;
    const int64_t steps = (a.k + BK - 1) / BK;
    const int64_t k0 = KIND == PRODUCT_PART ? steps * split / a.splits * BK : 0, k1 = KIND == PRODUCT_PART ? steps * (split + 1) / a.splits * BK : a.k;
    const T *pa = static_cast<const T *>(a.a.p), *pb = static_cast<const T *>(a.b.p);
    float v[4][8] = {};
    for (int64_t k = k0; k < k1; k += BK) {
        for (int i = threadIdx.x; i < BM * BK; i += 256) {
            const int r = a.a.along_k ? i / BK : i % BM, q = a.a.along_k ? i % BK : i / BM;
            const int64_t m = m0 + r, kk = k + q;
            sa[q][r] = m < a.m && kk < a.k ? to_f(a.a.along_k ? pa[m * a.a.ld + kk] : pa[kk * a.a.ld + m]) : 0.f;
        }
        for (int i = threadIdx.x; i < BN * BK; i += 256) {
            const int r = a.b.along_k ? i / BK : i % BN, q = a.b.along_k ? i % BK : i / BN;
            const int64_t n = n0 + r, kk = k + q;
            sb[q][r] = n < a.n && kk < a.k ? to_f(a.b.along_k ? pb[n * a.b.ld + kk] : pb[kk * a.b.ld + n]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < BK; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = fmaf(sa[q][ty * 4 + i], sb[q][tx * 8 + j], v[i][j]);
        __syncthreads();
    }
    const Drop drop(a.drop);
    const float scale = a.scale ? *a.scale : 1.f;
    const int64_t c = n0 + tx * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = m0 + ty * 4 + i;
        const bool in = row < a.m;
        if constexpr (KIND == PRODUCT_OUT) {
            if (in && c < a.n) finish8<T>(a, drop, scale, row, c, v[i]);
        } else if constexpr (KIND == PRODUCT_PART) {
            if (in && c < a.n) store8<float>(a.part + (int64_t(split) * a.m + row) * a.ld_acc, c, a.ld_acc, true, v[i]);
        } else if constexpr (KIND == PRODUCT_STATS) {
            float top = __uint_as_float(0xff800000u), sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < a.n) top = fmaxf(top, v[i][e]);
#pragma unroll
            for (int o = 8; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float at = top == __uint_as_float(0xff800000u) ? 0.f : top;
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < a.n) sum += ex2((v[i][e] - at) * LOG2E);
#pragma unroll
            for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (in) {
                if (tx == 0) a.stats[int64_t(blockIdx.x) * a.m + row] = make_float2(top, sum);
                const int64_t l = int64_t(a.label[row]) - a.first - c;
                if (l >= 0 && l < 8 && c + l < a.n) a.at_label[row] = v[i][l];
            }
        } else {
            if (in && c < a.ld_out) {
                const float base = a.base[row], rest = a.rest ? a.rest[row] : 0.f, w = a.weight[row];
                const int64_t l = int64_t(a.label[row]) - a.first - c;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = w == 0.f ? 0.f : w * (ex2(((v[i][e] - base) - rest) * LOG2E) - (e == l ? 1.f : 0.f));
                store8<T>(static_cast<T *>(a.out) + row * a.ld_out, c, a.ld_out, true, v[i]);
            }
        }
    }
}

// The sums of the splits joined, and PRODUCT_OUT's epilogue.
template <typename T> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ ProductArgs a)
{
    const Drop drop(a.drop);
    const float scale = a.scale ? *a.scale : 1.f;
    const int64_t units = (a.n + 7) / 8, all = a.m * units;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += int64_t(gridDim.x) * blockDim.x) {
        const int64_t row = i / units, c = (i - row * units) * 8;
        float v[8] = {};
        for (int s = 0; s < a.splits; ++s) {
            float p[8];
            load8<float>(a.part + (int64_t(s) * a.m + row) * a.ld_acc, c, a.ld_acc, true, p);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += p[e];
        }
        finish8<T>(a, drop, scale, row, c, v);
    }
}

template <typename T> cudaError_t product(ProductKind kind, const ProductArgs &a, int num_sms, cudaStream_t st)
{
    const dim3 grid(unsigned((a.n + BN - 1) / BN), unsigned((a.m + BM - 1) / BM), kind == PRODUCT_PART ? a.splits : 1);
    switch (kind) {
    case PRODUCT_OUT: product_kernel<T, PRODUCT_OUT><<<grid, 256, 0, st>>>(a); break;
    case PRODUCT_STATS: product_kernel<T, PRODUCT_STATS><<<grid, 256, 0, st>>>(a); break;
    case PRODUCT_GRAD: product_kernel<T, PRODUCT_GRAD><<<grid, 256, 0, st>>>(a); break;
    case PRODUCT_PART: {
        product_kernel<T, PRODUCT_PART><<<grid, 256, 0, st>>>(a);
        const int64_t blocks = (a.m * ((a.n + 7) / 8) + 255) / 256, most = int64_t(num_sms) * 8;
        join_kernel<T><<<int(blocks < most ? blocks : most), 256, 0, st>>>(a);
        count_launch();
        break;
    }
    }
    count_launch();
    return cudaGetLastError();
}

}  // namespace

int product_splits(const ProductArgs &a, int num_sms)
{
    const int64_t tiles = ((a.m + BM - 1) / BM) * ((a.n + BN - 1) / BN), most = (a.k + 255) / 256;
    const int64_t s = num_sms / (tiles < 1 ? 1 : tiles);
    return int(s < 2 || most < 2 ? 1 : s < most ? s : most);
}

cudaError_t launch_product(ProductKind kind, const ProductArgs &a, int num_sms, cudaStream_t st)
{
    return a.dtype == RUBICK_BF16 ? product<train::bf16>(kind, a, num_sms, st) : product<train::f16>(kind, a, num_sms, st);
}

}  // namespace rubick
