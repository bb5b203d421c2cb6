// What the training-step operators share: element types, 16-byte rows in registers, reductions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "rubick_internal.cuh"

namespace rubick {
namespace train {

using bf16 = __nv_bfloat16;
using f16 = __half;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(f16 v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ f16 from_f<f16>(float v) { return __float2half_rn(v); }

// elements of T in 16 bytes
template <typename T> struct Lanes { static constexpr int N = 16 / int(sizeof(T)); };

__device__ __forceinline__ void unpack(const uint4 &r, float (&v)[4])
{
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
}
// a bf16 is the upper half of a float: two integer operations unpack a pair
__device__ __forceinline__ void unpack_pair(uint32_t w, bf16, float &a, float &b)
{
    a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack_pair(uint32_t w, f16, float &a, float &b)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    a = f.x; b = f.y;
}
__device__ __forceinline__ uint32_t pack_pair(float a, float b, bf16)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ uint32_t pack_pair(float a, float b, f16)
{
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
template <typename T> __device__ __forceinline__ void unpack16(const uint4 &r, float (&v)[Lanes<T>::N])
{
    if constexpr (sizeof(T) == 4) {
        unpack(r, v);
    } else {
        unpack_pair(r.x, T(), v[0], v[1]); unpack_pair(r.y, T(), v[2], v[3]);
        unpack_pair(r.z, T(), v[4], v[5]); unpack_pair(r.w, T(), v[6], v[7]);
    }
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float (&v)[Lanes<T>::N])
{
    uint4 r;
    if constexpr (sizeof(T) == 4) {
        r.x = __float_as_uint(v[0]); r.y = __float_as_uint(v[1]); r.z = __float_as_uint(v[2]); r.w = __float_as_uint(v[3]);
    } else {
        r.x = pack_pair(v[0], v[1], T()); r.y = pack_pair(v[2], v[3], T());
        r.z = pack_pair(v[4], v[5], T()); r.w = pack_pair(v[6], v[7], T());
    }
    return r;
}

// Streaming 16-byte accesses: each byte of a row tensor is used once, so it is kept out of L1.
__device__ __forceinline__ uint4 ld_stream(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
__device__ __forceinline__ void st_stream(void *p, const uint4 &r)
{
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w) : "memory");
}

// VE consecutive elements of a row from column c (VE = 1, or 16 bytes' worth on a 16-byte boundary); columns from
// `cols` on are not touched and read as 0.
template <typename T, int VE> __device__ __forceinline__ void load_cols(const T *row, int c, int cols, float (&v)[VE])
{
    if constexpr (VE == Lanes<T>::N) {
        if (c + VE <= cols) { unpack16<T>(ld_stream(row + c), v); return; }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = c + e < cols ? to_f(row[c + e]) : 0.f;
}
template <typename T, int VE> __device__ __forceinline__ void store_cols(T *row, int c, int cols, const float (&v)[VE])
{
    if constexpr (VE == Lanes<T>::N) {
        if (c + VE <= cols) { st_stream(row + c, pack16<T>(v)); return; }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) if (c + e < cols) row[c + e] = from_f<T>(v[e]);
}
__device__ __forceinline__ uint4 ld_cached(const void *p)
{
    uint4 r;
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
// the same for a small vector that many rows read (kept in L1 and read again for each row: holding it in registers
// would cost the registers that rows in flight need), with a value for the columns past the end
template <typename W, int VE> __device__ __forceinline__ void load_shared_cols(const W *w, int c, int cols, float (&v)[VE], float other)
{
    if constexpr (VE > 1) {
        if (c + VE <= cols) {
            constexpr int N = Lanes<W>::N;
#pragma unroll
            for (int i = 0; i < VE; i += N) {
                float part[N];
                unpack16<W>(ld_cached(w + c + i), part);
#pragma unroll
                for (int e = 0; e < N && i + e < VE; ++e) v[i + e] = part[e];
            }
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = c + e < cols ? to_f(w[c + e]) : other;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// ---- pairs of single-precision numbers: one instruction adds, multiplies or fuses both halves --------------------
using f2 = unsigned long long;
__device__ __forceinline__ f2 pair(float lo, float hi) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ f2 both(float v) { return pair(v, v); }
__device__ __forceinline__ float lo(f2 v) { return __uint_as_float(uint32_t(v)); }
__device__ __forceinline__ float hi(f2 v) { return __uint_as_float(uint32_t(v >> 32)); }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
template <typename T> __device__ __forceinline__ void unpack16(const uint4 &r, f2 (&v)[Lanes<T>::N / 2])
{
    if constexpr (sizeof(T) == 4) {
        v[0] = pair(__uint_as_float(r.x), __uint_as_float(r.y)); v[1] = pair(__uint_as_float(r.z), __uint_as_float(r.w));
    } else {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { float a, b; unpack_pair(w[i], T(), a, b); v[i] = pair(a, b); }
    }
}
template <typename T> __device__ __forceinline__ uint4 pack16(const f2 (&v)[Lanes<T>::N / 2])
{
    uint4 r;
    if constexpr (sizeof(T) == 4) {
        r.x = __float_as_uint(lo(v[0])); r.y = __float_as_uint(hi(v[0])); r.z = __float_as_uint(lo(v[1])); r.w = __float_as_uint(hi(v[1]));
    } else {
        r.x = pack_pair(lo(v[0]), hi(v[0]), T()); r.y = pack_pair(lo(v[1]), hi(v[1]), T());
        r.z = pack_pair(lo(v[2]), hi(v[2]), T()); r.w = pack_pair(lo(v[3]), hi(v[3]), T());
    }
    return r;
}

// ---- rows copied into shared memory by the bulk-copy engine, with a barrier that counts the bytes that have arrived
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint64_t *bar)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
// dst, src and bytes: multiples of 16
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}
// Waits for the phase to end, a bounded number of times; false: it did not (the kernel then reports it and goes on with
// what is there -- no address depends on the data).
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity)
{
    const uint32_t at = smem_addr(bar);
    for (int i = 0; i < (1 << 18); ++i) {
        uint32_t done;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(at), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace train

// argument blocks of the kernels, filled by the entry points
struct NormArgs {
    rubick_block_norm_desc d;
    const void *x, *y, *w_after, *gate, *w_before;
    void *x_out, *h;
    float *rstd;
    // backward
    const float *rstd_in;
    const void *dx_out, *dh;
    void *dx, *dy, *dgate;
    float *dw_after, *dw_before;
    float *part;                 // scratch: partial column sums of the row chunks
    int64_t chunk_rows;
    int n_chunks;
    uint32_t *status;            // the context's status word
};
struct RouterArgs {
    rubick_router_desc d;
    const void *logits;
    const uint8_t *mask;
    int32_t *index; float *weight; int32_t *counts; float *prob_sum; int32_t *valid; float *loss;
    // backward
    const int32_t *index_in; const float *weight_in; const int32_t *counts_in; const int32_t *valid_in;
    const float *dloss, *dweight;
    void *dlogits;
    // scratch
    float *part;                 // [G][chunks][experts] probability sums
    int32_t *part_counts;        // [G][chunks][experts + 1] assignments, valid rows
    float *group_loss;           // [G] loss of a group
    const float *some;           // backward: number of groups with valid rows, counted beforehand (NULL: by every block)
    uint32_t *tickets;           // [G + 1] arrivals, zero between calls
    int64_t groups;
    int chunks;                  // row chunks of a group
};
struct DistillArgs {
    rubick_distill_desc d;
    const void *z, *teacher;
    const int32_t *index;
    const float *lse_in, *dloss;
    float *loss, *lse;
    float *lse_low;              // scratch of a step in two passes: what lse lacks by its rounding
    void *dz;
    uint32_t *status;            // the context's status word
};

size_t norm_backward_scratch(const NormArgs &a, int num_sms, int64_t *chunk_rows, int *n_chunks);
cudaError_t launch_norm_forward(const NormArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_norm_backward(const NormArgs &a, int num_sms, cudaStream_t st);
int router_chunks(const RouterArgs &a, int num_sms);
cudaError_t launch_router_forward(const RouterArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_router_backward(const RouterArgs &a, int num_sms, cudaStream_t st);
size_t distill_step_scratch(const DistillArgs &a);
cudaError_t launch_distill_forward(const DistillArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_distill_backward(const DistillArgs &a, int num_sms, cudaStream_t st);
cudaError_t launch_distill_step(const DistillArgs &a, int num_sms, cudaStream_t st);

}  // namespace rubick
