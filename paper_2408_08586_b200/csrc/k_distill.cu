// Distillation from a teacher's largest logits.  With c = log2(e) / T, q = softmax(teacher / T) over a row's K entries
// and p = softmax(z / T) over the vocabulary,
//   loss = T^2 sum_j q_j (log q_j - log p_j),   dz = dloss T (p - q).
//
// A row of the vocabulary is long (32 thousand to a quarter of a million logits) and rows can be few, so a row is cut
// over a thread-block cluster: every block reduces its part to (maximum, sum of exponentials), the blocks read each
// other's pair through distributed shared memory, and for the combined step the part waits in registers meanwhile, so
// that z is read once.  Rows start at any address: vectors are laid on 16-byte boundaries of memory, and the elements
// of the first and last vector that belong to other rows are left alone.
//
// Bound by memory: 2 bytes a logit forward, 4 for the step in 16-bit types, against one exponential (two for the
// step) from a pipe that gives 16 a clock and SM.

#include <cooperative_groups.h>

#include "train_common.cuh"

namespace rubick {

using namespace train;
namespace cg = cooperative_groups;

namespace {

constexpr int THREADS = 512;
constexpr int WARPS = THREADS / 32;
constexpr float LOG2E = 1.4426950408889634f;
constexpr double LOG2E_D = 1.4426950408889634;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The vectors of one row: vector v holds the elements v * VE - shift + e; those outside 0 .. vocab - 1 are other rows'.
template <typename T> struct RowView {
    static constexpr int VE = Lanes<T>::N;
    const T *row;
    int shift, vocab, vectors;
    __device__ RowView(const void *base, int64_t row_index, int64_t ld, int vocab_)
    {
        row = static_cast<const T *>(base) + row_index * ld;
        shift = int((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        vocab = vocab_;
        vectors = (vocab + shift + VE - 1) / VE;
    }
    __device__ __forceinline__ int first(int v) const { return v * VE - shift; }
    __device__ __forceinline__ bool whole(int v) const { return first(v) >= 0 && first(v) + VE <= vocab; }
    __device__ __forceinline__ uint4 load(int v) const
    {
        const int c = first(v);
        if (c >= 0 && c + VE <= vocab) return ld_stream(row + c);
        float f[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = c + e >= 0 && c + e < vocab ? to_f(row[c + e]) : -INFINITY;
        return pack16<T>(f);
    }
};

// A row's teacher entries in shared memory.
struct Teacher {
    int32_t index[RUBICK_MAX_TEACHER_LOGITS];     // -1: does not take part
    float q[RUBICK_MAX_TEACHER_LOGITS];
    float red[WARPS];
};

__device__ __forceinline__ float teacher_logit(const DistillArgs &a, int64_t at)
{
    if (a.d.ttype == RUBICK_BF16) return to_f(static_cast<const bf16 *>(a.teacher)[at]);
    if (a.d.ttype == RUBICK_F16) return to_f(static_cast<const f16 *>(a.teacher)[at]);
    return static_cast<const float *>(a.teacher)[at];
}

__device__ __forceinline__ float block_sum(float v, float *red)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < WARPS ? red[threadIdx.x & 31] : 0.f;
    return warp_sum(v);
}
__device__ __forceinline__ float block_max(float v, float *red)
{
    v = warp_max(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < WARPS ? red[threadIdx.x & 31] : -INFINITY;
    return warp_max(v);
}

// Softmax over the entries of a row, by the whole block; log_q and z are handed back for the entry of this thread's
// turn through f(j, q, log q).  Returns whether the row has entries.
__device__ __forceinline__ bool teacher_softmax(const DistillArgs &a, int64_t row, Teacher &t)
{
    const int k = a.d.k;
    float top = -INFINITY;
    for (int j = threadIdx.x; j < k; j += THREADS) {
        const int i = a.index[row * k + j];
        const float l = teacher_logit(a, row * k + j);
        const bool in = i >= 0 && i < a.d.vocab && !(l == -INFINITY);
        t.index[j] = in ? i : -1;
        t.q[j] = l;
        // a NaN must reach the sum: it does not win a maximum, but exp(NaN - top) is NaN
        if (in) top = fmaxf(top, l != l ? -3e38f : l);
    }
    top = block_max(top, t.red);
    if (top == -INFINITY) return false;
    const float c = LOG2E / a.d.temperature;
    float total = 0.f;
    for (int j = threadIdx.x; j < k; j += THREADS) total += t.index[j] >= 0 ? ex2((t.q[j] - top) * c) : 0.f;
    total = block_sum(total, t.red);
    // q in place of the logit; log q is taken again from it where the loss needs it
    const float log2_total = log2f(total);
    for (int j = threadIdx.x; j < k; j += THREADS) t.q[j] = t.index[j] >= 0 ? (t.q[j] - top) * c - log2_total : -INFINITY;   // log2 q
    return true;
}

// q of vocabulary entry i: an index listed twice counts with the sum of its entries
__device__ __forceinline__ float teacher_mass(const Teacher &t, int k, int i)
{
    float s = 0.f;
    for (int j = 0; j < k; ++j) if (t.index[j] == i) s += ex2(t.q[j]);
    return s;
}

struct Pair { float m, s; };      // maximum of z, sum of 2^((z - m) c)

__device__ __forceinline__ Pair merge(Pair a, Pair b, float c)
{
    const float m = fmaxf(a.m, b.m);
    const float shift = m == -INFINITY ? 0.f : m;
    Pair r;
    r.m = m;
    r.s = a.s * ex2((a.m - shift) * c) + b.s * ex2((b.m - shift) * c);
    return r;
}
__device__ __forceinline__ Pair warp_merge(Pair p, float c)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        Pair q;
        q.m = __shfl_xor_sync(0xffffffffu, p.m, o);
        q.s = __shfl_xor_sync(0xffffffffu, p.s, o);
        // both sides of a pair must get the same bits: the lower lane's pair first
        p = (threadIdx.x & o) ? merge(q, p, c) : merge(p, q, c);
    }
    return p;
}

template <typename T> __device__ __forceinline__ float vector_max(const uint4 &r, float m)
{
    float v[Lanes<T>::N];
    unpack16<T>(r, v);
#pragma unroll
    for (int e = 0; e < Lanes<T>::N; ++e) m = fmaxf(m, v[e]);
    return m;
}
// sum of 2^(v c - mc)
template <typename T> __device__ __forceinline__ float vector_sum(const uint4 &r, float c, float mc)
{
    float v[Lanes<T>::N], s = 0.f;
    unpack16<T>(r, v);
#pragma unroll
    for (int e = 0; e < Lanes<T>::N; ++e) s += ex2(fmaf(v[e], c, -mc));
    return s;
}

// One row per cluster.  STEP: the row's vectors stay in registers (NV a thread) and the gradient is written; otherwise
// any number of vectors is read in batches of NV.
template <typename T, int NV, bool STEP>
__global__ void __launch_bounds__(THREADS, 2) distill_row_kernel(const __grid_constant__ DistillArgs a)
{
    __shared__ Teacher teacher;
    __shared__ Pair parts[WARPS];
    __shared__ Pair mine;
    constexpr int VE = Lanes<T>::N;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int64_t row = blockIdx.x / ranks;
    const int k = a.d.k;
    const RowView<T> z(a.z, row, a.d.ld, a.d.vocab);
    const int per = (z.vectors + ranks - 1) / ranks;
    const int v0 = rank * per, v1 = v0 + per < z.vectors ? v0 + per : z.vectors;
    const float c = LOG2E / a.d.temperature;

    uint4 r[NV];
    if constexpr (STEP) {
        // the loads go out before anything else is waited for
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = v0 + i * THREADS + int(threadIdx.x);
            if (v < v1) r[i] = z.load(v);
        }
    }
    const bool live = teacher_softmax(a, row, teacher);      // the same in every block of the cluster
    Pair p{-INFINITY, 0.f};
    if constexpr (STEP) {
#pragma unroll
        for (int i = 0; i < NV; ++i) if (v0 + i * THREADS + int(threadIdx.x) < v1) p.m = vector_max<T>(r[i], p.m);
        p.m = block_max(p.m, teacher.red);                   // one maximum for the block: no rescaling between its threads
        const float mc = p.m == -INFINITY ? 0.f : p.m * c;
#pragma unroll
        for (int i = 0; i < NV; ++i) if (v0 + i * THREADS + int(threadIdx.x) < v1) p.s += vector_sum<T>(r[i], c, mc);
        p.s = block_sum(p.s, teacher.red);
        if (threadIdx.x == 0) mine = p;
    } else if (live) {
        for (int v = v0 + int(threadIdx.x); v < v1; v += NV * THREADS) {
            uint4 b[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) if (v + i * THREADS < v1) b[i] = z.load(v + i * THREADS);
            float m = p.m;
#pragma unroll
            for (int i = 0; i < NV; ++i) if (v + i * THREADS < v1) m = vector_max<T>(b[i], m);
            const float mc = m == -INFINITY ? 0.f : m * c;
            p.s *= ex2(fmaf(p.m, c, -mc));
            p.m = m;
#pragma unroll
            for (int i = 0; i < NV; ++i) if (v + i * THREADS < v1) p.s += vector_sum<T>(b[i], c, mc);
        }
        p = warp_merge(p, c);
        if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = p;
        __syncthreads();
        if (threadIdx.x < 32) {
            p = threadIdx.x < WARPS ? parts[threadIdx.x] : Pair{-INFINITY, 0.f};
            p = warp_merge(p, c);
            if (threadIdx.x == 0) mine = p;
        }
    }
    // the student's logits at the teacher's entries, before any block of the cluster writes a gradient over them
    constexpr int PER = RUBICK_MAX_TEACHER_LOGITS / THREADS;
    float zk[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int j = threadIdx.x + u * THREADS;
        zk[u] = live && j < k && teacher.index[j] >= 0 ? to_f(z.row[teacher.index[j]]) : -INFINITY;
    }
    cluster.sync();
    p = Pair{-INFINITY, 0.f};
    if (ranks == 1) p = mine;
    else for (int q = 0; q < ranks; ++q) p = merge(p, *cluster.map_shared_rank(&mine, q), c);
    cluster.sync();                                          // no block leaves while others read its pair
    const float shift = p.m == -INFINITY ? 0.f : p.m;
    const float log2_s = log2f(p.s);
    if (rank == 0) {
        float loss = 0.f;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int j = threadIdx.x + u * THREADS;
            if (live && j < k && teacher.index[j] >= 0) {
                const float lq = teacher.q[j];
                const float lp = zk[u] == -INFINITY ? -INFINITY : (zk[u] - shift) * c - log2_s;
                const float q = ex2(lq);
                if (q > 0.f || q != q) loss = fmaf(q, lq - lp, loss);
            }
        }
        loss = block_sum(loss, teacher.red);
        if (threadIdx.x == 0) {
            a.loss[row] = live ? a.d.temperature * a.d.temperature * LN2 * loss : 0.f;
            if (a.lse) a.lse[row] = live ? fmaf(shift, 1.f / a.d.temperature, LN2 * log2_s) : 0.f;
        }
    }
    if constexpr (STEP) {
        const float up = (a.dloss ? a.dloss[row] : 1.f) * a.d.temperature;
        T *dz = static_cast<T *>(a.dz) + row * a.d.ld;
        const bool same = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z.row) & 15);
        const float mc = shift * c, scale = live ? up * (1.f / p.s) : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = v0 + i * THREADS + int(threadIdx.x);
            if (v < v1) {
                float f[VE];
                unpack16<T>(r[i], f);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[e] = live ? (f[e] == -INFINITY ? 0.f : scale * ex2(fmaf(f[e], c, -mc))) : 0.f;
                const int c0 = z.first(v);
                if (same && z.whole(v)) st_stream(dz + c0, pack16<T>(f));
                else {
#pragma unroll
                    for (int e = 0; e < VE; ++e) if (c0 + e >= 0 && c0 + e < z.vocab) dz[c0 + e] = from_f<T>(f[e]);
                }
            }
        }
        if (live) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int j = threadIdx.x + u * THREADS;
                if (j < k && teacher.index[j] >= 0) {
                    const int i = teacher.index[j], v = (i + z.shift) / VE;
                    if (v >= v0 && v < v1) {
                        const float pj = zk[u] == -INFINITY ? 0.f : ex2(fmaf(zk[u], c, -mc)) / p.s;
                        dz[i] = from_f<T>(up * (pj - teacher_mass(teacher, k, i)));
                    }
                }
            }
        }
    }
}

// Gradient from a saved log-sum: element-wise, so a row is cut into blockIdx.x parts that need nothing of each other.
template <typename T>
__global__ void __launch_bounds__(THREADS, 2) distill_backward_kernel(const __grid_constant__ DistillArgs a, int parts)
{
    __shared__ Teacher teacher;
    constexpr int VE = Lanes<T>::N, NV = 4;
    const int64_t row = blockIdx.x / parts;
    const int part = blockIdx.x % parts, k = a.d.k;
    const RowView<T> z(a.z, row, a.d.ld, a.d.vocab);
    const int per = (z.vectors + parts - 1) / parts;
    const int v0 = part * per, v1 = v0 + per < z.vectors ? v0 + per : z.vectors;
    const bool live = teacher_softmax(a, row, teacher);
    constexpr int PER = RUBICK_MAX_TEACHER_LOGITS / THREADS;
    float zk[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int j = threadIdx.x + u * THREADS;
        const int i = live && j < k ? teacher.index[j] : -1, v = (i + z.shift) / VE;
        zk[u] = i >= 0 && v >= v0 && v < v1 ? to_f(z.row[i]) : -INFINITY;
    }
    __syncthreads();                                         // read before anything is written over them
    const float c = LOG2E / a.d.temperature, lse = a.lse_in[row] * LOG2E;
    // single-precision gradients: what the two factors lose by rounding shows in p, so it is added back
    const float c_low = float(double(LOG2E_D) / double(a.d.temperature) - double(c)), lse_low = float(double(a.lse_in[row]) * LOG2E_D - double(lse));
    const auto prob = [&](float v) { return ex2(sizeof(T) == 4 ? fmaf(v, c, -lse) + fmaf(v, c_low, -lse_low) : fmaf(v, c, -lse)); };
    const float up = (a.dloss ? a.dloss[row] : 1.f) * a.d.temperature;
    T *dz = static_cast<T *>(a.dz) + row * a.d.ld;
    const bool same = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z.row) & 15);
    for (int v = v0 + int(threadIdx.x); v < v1; v += NV * THREADS) {
        uint4 b[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) if (live && v + i * THREADS < v1) b[i] = z.load(v + i * THREADS);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int w = v + i * THREADS;
            if (w < v1) {
                float f[VE];
                unpack16<T>(b[i], f);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[e] = live ? (f[e] == -INFINITY ? 0.f : up * prob(f[e])) : 0.f;
                const int c0 = z.first(w);
                if (same && z.whole(w)) st_stream(dz + c0, pack16<T>(f));
                else {
#pragma unroll
                    for (int e = 0; e < VE; ++e) if (c0 + e >= 0 && c0 + e < z.vocab) dz[c0 + e] = from_f<T>(f[e]);
                }
            }
        }
    }
    if (!live) return;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int j = threadIdx.x + u * THREADS;
        const int i = j < k ? teacher.index[j] : -1, v = (i + z.shift) / VE;
        if (i >= 0 && v >= v0 && v < v1) {
            const float pj = zk[u] == -INFINITY ? 0.f : prob(zk[u]);
            dz[i] = from_f<T>(up * (pj - teacher_mass(teacher, k, i)));
        }
    }
}

template <typename T, int NV, bool STEP> cudaError_t launch_rows(const DistillArgs &a, int ranks, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(a.d.rows * ranks));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, distill_row_kernel<T, NV, STEP>, a);
    count_launch();
    return e;
}

// blocks of a row: a power of two up to 8 (the portable cluster size)
template <typename T> cudaError_t forward_of(const DistillArgs &a, int num_sms, cudaStream_t st)
{
    const int vectors = a.d.vocab / Lanes<T>::N + 2;
    int ranks = 1;
    while (ranks < 8 && a.d.rows * ranks < 2 * int64_t(num_sms) && vectors > ranks * THREADS) ranks *= 2;
    return launch_rows<T, 4, false>(a, ranks, st);
}

template <typename T> cudaError_t backward_of(const DistillArgs &a, int num_sms, cudaStream_t st)
{
    const int64_t vectors = a.d.vocab / Lanes<T>::N + 2;
    // 16 KB or more of z a block; fewer where the rows do not fill the SMs
    int64_t parts = (vectors + 4 * THREADS - 1) / (4 * THREADS);
    while (parts * a.d.rows < 2 * int64_t(num_sms) && parts * THREADS < vectors) parts *= 2;
    if (parts * a.d.rows > 0x7fffffff) parts = 0x7fffffff / a.d.rows;
    distill_backward_kernel<T><<<unsigned(a.d.rows * parts), THREADS, 0, st>>>(a, int(parts));
    count_launch();
    return cudaGetLastError();
}

template <typename T> cudaError_t step_of(const DistillArgs &a, int num_sms, cudaStream_t st)
{
    constexpr int NV = 8;
    const int vectors = (a.d.vocab + 2 * Lanes<T>::N - 2) / Lanes<T>::N;       // of a row at the worst shift
    int ranks = 1;
    while (ranks < 8 && ranks * NV * THREADS < vectors) ranks *= 2;
    while (ranks < 8 && a.d.rows * ranks < 2 * int64_t(num_sms) && vectors > ranks * THREADS) ranks *= 2;
    if (ranks * NV * THREADS >= vectors) return launch_rows<T, NV, true>(a, ranks, st);
    // longer than a cluster's registers: two passes
    DistillArgs b = a;
    const cudaError_t e = forward_of<T>(a, num_sms, st);
    if (e != cudaSuccess) return e;
    b.lse_in = a.lse;
    return backward_of<T>(b, num_sms, st);
}

}  // namespace

#define BY_TYPE(call) (a.d.dtype == RUBICK_BF16 ? call<bf16>(a, num_sms, st) : a.d.dtype == RUBICK_F16 ? call<f16>(a, num_sms, st) : call<float>(a, num_sms, st))
cudaError_t launch_distill_forward(const DistillArgs &a, int num_sms, cudaStream_t st) { return BY_TYPE(forward_of); }
cudaError_t launch_distill_backward(const DistillArgs &a, int num_sms, cudaStream_t st) { return BY_TYPE(backward_of); }
cudaError_t launch_distill_step(const DistillArgs &a, int num_sms, cudaStream_t st) { return BY_TYPE(step_of); }
#undef BY_TYPE

}  // namespace rubick
