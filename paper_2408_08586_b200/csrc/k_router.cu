// Router of a mixture of experts with its balance loss: softmax over the experts, the k largest logits, their
// weights, and per group of rows the assignments and probability sums that the loss is made of; and its gradient.
//
//   loss = coef / groups * sum_g E / (k n_g^2) sum_e counts_ge S_ge,   S_ge = sum over the group's rows of p_e
//   dlogit_e = p_e (a_e - sum_j a_j p_j),  a_e = dloss coef E counts_ge / (groups k n_g^2),
//   and from the weights' gradients  + w_j (d_j - sum_i w_i d_i) at the chosen (weights that sum to one), or
//   + w_j d_j at the chosen and - p_e sum_i w_i d_i everywhere (raw weights).
//
// A row is spread over a power of two of lanes, EPL elements a lane, so that a warp works on 32 / lanes rows at once
// and nothing of a row leaves the registers.  The choice compares 32-bit keys whose unsigned order is that of the
// logits; the lowest index wins among equal ones.  Probability sums stay in the lane that owns the column until
// its chunk of rows ends, then go chunk by chunk, in order, into the group's sum: the last block of a group to arrive
// adds them up, the last group to arrive adds up the loss.

#include "train_common.cuh"

namespace rubick {

using namespace train;

namespace {

constexpr int ROUTER_THREADS = 256;
constexpr int ROUTER_WARPS = ROUTER_THREADS / 32;

// unsigned keys in the order of the values: -inf gets 0x007fffff, NaN of either sign 0 (never chosen)
__device__ __forceinline__ uint32_t order_key(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);          // -0 and 0 are equal
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0u;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_NINF = 0x007fffffu;

// column of element i of lane `sub` of a row
template <bool VEC, int VE> __device__ __forceinline__ int column(int i, int sub, int lanes)
{
    return VEC ? ((i / VE) * lanes + sub) * VE + i % VE : i * lanes + sub;
}

template <typename T, int EPL, bool VEC>
__device__ __forceinline__ void load_logits(const T *row, int sub, int lanes, int experts, float (&v)[EPL])
{
    constexpr int VE = Lanes<T>::N;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < EPL; i += VE) {
            const int c = column<VEC, VE>(i, sub, lanes);
            float part[VE];
            if (c + VE <= experts) unpack16<T>(ld_stream(row + c), part);
            else {
#pragma unroll
                for (int e = 0; e < VE; ++e) part[e] = c + e < experts ? to_f(row[c + e]) : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) v[i + e] = part[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const int c = column<VEC, VE>(i, sub, lanes);
            v[i] = c < experts ? to_f(row[c]) : -INFINITY;
        }
    }
}

__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) { const float t = __shfl_xor_sync(0xffffffffu, v, o); if (o < lanes) v += t; }
    return v;
}
__device__ __forceinline__ float lanes_max(float v, int lanes)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) { const float t = __shfl_xor_sync(0xffffffffu, v, o); if (o < lanes) v = fmaxf(v, t); }
    return v;
}

// What is left of a group once every row is counted: dot = sum_e counts_e S_e of this thread's experts
__device__ void finish_group(const RouterArgs &a, int64_t g, float dot, int valid)
{
    __shared__ float red[ROUTER_WARPS];
    dot = warp_sum(dot);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
        dot = 0.f;
        for (int w = 0; w < ROUTER_WARPS; ++w) dot += red[w];
        const float n = float(valid);
        a.valid[g] = valid;
        a.group_loss[g] = valid > 0 ? dot * float(a.d.experts) / (float(a.d.k) * n * n) : 0.f;
    }
}

// What the last block of a group does: the chunks' sums in chunk order
__device__ void join_group(const RouterArgs &a, int64_t g)
{
    const int E = a.d.experts, C = a.chunks;
    const int32_t *pc = a.part_counts + g * C * (E + 1);
    const float *ps = a.part + g * C * E;
    int valid = 0;
    for (int q = 0; q < C; ++q) valid += __ldcg(pc + int64_t(q) * (E + 1) + E);
    float dot = 0.f;
    for (int e = threadIdx.x; e < E; e += ROUTER_THREADS) {
        int n = 0;
        float s = 0.f;
#pragma unroll 4
        for (int q = 0; q < C; ++q) { n += __ldcg(pc + int64_t(q) * (E + 1) + e); s += __ldcg(ps + int64_t(q) * E + e); }
        a.counts[g * E + e] = n;
        a.prob_sum[g * E + e] = s;
        dot = fmaf(float(n), s, dot);
    }
    finish_group(a, g, dot, valid);
}

__device__ void join_loss(const RouterArgs &a)
{
    __shared__ float red[ROUTER_WARPS], cnt[ROUTER_WARPS];
    float s = 0.f, n = 0.f;
    for (int64_t g = threadIdx.x; g < a.groups; g += ROUTER_THREADS) {
        s += __ldcg(a.group_loss + g);
        n += __ldcg(a.valid + g) > 0 ? 1.f : 0.f;
    }
    s = warp_sum(s); n = warp_sum(n);
    if ((threadIdx.x & 31) == 0) { red[threadIdx.x >> 5] = s; cnt[threadIdx.x >> 5] = n; }
    __syncthreads();
    if (threadIdx.x == 0) {
        s = n = 0.f;
        for (int w = 0; w < ROUTER_WARPS; ++w) { s += red[w]; n += cnt[w]; }
        *a.loss = n > 0.f ? a.d.coef * s / n : 0.f;
    }
}

// blockIdx.x = chunk of rows within the group, blockIdx.y (and z) = group
template <typename T, int EPL, bool VEC>
__global__ void __launch_bounds__(ROUTER_THREADS) router_forward_kernel(const __grid_constant__ RouterArgs a, int lanes)
{
    constexpr int VE = Lanes<T>::N;
    extern __shared__ int32_t smem[];             // [E] assignments, then [warps][E] probability sums
    __shared__ int32_t valid_rows;
    __shared__ bool last;
    const int E = a.d.experts, k = a.d.k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane & (lanes - 1), per_warp = 32 / lanes;
    int32_t *hist = smem;
    float *psum = reinterpret_cast<float *>(smem + E);
    for (int e = threadIdx.x; e < E; e += ROUTER_THREADS) hist[e] = 0;
    if (threadIdx.x == 0) valid_rows = 0;
    __syncthreads();
    for (int64_t g = blockIdx.y; g < a.groups; g += gridDim.y) {
        const int64_t g0 = g * a.d.group_rows;
        const int64_t g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
        float acc[EPL];
#pragma unroll
        for (int i = 0; i < EPL; ++i) acc[i] = 0.f;
        int n_valid = 0;
        const int64_t stride = int64_t(a.chunks) * ROUTER_WARPS * per_warp;
        for (int64_t first = g0 + (int64_t(blockIdx.x) * ROUTER_WARPS + warp) * per_warp; first < g1; first += stride) {
            const int64_t row = first + lane / lanes;
            const bool here = row < g1, keep = here && (!a.mask || a.mask[row]);
            float v[EPL];
            load_logits<T, EPL, VEC>(static_cast<const T *>(a.logits) + (keep ? row : g0) * a.d.ld, sub, lanes, keep ? E : 0, v);
            uint32_t key[EPL];
            float top = -INFINITY, total = 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) { key[i] = order_key(v[i]); top = fmaxf(top, v[i]); }
            top = lanes_max(top, lanes);
            const bool some = top > -INFINITY;
            const float shift = some ? top : 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) { v[i] = some ? __expf(v[i] - shift) : 0.f; total += v[i]; }
            total = lanes_sum(total, lanes);
            const float inv = some ? 1.f / total : 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) acc[i] = fmaf(v[i], inv, acc[i]);
            n_valid += some && sub == 0 ? 1 : 0;
            // the k largest, one after the other: best of the lane, best of the row, out of the race
            float chosen_sum = 0.f;
            for (int j = 0; j < k; ++j) {
                uint32_t best = 0u;
                int col = 0x7fffffff;
#pragma unroll
                for (int i = 0; i < EPL; ++i)
                    if (key[i] > best) { best = key[i]; col = column<VEC, VE>(i, sub, lanes); }
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const uint32_t kb = __shfl_xor_sync(0xffffffffu, best, o);
                    const int cb = __shfl_xor_sync(0xffffffffu, col, o);
                    if (o < lanes && (kb > best || (kb == best && cb < col))) { best = kb; col = cb; }
                }
                const bool ok = best > KEY_NINF;
                const float w = ok ? __expf(__uint_as_float(best & 0x80000000u ? best & 0x7fffffffu : ~best) - shift) * inv : 0.f;
                chosen_sum += w;
#pragma unroll
                for (int i = 0; i < EPL; ++i) if (column<VEC, VE>(i, sub, lanes) == col) key[i] = 0u;
                if (j % lanes == sub) {
                    // lanes < k: a lane hands out several places; weights that are normalised are rewritten below
                    if (here) { a.index[row * k + j] = ok ? col : -1; a.weight[row * k + j] = w; }
                    if (here && ok) atomicAdd(&hist[col], 1);
                }
            }
            if ((a.d.flags & RUBICK_ROUTER_RENORM) && here && chosen_sum > 0.f)
                for (int j = sub; j < k; j += lanes) a.weight[row * k + j] = a.weight[row * k + j] / chosen_sum;
        }
        // rows of a warp, then warps of the block
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
#pragma unroll
            for (int o = 16; o; o >>= 1) { const float t = __shfl_xor_sync(0xffffffffu, acc[i], o); if (o >= lanes) acc[i] += t; }
            const int c = column<VEC, VE>(i, sub, lanes);
            if (lane < lanes && c < E) psum[warp * E + c] = acc[i];
        }
        n_valid = __reduce_add_sync(0xffffffffu, n_valid);
        if (lane == 0 && n_valid) atomicAdd(&valid_rows, n_valid);
        __syncthreads();
        const int64_t slot = g * a.chunks + blockIdx.x;
        const bool alone = a.chunks == 1;
        float dot = 0.f;
        for (int e = threadIdx.x; e < E; e += ROUTER_THREADS) {
            float s = 0.f;
            for (int w = 0; w < ROUTER_WARPS; ++w) s += psum[w * E + e];
            const int n = hist[e];
            hist[e] = 0;
            if (alone) {
                a.counts[g * E + e] = n;
                a.prob_sum[g * E + e] = s;
                dot = fmaf(float(n), s, dot);
            } else {
                __stcg(a.part + slot * E + e, s);
                __stcg(a.part_counts + slot * (E + 1) + e, n);
            }
        }
        const int rows_here = valid_rows;
        if (threadIdx.x == 0 && !alone) __stcg(a.part_counts + slot * (E + 1) + E, rows_here);
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            valid_rows = 0;
            last = alone || atomicAdd(a.tickets + g, 1u) == uint32_t(a.chunks - 1);
        }
        __syncthreads();
        if (last) {                                // every chunk of the group has arrived
            __threadfence();
            if (alone) finish_group(a, g, dot, rows_here);
            else join_group(a, g);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                if (!alone) a.tickets[g] = 0u;
                last = atomicAdd(a.tickets + a.groups, 1u) == uint32_t(a.groups - 1);
            }
            __syncthreads();
            if (last) {
                __threadfence();
                join_loss(a);
                if (threadIdx.x == 0) a.tickets[a.groups] = 0u;
            }
        }
        __syncthreads();
    }
}

template <typename T, int EPL, bool VEC>
__global__ void __launch_bounds__(ROUTER_THREADS) router_backward_kernel(const __grid_constant__ RouterArgs a, int lanes, int smem_cols)
{
    constexpr int VE = Lanes<T>::N;
    extern __shared__ float add[];                // [warps][rows of a warp][smem_cols]: what the weights' gradients add
    const int E = a.d.experts, k = a.d.k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane & (lanes - 1), per_warp = 32 / lanes;
    float *mine = add + (warp * per_warp + lane / lanes) * smem_cols;
    for (int c = sub; c < smem_cols; c += lanes) mine[c] = 0.f;
    __syncthreads();
    // groups that take part in the loss
    __shared__ float red[ROUTER_WARPS];
    float n = 0.f;
    for (int64_t g = threadIdx.x; g < a.groups; g += ROUTER_THREADS) n += a.valid_in[g] > 0 ? 1.f : 0.f;
    n = warp_sum(n);
    if (lane == 0) red[warp] = n;
    __syncthreads();
    n = 0.f;
    for (int w = 0; w < ROUTER_WARPS; ++w) n += red[w];
    const float pull = (a.dloss ? *a.dloss : 1.f) * a.d.coef * float(E) / (float(k) * fmaxf(n, 1.f));
    const bool renorm = a.d.flags & RUBICK_ROUTER_RENORM;
    const int64_t stride = int64_t(gridDim.x) * ROUTER_WARPS * per_warp;
    for (int64_t first = (int64_t(blockIdx.x) * ROUTER_WARPS + warp) * per_warp; first < a.d.rows; first += stride) {
        const int64_t row = first + lane / lanes;
        const bool here = row < a.d.rows, live = here && a.index_in[row * k] >= 0;
        float v[EPL];
        load_logits<T, EPL, VEC>(static_cast<const T *>(a.logits) + (live ? row : 0) * a.d.ld, sub, lanes, live ? E : 0, v);
        // the chosen: d_j w_j, and their sum over the row
        float wd = 0.f;
        if (live && a.dweight)
            for (int j = sub; j < k; j += lanes) wd = fmaf(a.weight_in[row * k + j], a.index_in[row * k + j] >= 0 ? a.dweight[row * k + j] : 0.f, wd);
        wd = lanes_sum(wd, lanes);
        if (live && a.dweight)
            for (int j = sub; j < k; j += lanes) {
                const int e = a.index_in[row * k + j];
                if (e >= 0 && e < E) atomicAdd(mine + e, a.weight_in[row * k + j] * (a.dweight[row * k + j] - (renorm ? wd : 0.f)));
            }
        float top = -INFINITY, total = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) top = fmaxf(top, v[i]);
        top = lanes_max(top, lanes);
        const float shift = top > -INFINITY ? top : 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) { v[i] = __expf(v[i] - shift); total += v[i]; }
        total = lanes_sum(total, lanes);
        const float inv = live ? 1.f / total : 0.f;
        const int64_t g = live ? row / a.d.group_rows : 0;
        const float m = fmaxf(float(a.valid_in[g]), 1.f), scale = pull / (m * m);
        float f[EPL], dot = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const int c = column<VEC, VE>(i, sub, lanes);
            f[i] = c < E ? scale * float(__ldg(a.counts_in + g * E + c)) : 0.f;
            v[i] *= inv;
            dot = fmaf(f[i], v[i], dot);
        }
        dot = lanes_sum(dot, lanes) + (renorm ? 0.f : wd);
        __syncwarp();
        T *out = static_cast<T *>(a.dlogits) + (here ? row : 0) * a.d.ld;
        const int end = here ? E : 0;
#pragma unroll
        for (int i = 0; i < EPL; i += VEC ? VE : 1) {
            const int c = column<VEC, VE>(i, sub, lanes);
            if constexpr (VEC) {
                float r[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float more = c + e < E ? mine[c + e] : 0.f;
                    r[e] = live ? fmaf(v[i + e], f[i + e] - dot, more) : 0.f;
                }
                store_cols<T, VE>(out, c, end, r);
            } else if (c < end) {
                out[c] = from_f<T>(live ? fmaf(v[i], f[i] - dot, mine[c]) : 0.f);
            }
        }
        __syncwarp();
        if (live && a.dweight)
            for (int j = sub; j < k; j += lanes) {
                const int e = a.index_in[row * k + j];
                if (e >= 0 && e < E) mine[e] = 0.f;
            }
        __syncwarp();
    }
}

struct RouterShape { int epl, lanes; bool vec; };

RouterShape router_shape(const RouterArgs &a)
{
    RouterShape s;
    const int es = a.d.dtype == RUBICK_F32 ? 4 : 2, ve = 16 / es;
    s.vec = aligned16(a.logits) && (!a.dlogits || aligned16(a.dlogits)) && a.d.ld * es % 16 == 0;
    s.epl = a.d.experts > 512 ? 32 : a.d.experts > 256 ? 16 : s.vec && ve == 4 && a.d.experts <= 128 ? 4 : 8;
    s.lanes = 1;
    while (s.lanes * s.epl < a.d.experts) s.lanes *= 2;
    return s;
}

template <typename T, bool BACK, int EPL, bool VEC> cudaError_t launch_router(const RouterArgs &a, const RouterShape &s, int num_sms, cudaStream_t st)
{
    if constexpr (BACK) {
        const int per_warp = 32 / s.lanes, cols = s.lanes * s.epl + 1;        // one word more: rows start in different banks
        const int smem = ROUTER_WARPS * per_warp * cols * int(sizeof(float));
        const int64_t blocks = (a.d.rows + ROUTER_WARPS * per_warp - 1) / (ROUTER_WARPS * per_warp);
        const int64_t most = int64_t(num_sms) * 8;
        router_backward_kernel<T, EPL, VEC><<<unsigned(blocks < most ? blocks : most), ROUTER_THREADS, smem, st>>>(a, s.lanes, cols);
    } else {
        const int smem = a.d.experts * int(sizeof(float)) * (ROUTER_WARPS + 1);
        router_forward_kernel<T, EPL, VEC><<<dim3(a.chunks, unsigned(a.groups < 32768 ? a.groups : 32768)), ROUTER_THREADS, smem, st>>>(a, s.lanes);
    }
    count_launch();
    return cudaGetLastError();
}

template <typename T, bool BACK> cudaError_t router_epl(const RouterArgs &a, int num_sms, cudaStream_t st)
{
    const RouterShape s = router_shape(a);
    if constexpr (sizeof(T) == 4)
        if (s.epl == 4) return launch_router<T, BACK, 4, true>(a, s, num_sms, st);
    if (s.epl == 8) return s.vec ? launch_router<T, BACK, 8, true>(a, s, num_sms, st) : launch_router<T, BACK, 8, false>(a, s, num_sms, st);
    if (s.epl == 16) return s.vec ? launch_router<T, BACK, 16, true>(a, s, num_sms, st) : launch_router<T, BACK, 16, false>(a, s, num_sms, st);
    return s.vec ? launch_router<T, BACK, 32, true>(a, s, num_sms, st) : launch_router<T, BACK, 32, false>(a, s, num_sms, st);
}

template <bool BACK> cudaError_t router_type(const RouterArgs &a, int num_sms, cudaStream_t st)
{
    switch (a.d.dtype) {
    case RUBICK_BF16: return router_epl<bf16, BACK>(a, num_sms, st);
    case RUBICK_F16: return router_epl<f16, BACK>(a, num_sms, st);
    default: return router_epl<float, BACK>(a, num_sms, st);
    }
}

}  // namespace

// blocks per group: enough to fill the SMs, at least one pass of a block's warps each
int router_chunks(const RouterArgs &a, int num_sms)
{
    const RouterShape s = router_shape(a);
    const int64_t rows = a.d.group_rows < a.d.rows ? a.d.group_rows : a.d.rows;
    const int64_t most = (rows + ROUTER_WARPS * (32 / s.lanes) - 1) / (ROUTER_WARPS * (32 / s.lanes));
    const int64_t want = (int64_t(num_sms) * 4 + a.groups - 1) / a.groups;
    return int(most < want ? most : want);
}

cudaError_t launch_router_forward(const RouterArgs &a, int num_sms, cudaStream_t st) { return router_type<false>(a, num_sms, st); }
cudaError_t launch_router_backward(const RouterArgs &a, int num_sms, cudaStream_t st) { return router_type<true>(a, num_sms, st); }

}  // namespace rubick
