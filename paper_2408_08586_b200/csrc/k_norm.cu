// The edge between two blocks of a transformer: norm after the block, gate, scaled residual sum, norm before the
// next block, in one pass over the rows, forward and backward.
//
// With a = rstd(y), b = rstd(x'), W = w + o, k = alpha g a W_after:
//   forward   x' = x + k y,  h = x' b W_before
//   backward  xh = x' b, e = dh W_before, D = columns:
//             G  = dx' + b (e - xh m1),   m1 = mean(e xh)                 (gradient of the stream; dx = G)
//             yh = y a, f = alpha g W_after G,
//             dy = a (f - yh m2),         m2 = mean(f yh)
//             dW_before = sum dh xh,  dW_after = sum alpha g G yh,  dgate = g' sum_group alpha G yh W_after.
// The backward pass needs m1 before G and G before m2.  m2 is linear in G, so with q = alpha g W_after yh it is
//   D m2 = sum q (dx' + b e) - b m1 sum q xh,
// and the three sums (e xh, q (dx' + b e), q xh) come from one reduction: one barrier a row instead of two.
//
// 4 row elements move per column forward, 6 backward, for a dozen operations: the floor is memory's.  Many rows travel
// through a ring of shared-memory stages; few rows forward stay in the registers of a warp or a block between their loads and
// their stores; rows too wide for the ring backward are read twice.
//
// Measured on a B200 (6.54 TB/s copy): forward 8,192 x 5,120 bf16 71 us = 4.7 TB/s, backward 16,384 x 4,096 bf16
// 151 us = 5.3 TB/s with its join, 2,048 x 1,280 fp16 24 us (13 the rows, 8 the join, which reads again what 683 runs of
// three rows have left: 10 MB beside 31 MB of rows); 1,000 x 1,537 fp32 forward 8.2 us; four rows 5 us; over 8,192 columns
// 2,048 x 16,384 bf16 forward 129 us = 2.1 TB/s, backward 520 us = 0.8 TB/s (one block of 512 threads an SM, every row twice).

#include "train_common.cuh"

namespace rubick {

using namespace train;

namespace {

// tanh(x) and its slope 4 e / (1 + e)^2, e = e^(-2|x|), which keeps its digits where tanh is close to one (1 - tanh^2
// does not).
__device__ __forceinline__ float tanh_slope(float x, float &slope)
{
    const float e = expf(-2.f * fabsf(x)), inv = __fdividef(1.f, 1.f + e);
    slope = 4.f * e * inv * inv;
    return tanhf(x);
}

// sum of v[0..N) over the TPR threads of a row; `red` has a slot per warp of the block, alternated by the caller
template <int N> __device__ __forceinline__ void row_sum(float (&v)[N], float *red, int warps, int row_slot)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if (warps == 1) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *mine = red + row_slot * warps * N;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) mine[warp * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < warps ? mine[lane * N + i] : 0.f);
}

template <typename T, typename W, int VE, int NV>
__global__ void __launch_bounds__(NV == 1 ? 1024 : 512) norm_forward_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float red[2][32];
    const int tpr = blockDim.x, warps = tpr >> 5, cols = a.d.cols;
    const int64_t row = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
    const bool live = row < a.d.rows;
    const int end = live ? cols : 0;              // a row slot past the end only takes part in the barriers
    const T *x = static_cast<const T *>(a.x) + row * a.d.ld_x;
    float v[NV][VE];
#pragma unroll
    for (int i = 0; i < NV; ++i) load_cols<T, VE>(x, (i * tpr + int(threadIdx.x)) * VE, end, v[i]);
    const float o = a.d.flags & RUBICK_NORM_UNIT_OFFSET ? 1.f : 0.f;
    const float inv_cols = 1.f / float(cols);
    float rstd_after = 0.f, rstd_before = 0.f;
    if (a.y) {
        const T *y = static_cast<const T *>(a.y) + row * a.d.ld_y;
        float u[NV][VE];
#pragma unroll
        for (int i = 0; i < NV; ++i) load_cols<T, VE>(y, (i * tpr + int(threadIdx.x)) * VE, end, u[i]);
        float scale = a.d.alpha;
        if (a.d.flags & RUBICK_NORM_AFTER) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VE; ++e) s[0] = fmaf(u[i][e], u[i][e], s[0]);
            row_sum<1>(s, red[0], warps, threadIdx.y);
            rstd_after = rsqrtf(s[0] * inv_cols + a.d.eps);
            scale *= rstd_after;
            if (a.w_after) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float w[VE];
                    load_shared_cols<W, VE>(static_cast<const W *>(a.w_after), (i * tpr + int(threadIdx.x)) * VE, end, w, 0.f);
#pragma unroll
                    for (int e = 0; e < VE; ++e) u[i][e] *= w[e] + o;
                }
            }
        }
        if (a.gate && live) {
            const T *gate = static_cast<const T *>(a.gate) + (row / a.d.group_rows) * a.d.ld_gate;
            const bool th = a.d.flags & RUBICK_NORM_TANH_GATE;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float g[VE];
                load_shared_cols<T, VE>(gate, (i * tpr + int(threadIdx.x)) * VE, end, g, 0.f);
#pragma unroll
                for (int e = 0; e < VE; ++e) u[i][e] *= th ? tanhf(g[e]) : g[e];
            }
        }
        T *x_out = static_cast<T *>(a.x_out) + row * a.d.ld_x;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < VE; ++e) v[i][e] = fmaf(scale, u[i][e], v[i][e]);
            store_cols<T, VE>(x_out, (i * tpr + int(threadIdx.x)) * VE, end, v[i]);
        }
    }
    if (a.d.flags & RUBICK_NORM_BEFORE) {
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) s[0] = fmaf(v[i][e], v[i][e], s[0]);
        row_sum<1>(s, red[1], warps, threadIdx.y);
        rstd_before = rsqrtf(s[0] * inv_cols + a.d.eps);
        T *h = static_cast<T *>(a.h) + row * a.d.ld_h;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * tpr + int(threadIdx.x)) * VE;
            float w[VE], r[VE];
            if (a.w_before) load_shared_cols<W, VE>(static_cast<const W *>(a.w_before), c, end, w, 0.f);
#pragma unroll
            for (int e = 0; e < VE; ++e) r[e] = v[i][e] * rstd_before * (a.w_before ? w[e] + o : 1.f);
            store_cols<T, VE>(h, c, end, r);
        }
    }
    if (a.rstd && live && threadIdx.x == 0) { a.rstd[2 * row] = rstd_after; a.rstd[2 * row + 1] = rstd_before; }
}

// Scratch of the backward pass, per row chunk c and column: [dW_after | dW_before | gate group that began before the
// chunk | gate group that began in the chunk and goes on behind it], each [n_chunks][cols].
__device__ __forceinline__ float *part_row(const NormArgs &a, int which, int chunk)
{
    return a.part + (int64_t(which) * a.n_chunks + chunk) * a.d.cols;
}

// One chunk has the weights' sums whole: the ring writes them to their places, sixteen bytes at a time, where these allow it.
__host__ __device__ __forceinline__ bool sums_go_straight(const NormArgs &a)
{
    return a.n_chunks == 1 && ((reinterpret_cast<uintptr_t>(a.dw_after) | reinterpret_cast<uintptr_t>(a.dw_before)) & 15) == 0;
}

// Rows too wide for the ring below: the column sums are in shared memory, and a row is read twice (the second time from
// L2), once for its sums and once for its gradients.
template <typename T, typename W, int VE>
__global__ void __launch_bounds__(512) norm_backward_wide_kernel(const __grid_constant__ NormArgs a)
{
    extern __shared__ float sums[];               // [3][cols]: dW_after, dW_before, gate
    __shared__ float red[2][3 * 32];
    const int warps = blockDim.x >> 5, cols = a.d.cols, chunk = blockIdx.x;
    const int64_t begin = chunk * a.chunk_rows;
    const int64_t stop = begin + a.chunk_rows < a.d.rows ? begin + a.chunk_rows : a.d.rows;
    const bool after = a.d.flags & RUBICK_NORM_AFTER, before = a.d.flags & RUBICK_NORM_BEFORE;
    const bool th = a.d.flags & RUBICK_NORM_TANH_GATE, need_y = a.y && (after || a.gate);
    const float o = a.d.flags & RUBICK_NORM_UNIT_OFFSET ? 1.f : 0.f;
    const float inv_cols = 1.f / float(cols);
    // every thread owns the columns it visits: no barrier is needed around the sums
    for (int c = int(threadIdx.x) * VE; c < cols; c += int(blockDim.x) * VE)
        for (int e = 0; e < VE && c + e < cols; ++e) sums[c + e] = sums[cols + c + e] = sums[2 * cols + c + e] = 0.f;
    int64_t group = -1, group_end = begin;
    for (int64_t row = begin; row <= stop; ++row) {
        if (a.gate && (row == stop || row >= group_end)) {
            if (group >= 0 && a.dgate) {
                const int64_t g0 = group * a.d.group_rows, g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
                const bool whole = g0 >= begin && g1 <= stop;
                const T *gate = static_cast<const T *>(a.gate) + group * a.d.ld_gate;
                for (int c = int(threadIdx.x) * VE; c < cols; c += int(blockDim.x) * VE)
                    for (int e = 0; e < VE && c + e < cols; ++e) {
                        float v = sums[2 * cols + c + e];
                        if (th) { float slope; tanh_slope(to_f(gate[c + e]), slope); v *= slope; }
                        if (whole) static_cast<T *>(a.dgate)[group * a.d.ld_gate + c + e] = from_f<T>(v);
                        else part_row(a, g0 < begin ? 2 : 3, chunk)[c + e] = v;
                        sums[2 * cols + c + e] = 0.f;
                    }
            }
            group = row < stop ? row / a.d.group_rows : -1;
            group_end = (group + 1) * a.d.group_rows;
        }
        if (row == stop) break;
        const float ra = after ? a.rstd_in[2 * row] : 1.f, rb = before ? a.rstd_in[2 * row + 1] : 0.f;
        float m1 = 0.f, m2 = 0.f, s[3] = {0.f, 0.f, 0.f};
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            for (int c = int(threadIdx.x) * VE; c < cols; c += int(blockDim.x) * VE) {
                float dxo[VE], xh[VE], dh[VE], yh[VE], g[VE], wa[VE], wb[VE], dx[VE], dy[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) { dxo[e] = xh[e] = dh[e] = yh[e] = 0.f; g[e] = 1.f; wa[e] = wb[e] = 1.f - o; }
                if (a.dx_out) load_cols<T, VE>(static_cast<const T *>(a.dx_out) + row * a.d.ld_x, c, cols, dxo);
                if (before) load_cols<T, VE>(static_cast<const T *>(a.x) + row * a.d.ld_x, c, cols, xh);
                if (before) load_cols<T, VE>(static_cast<const T *>(a.dh) + row * a.d.ld_h, c, cols, dh);
                if (need_y) load_cols<T, VE>(static_cast<const T *>(a.y) + row * a.d.ld_y, c, cols, yh);
                if (a.gate) load_shared_cols<T, VE>(static_cast<const T *>(a.gate) + group * a.d.ld_gate, c, cols, g, 0.f);
                if (a.w_after) load_shared_cols<W, VE>(static_cast<const W *>(a.w_after), c, cols, wa, 0.f);
                if (a.w_before) load_shared_cols<W, VE>(static_cast<const W *>(a.w_before), c, cols, wb, 0.f);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    if (th) g[e] = tanhf(g[e]);
                    xh[e] *= rb; yh[e] *= ra;
                    const float ew = dh[e] * (wb[e] + o), w = wa[e] + o;
                    if (pass == 0) {
                        const float q = a.d.alpha * g[e] * w * yh[e];
                        s[0] = fmaf(ew, xh[e], s[0]);
                        s[1] = fmaf(q, fmaf(rb, ew, dxo[e]), s[1]);
                        s[2] = fmaf(q, xh[e], s[2]);
                    } else {
                        dx[e] = fmaf(rb, ew - xh[e] * m1, dxo[e]);
                        const float f = a.d.alpha * dx[e], fg = f * g[e];
                        dy[e] = after ? ra * (fg * w - yh[e] * m2) : fg;
                        if (c + e < cols) {
                            sums[c + e] = fmaf(fg, yh[e], sums[c + e]);
                            sums[cols + c + e] = fmaf(dh[e], xh[e], sums[cols + c + e]);
                            sums[2 * cols + c + e] = fmaf(f * w, yh[e], sums[2 * cols + c + e]);
                        }
                    }
                }
                if (pass) {
                    store_cols<T, VE>(static_cast<T *>(a.dx) + row * a.d.ld_x, c, cols, dx);
                    if (a.dy) store_cols<T, VE>(static_cast<T *>(a.dy) + row * a.d.ld_y, c, cols, dy);
                }
            }
            if (pass == 0) {
                row_sum<3>(s, red[(row - begin) & 1], warps, 0);
                m1 = s[0] * inv_cols;
                m2 = after ? (s[1] - rb * m1 * s[2]) * inv_cols : 0.f;
            }
        }
    }
    for (int c = int(threadIdx.x) * VE; c < cols; c += int(blockDim.x) * VE)
        for (int e = 0; e < VE && c + e < cols; ++e) {
            if (a.dw_after) part_row(a, 0, chunk)[c + e] = sums[c + e];
            if (a.dw_before) part_row(a, 1, chunk)[c + e] = sums[cols + c + e];
        }
}

// ---- rows through a ring of shared-memory stages ---------------------------------------------------------------
//
// A block takes a run of consecutive rows and one thread copies them with the bulk-copy engine, several rows ahead: the
// copies in flight do not depend on how many warps are waiting, and a row that waits for its sums holds no registers.
// Rows that are a whole number of 16-byte units are read and written 16 bytes at a time.  Others are copied with the
// units that they begin and end in and taken element by element, column c by thread c mod (threads), so that a column
// stays with its thread whatever the row's place in its unit.  What is the same for all rows of a gate group,
// k = alpha g W_after, is kept per column; a column's gradients of gate and weight are both
// sum G yh times a factor of the group, so one running sum serves both:
//   dgate = g' alpha W_after t,   dW_after += alpha g t,   t = sum over the group's rows of G yh.

//
// Forward 8,192 x 5,120 bf16 took 182 us and backward 16,384 x 4,096 335 us with rows loaded straight into registers:
// half the warps waited for memory, the registers left no room for more of them.
constexpr int RING_MOST = 8;      // stages

struct Ring {
    int stages, tensors;
    int i_x, i_y, i_dxo, i_dh, i_gate;    // place of a tensor in a stage, -1: not copied
    uint32_t slot_bytes;                  // of a row in a stage
};

// A thread's i-th set of columns: VE neighbours, or (VEC = false) two that are a row of threads apart
template <typename T, bool VEC> struct Cols {
    static constexpr int VE = VEC ? Lanes<T>::N : 2, VP = VE / 2;
    static __device__ __forceinline__ int first(int i, int tpr) { return VEC ? (i * tpr + int(threadIdx.x)) * VE : 2 * i * tpr + int(threadIdx.x); }
    static __device__ __forceinline__ void load(const T *from, int c, int tpr, int cols, f2 (&v)[VP])
    {
        if constexpr (VEC) unpack16<T>(*reinterpret_cast<const uint4 *>(from + c), v);
        else v[0] = pair(to_f(from[c]), c + tpr < cols ? to_f(from[c + tpr]) : 0.f);
    }
    static __device__ __forceinline__ void store(T *to, int c, int tpr, int cols, const f2 (&v)[VP])
    {
        if constexpr (VEC) {
            st_stream(to + c, pack16<T>(v));
        } else {
            to[c] = from_f<T>(lo(v[0]));
            if (c + tpr < cols) to[c + tpr] = from_f<T>(hi(v[0]));
        }
    }
    template <typename W> static __device__ __forceinline__ void weights(const W *from, int c, int tpr, int cols, float (&v)[VE])
    {
        if constexpr (VEC) load_shared_cols<W, VE>(from, c, cols, v, 0.f);
        else { v[0] = to_f(from[c]); v[1] = c + tpr < cols ? to_f(from[c + tpr]) : 0.f; }
    }
    static __device__ __forceinline__ void put(float *to, int c, int tpr, int cols, const f2 (&v)[VP])
    {
        if constexpr (VEC) {
#pragma unroll
            for (int e = 0; e < VP; e += 2) *reinterpret_cast<ulonglong2 *>(to + c + 2 * e) = make_ulonglong2(v[e], v[e + 1]);
        } else {
            to[c] = lo(v[0]);
            if (c + tpr < cols) to[c + tpr] = hi(v[0]);
        }
    }
};

// One barrier for the threads of a block (a warp where it is one).
__device__ __forceinline__ void row_barrier(int warps) { if (warps == 1) __syncwarp(); else __syncthreads(); }

// Sums of N values over the block; red: N x 16 words, those of absent warps 0.  Every thread adds up the warps' sums
// itself: a handful of 16-byte loads instead of a second chain of shuffles.
template <int N> __device__ __forceinline__ void ring_sum(const f2 (&in)[N], float (&v)[N], float *red, int warps)
{
    static_assert(N == 1 || N == 3, "one sum or three");
    const int lane = threadIdx.x & 31;
    if constexpr (N == 1) {
        v[0] = warp_sum(lo(in[0]) + hi(in[0]));
        if (warps > 1 && lane == 0) red[threadIdx.x >> 5] = v[0];
    } else {
        // two exchanges leave a quarter of the warp with one sum each (the fourth is 0), three more steps finish it:
        // 6 shuffles instead of 15
        const float a0 = lo(in[0]) + hi(in[0]), a1 = lo(in[1]) + hi(in[1]), a2 = lo(in[2]) + hi(in[2]);
        const bool up = lane & 16, odd = lane & 8;
        const float x0 = (up ? a2 : a0) + __shfl_xor_sync(0xffffffffu, up ? a0 : a2, 16);
        const float x1 = (up ? 0.f : a1) + __shfl_xor_sync(0xffffffffu, up ? a1 : 0.f, 16);
        float z = (odd ? x1 : x0) + __shfl_xor_sync(0xffffffffu, odd ? x0 : x1, 8);
#pragma unroll
        for (int o = 4; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        if (warps == 1) {
            v[0] = __shfl_sync(0xffffffffu, z, 0); v[1] = __shfl_sync(0xffffffffu, z, 8); v[2] = __shfl_sync(0xffffffffu, z, 16);
        } else if ((lane & 7) == 0 && lane < 24) {
            red[(lane >> 3) * 16 + (threadIdx.x >> 5)] = z;
        }
    }
    if (warps == 1) { __syncwarp(); return; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = 0; w < warps; w += 4)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float4 t = *reinterpret_cast<const float4 *>(red + i * 16 + w);
            v[i] += (t.x + t.y) + (t.z + t.w);
        }
}

// The copies of row `row` into stage `s`, by one warp: by its first lane, or, where rows are ragged, lane t copies the
// t-th tensor's (x, y, dx_out, dh, gate).  Ragged rows come with the 16-byte units that they begin and end in; units that
// may reach out of the tensor itself (of rows that begin or end less than 16 bytes from the tensor's own ends: the first and
// the last, and more where rows are short) are put together by the lanes, element by element, eight lanes a tensor.
template <typename T, bool VEC> __device__ __forceinline__ void ring_issue(const NormArgs &a, const Ring &r, uint8_t *smem, uint64_t *bars, int s, int64_t row)
{
    const int lane = threadIdx.x & 31;
    uint8_t *stage = smem + size_t(s) * r.tensors * r.slot_bytes;
    if constexpr (VEC) {
        if (lane) return;
        bar_expect(bars + s, r.slot_bytes * r.tensors);
        if (r.i_x >= 0) bulk_load(stage + r.i_x * r.slot_bytes, static_cast<const T *>(a.x) + row * a.d.ld_x, r.slot_bytes, bars + s);
        if (r.i_y >= 0) bulk_load(stage + r.i_y * r.slot_bytes, static_cast<const T *>(a.y) + row * a.d.ld_y, r.slot_bytes, bars + s);
        if (r.i_dxo >= 0) bulk_load(stage + r.i_dxo * r.slot_bytes, static_cast<const T *>(a.dx_out) + row * a.d.ld_x, r.slot_bytes, bars + s);
        if (r.i_dh >= 0) bulk_load(stage + r.i_dh * r.slot_bytes, static_cast<const T *>(a.dh) + row * a.d.ld_h, r.slot_bytes, bars + s);
        if (r.i_gate >= 0) bulk_load(stage + r.i_gate * r.slot_bytes, static_cast<const T *>(a.gate) + (row / a.d.group_rows) * a.d.ld_gate, r.slot_bytes, bars + s);
    } else {
        const int place = lane == 0 ? r.i_x : lane == 1 ? r.i_y : lane == 2 ? r.i_dxo : lane == 3 ? r.i_dh : lane == 4 ? r.i_gate : -1;
        const bool gate = lane == 4, copied = place >= 0;
        const void *base = lane == 0 ? a.x : lane == 1 ? a.y : lane == 2 ? a.dx_out : lane == 3 ? a.dh : a.gate;
        const int64_t ld = lane == 0 || lane == 2 ? a.d.ld_x : lane == 1 ? a.d.ld_y : lane == 3 ? a.d.ld_h : a.d.ld_gate;
        const int64_t at = gate && copied ? row / a.d.group_rows : row;
        const int64_t left = gate && copied ? int64_t(uint32_t(a.d.rows - 1) / uint32_t(a.d.group_rows)) - at : a.d.rows - 1 - at;      // rows behind it
        const uintptr_t p = copied ? reinterpret_cast<uintptr_t>(base) + uintptr_t(at * ld) * sizeof(T) : 0;
        const uint32_t my_slot = copied ? place * r.slot_bytes : 0u;
        const uint32_t bytes = a.d.cols * uint32_t(sizeof(T));
        constexpr int64_t near = 16 / int64_t(sizeof(T));
        const bool first = at * ld < near, last = left * ld < near;
        // first whole unit, and the end of the last one
        const uintptr_t low = p & ~uintptr_t(15), end = p + bytes;
        const uintptr_t b0 = first ? (p + 15) & ~uintptr_t(15) : low;
        uintptr_t b1 = last ? end & ~uintptr_t(15) : (end + 15) & ~uintptr_t(15);
        if (b1 < b0) b1 = b0;                     // (within one unit: all of it by hand)
        if (__any_sync(0xffffffffu, copied && (first || last))) {
#pragma unroll
            for (int t0 = 0; t0 < 8; t0 += 4) {
                const int t = t0 + (lane >> 3);
                const uintptr_t tp = __shfl_sync(0xffffffffu, (unsigned long long)p, t);
                const uintptr_t tb0 = __shfl_sync(0xffffffffu, (unsigned long long)b0, t), tb1 = __shfl_sync(0xffffffffu, (unsigned long long)b1, t);
                const uint32_t slot = __shfl_sync(0xffffffffu, my_slot, t);
                const uintptr_t tend = tp + bytes, tlow = tp & ~uintptr_t(15);
                const uintptr_t head = tp + (lane & 7) * sizeof(T), tail = tb1 + (lane & 7) * sizeof(T);
                const bool has_head = tp && head < tb0 && head < tend, has_tail = tp && tail < tend && tail >= tb0 && tail >= tp;
                T h, e;
                if (has_head) h = *reinterpret_cast<const T *>(head);
                if (has_tail) e = *reinterpret_cast<const T *>(tail);
                if (has_head) *reinterpret_cast<T *>(stage + slot + (head - tlow)) = h;
                if (has_tail) *reinterpret_cast<T *>(stage + slot + (tail - tlow)) = e;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // a later copy comes behind these stores
        }
        const uint32_t mine = copied ? uint32_t(b1 - b0) : 0u, total = __reduce_add_sync(0xffffffffu, mine);
        __syncwarp();                             // the stores of all lanes come before the arrival that stands for them
        if (lane == 0) bar_expect(bars + s, total);
        __syncwarp();
        if (mine) bulk_load(stage + my_slot + (b0 - low), reinterpret_cast<const void *>(b0), mine, bars + s);
    }
}

// the row of a tensor in a stage: where its unit begins, or its place in it
template <typename T, bool VEC> __device__ __forceinline__ const T *stage_row(const uint8_t *stage, const Ring &r, int place, const void *base, int64_t row, int64_t ld)
{
    const uint32_t shift = VEC ? 0u : (uint32_t(reinterpret_cast<uintptr_t>(base)) + uint32_t(row) * uint32_t(ld) * uint32_t(sizeof(T))) & 15u;
    return reinterpret_cast<const T *>(stage + place * r.slot_bytes + shift);
}

template <int VP> __device__ __forceinline__ void zero_cols(f2 (&v)[VP])
{
#pragma unroll
    for (int e = 0; e < VP; ++e) v[e] = 0ull;
}

// k = alpha g W_after of this thread's columns for the gate row at `gate` (NULL: g = 1)
template <typename T, typename W, bool VEC, int NV>
__device__ __forceinline__ void group_factors(const NormArgs &a, const T *gate, int tpr, float o, f2 (&k)[NV][Cols<T, VEC>::VP])
{
    using C = Cols<T, VEC>;
    const bool th = a.d.flags & RUBICK_NORM_TANH_GATE;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = C::first(i, tpr);
        float w[C::VE];
        f2 g[C::VP];
#pragma unroll
        for (int e = 0; e < C::VE; ++e) { w[e] = 1.f - o; g[e / 2] = both(1.f); }
        if (c < a.d.cols) {
            if (a.w_after) C::weights(static_cast<const W *>(a.w_after), c, tpr, a.d.cols, w);
            if (gate) C::load(gate, c, tpr, a.d.cols, g);
        }
#pragma unroll
        for (int e = 0; e < C::VP; ++e) {
            const float g0 = th ? tanhf(lo(g[e])) : lo(g[e]), g1 = th ? tanhf(hi(g[e])) : hi(g[e]);
            k[i][e] = pair(a.d.alpha * g0 * (w[2 * e] + o), a.d.alpha * g1 * (w[2 * e + 1] + o));
        }
    }
}

// W_before of this thread's columns
template <typename T, typename W, bool VEC, int NV> __device__ __forceinline__ void before_factors(const NormArgs &a, int tpr, float o, f2 (&wb)[NV][Cols<T, VEC>::VP])
{
    using C = Cols<T, VEC>;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = C::first(i, tpr);
        float w[C::VE];
#pragma unroll
        for (int e = 0; e < C::VE; ++e) w[e] = 1.f - o;
        if (a.w_before && c < a.d.cols) C::weights(static_cast<const W *>(a.w_before), c, tpr, a.d.cols, w);
#pragma unroll
        for (int e = 0; e < C::VP; ++e) wb[i][e] = pair(w[2 * e] + o, w[2 * e + 1] + o);
    }
}

// FULL: both norms and a block between them, known when the kernel is compiled; 96 registers: 640 threads an SM
template <typename T, typename W, int NV, bool FULL, bool VEC>
__global__ void __maxnreg__(NV == 1 ? 64 : 96) norm_forward_ring_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ Ring r)
{
    using C = Cols<T, VEC>;
    constexpr int VP = C::VP;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float red[4][16];                  // one row's sums may still be read when the next row's are written
    __shared__ __align__(8) uint64_t bars[RING_MOST];
    const int tpr = blockDim.x, warps = tpr >> 5, cols = a.d.cols;
    const int64_t begin = blockIdx.x * a.chunk_rows;
    const int n = int(begin + a.chunk_rows < a.d.rows ? a.chunk_rows : a.d.rows - begin);
    if (threadIdx.x == 0) {
        for (int s = 0; s < r.stages; ++s) bar_init(bars + s);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (threadIdx.x < 32)
        for (int s = 0; s < r.stages && s < n; ++s) ring_issue<T, VEC>(a, r, smem, bars, s, begin + s);
    if (threadIdx.x < 32) {                       // the 64 words by one warp: the smallest block has no more
        (&red[0][0])[threadIdx.x] = 0.f;
        (&red[0][0])[threadIdx.x + 32] = 0.f;
    }
    const bool block = FULL || a.y, after = FULL || (a.d.flags & RUBICK_NORM_AFTER), before = FULL || (a.d.flags & RUBICK_NORM_BEFORE);
    const float o = a.d.flags & RUBICK_NORM_UNIT_OFFSET ? 1.f : 0.f, inv_cols = 1.f / float(cols);
    f2 wb[NV][VP], k[NV][VP];
    before_factors<T, W, VEC, NV>(a, tpr, o, wb);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VP; ++e) k[i][e] = 0ull;
    __syncthreads();
    T *x_out = static_cast<T *>(a.x_out) + begin * a.d.ld_x, *h = static_cast<T *>(a.h) + begin * a.d.ld_h;
    int64_t group_end = begin;
    bool lost = false;
    int s = 0;
    uint32_t parity = 0;
    for (int i_row = 0; i_row < n; ++i_row) {
        const int64_t row = begin + i_row;
        const uint8_t *stage = smem + size_t(s) * r.tensors * r.slot_bytes;
        if (!lost && !bar_wait(bars + s, parity)) { lost = true; atomicOr(a.status, DS_COPY_LOST); }
        const T *x_row = stage_row<T, VEC>(stage, r, r.i_x, a.x, row, a.d.ld_x), *y_row = stage_row<T, VEC>(stage, r, r.i_y, a.y, row, a.d.ld_y);
        if (block && row >= group_end) {
            const int64_t group = row / a.d.group_rows;
            group_end = (group + 1) * a.d.group_rows;
            const T *gate = !a.gate ? nullptr : r.i_gate >= 0 ? stage_row<T, VEC>(stage, r, r.i_gate, a.gate, row / a.d.group_rows, a.d.ld_gate)
                                                              : static_cast<const T *>(a.gate) + group * a.d.ld_gate;
            group_factors<T, W, VEC, NV>(a, gate, tpr, o, k);
        }
        f2 v[NV][VP], y[NV][VP], part[1] = {0ull};
        float sum[1], ra = 0.f, rb = 0.f, scale = 1.f;
        if (after) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = C::first(i, tpr);
                if (c < cols) {
                    C::load(y_row, c, tpr, cols, y[i]);
#pragma unroll
                    for (int e = 0; e < VP; ++e) part[0] = fma2(y[i][e], y[i][e], part[0]);
                }
            }
            ring_sum<1>(part, sum, red[i_row & 1], warps);
            scale = ra = rsqrtf(sum[0] * inv_cols + a.d.eps);
        } else row_barrier(warps);
        // every thread has left the stage of the row before
        if (threadIdx.x < 32 && i_row >= 1 && i_row - 1 + r.stages < n)
            ring_issue<T, VEC>(a, r, smem, bars, s ? s - 1 : r.stages - 1, row - 1 + r.stages);
        part[0] = 0ull;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = C::first(i, tpr);
            if (c < cols) {
                C::load(x_row, c, tpr, cols, v[i]);
                if (block) {
                    if (!after) C::load(y_row, c, tpr, cols, y[i]);
#pragma unroll
                    for (int e = 0; e < VP; ++e) v[i][e] = fma2(mul2(k[i][e], both(scale)), y[i][e], v[i][e]);
                    C::store(x_out, c, tpr, cols, v[i]);
                }
#pragma unroll
                for (int e = 0; e < VP; ++e) part[0] = fma2(v[i][e], v[i][e], part[0]);
            }
        }
        if (before) {
            ring_sum<1>(part, sum, red[2 + (i_row & 1)], warps);
            rb = rsqrtf(sum[0] * inv_cols + a.d.eps);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = C::first(i, tpr);
                if (c < cols) {
#pragma unroll
                    for (int e = 0; e < VP; ++e) v[i][e] = mul2(mul2(v[i][e], both(rb)), wb[i][e]);
                    C::store(h, c, tpr, cols, v[i]);
                }
            }
        }
        if (a.rstd && threadIdx.x == 0) *reinterpret_cast<float2 *>(a.rstd + 2 * row) = make_float2(ra, rb);
        x_out += a.d.ld_x;
        h += a.d.ld_h;
        if (++s == r.stages) { s = 0; parity ^= 1u; }
    }
}

// the gradients of a gate group whose rows this chunk has summed up in t
template <typename T, typename W, bool VEC, int NV>
__device__ __forceinline__ void ring_flush(const NormArgs &a, int chunk, int64_t begin, int64_t stop, int64_t group, const T *gate, int tpr, float o,
                                           f2 (&t)[NV][Cols<T, VEC>::VP], f2 (&acc_a)[NV][Cols<T, VEC>::VP])
{
    using C = Cols<T, VEC>;
    const int64_t g0 = group * a.d.group_rows;
    const int64_t g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
    const bool whole = g0 >= begin && g1 <= stop, th = a.d.flags & RUBICK_NORM_TANH_GATE;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = C::first(i, tpr);
        if (c >= a.d.cols) continue;
        float w[C::VE];
        f2 g[C::VP], d[C::VP];
#pragma unroll
        for (int e = 0; e < C::VE; ++e) { w[e] = 1.f - o; g[e / 2] = both(1.f); }
        if (a.w_after) C::weights(static_cast<const W *>(a.w_after), c, tpr, a.d.cols, w);
        if (gate) C::load(gate, c, tpr, a.d.cols, g);
#pragma unroll
        for (int e = 0; e < C::VP; ++e) {
            float s0 = 1.f, s1 = 1.f, g0f = lo(g[e]), g1f = hi(g[e]);
            if (th) { g0f = tanh_slope(g0f, s0); g1f = tanh_slope(g1f, s1); }
            const f2 at = mul2(both(a.d.alpha), t[i][e]);
            acc_a[i][e] = fma2(pair(g0f, g1f), at, acc_a[i][e]);
            d[e] = mul2(at, pair((w[2 * e] + o) * s0, (w[2 * e + 1] + o) * s1));
            t[i][e] = 0ull;
        }
        if (!a.dgate) continue;
        if (whole) C::store(static_cast<T *>(a.dgate) + group * a.d.ld_gate, c, tpr, a.d.cols, d);
        else C::put(part_row(a, g0 < begin ? 2 : 3, chunk), c, tpr, a.d.cols, d);
    }
}

template <typename T, typename W, int NV, bool FULL, bool VEC>
__global__ void __launch_bounds__(512) norm_backward_ring_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ Ring r)
{
    using C = Cols<T, VEC>;
    constexpr int VP = C::VP;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float red[2][3 * 16];
    __shared__ __align__(8) uint64_t bars[RING_MOST];
    const int tpr = blockDim.x, warps = tpr >> 5, cols = a.d.cols, chunk = blockIdx.x;
    const int64_t begin = chunk * a.chunk_rows;
    const int n = int(begin + a.chunk_rows < a.d.rows ? a.chunk_rows : a.d.rows - begin);
    if (threadIdx.x == 0) {
        for (int s = 0; s < r.stages; ++s) bar_init(bars + s);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (threadIdx.x < 32)
        for (int s = 0; s < r.stages && s < n; ++s) ring_issue<T, VEC>(a, r, smem, bars, s, begin + s);
    if (threadIdx.x < 32) {
#pragma unroll
        for (int i = 0; i < 3; ++i) (&red[0][0])[threadIdx.x + 32 * i] = 0.f;
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const bool block = FULL || a.y, after = FULL || (a.d.flags & RUBICK_NORM_AFTER), before = FULL || (a.d.flags & RUBICK_NORM_BEFORE);
    const bool stream = FULL || a.dx_out, need_y = FULL || r.i_y >= 0;
    const float o = a.d.flags & RUBICK_NORM_UNIT_OFFSET ? 1.f : 0.f, inv_cols = 1.f / float(cols);
    f2 wb[NV][VP], k[NV][VP], t[NV][VP], acc_a[NV][VP], acc_b[NV][VP];
    before_factors<T, W, VEC, NV>(a, tpr, o, wb);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VP; ++e) k[i][e] = t[i][e] = acc_a[i][e] = acc_b[i][e] = 0ull;
    float2 next = make_float2(1.f, 0.f);
    if (a.rstd_in) next = *reinterpret_cast<const float2 *>(a.rstd_in + 2 * begin);
    __syncthreads();
    T *dx = static_cast<T *>(a.dx) + begin * a.d.ld_x, *dy = static_cast<T *>(a.dy) + begin * a.d.ld_y;
    int64_t group = -1, group_end = begin;
    const T *gate = nullptr;                      // of the current group
    bool lost = false;
    int s = 0;
    uint32_t parity = 0;
    for (int i_row = 0; i_row < n; ++i_row) {
        const int64_t row = begin + i_row;
        const uint8_t *stage = smem + size_t(s) * r.tensors * r.slot_bytes;
        const float ra = after ? next.x : 1.f, rb = before ? next.y : 0.f;
        if (a.rstd_in && i_row + 1 < n) next = *reinterpret_cast<const float2 *>(a.rstd_in + 2 * row + 2);
        if (!lost && !bar_wait(bars + s, parity)) { lost = true; atomicOr(a.status, DS_COPY_LOST); }
        const T *x_row = stage_row<T, VEC>(stage, r, r.i_x, a.x, row, a.d.ld_x), *y_row = stage_row<T, VEC>(stage, r, r.i_y, a.y, row, a.d.ld_y);
        const T *d_row = stage_row<T, VEC>(stage, r, r.i_dxo, a.dx_out, row, a.d.ld_x), *h_row = stage_row<T, VEC>(stage, r, r.i_dh, a.dh, row, a.d.ld_h);
        if (block && row >= group_end) {
            if (group >= 0) ring_flush<T, W, VEC, NV>(a, chunk, begin, begin + n, group, gate, tpr, o, t, acc_a);
            group = row / a.d.group_rows;
            group_end = (group + 1) * a.d.group_rows;
            gate = a.gate ? static_cast<const T *>(a.gate) + group * a.d.ld_gate : nullptr;
            group_factors<T, W, VEC, NV>(a, gate, tpr, o, k);
        }
        f2 part[3] = {0ull, 0ull, 0ull};
        const f2 rb2 = both(rb);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = C::first(i, tpr);
            if (c < cols) {
                f2 d[VP], x[VP], h[VP], y[VP];
                if (stream) C::load(d_row, c, tpr, cols, d); else zero_cols(d);
                if (before) C::load(x_row, c, tpr, cols, x); else zero_cols(x);
                if (before) C::load(h_row, c, tpr, cols, h); else zero_cols(h);
                if (need_y) C::load(y_row, c, tpr, cols, y); else zero_cols(y);
#pragma unroll
                for (int e = 0; e < VP; ++e) {
                    // the sums without the row's factors ra and rb, which come in behind the reduction
                    const f2 hw = mul2(h[e], wb[i][e]), q = mul2(k[i][e], y[e]);
                    acc_b[i][e] = fma2(mul2(h[e], rb2), x[e], acc_b[i][e]);
                    part[0] = fma2(hw, x[e], part[0]);
                    part[1] = fma2(q, fma2(rb2, hw, d[e]), part[1]);
                    part[2] = fma2(q, x[e], part[2]);
                }
            }
        }
        float sum[3];
        ring_sum<3>(part, sum, red[i_row & 1], warps);
        if (threadIdx.x < 32 && i_row >= 1 && i_row - 1 + r.stages < n)
            ring_issue<T, VEC>(a, r, smem, bars, s ? s - 1 : r.stages - 1, row - 1 + r.stages);
        const float m1 = rb * sum[0] * inv_cols, m2 = after ? ra * (sum[1] - rb * rb * m1 * sum[2]) * inv_cols : 0.f;
        const f2 f1 = both(-rb * rb * m1), f2y = both(-ra * ra * m2), ra2 = both(ra);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = C::first(i, tpr);
            if (c < cols) {
                f2 d[VP], x[VP], h[VP], y[VP];
                if (stream) C::load(d_row, c, tpr, cols, d); else zero_cols(d);
                if (before) C::load(x_row, c, tpr, cols, x); else zero_cols(x);
                if (before) C::load(h_row, c, tpr, cols, h); else zero_cols(h);
                if (need_y) C::load(y_row, c, tpr, cols, y); else zero_cols(y);
#pragma unroll
                for (int e = 0; e < VP; ++e) {
                    d[e] = fma2(f1, x[e], fma2(rb2, mul2(h[e], wb[i][e]), d[e]));           // G
                    const f2 rg = mul2(ra2, d[e]);
                    t[i][e] = fma2(rg, y[e], t[i][e]);
                    const f2 du = mul2(k[i][e], rg);
                    y[e] = after ? fma2(f2y, y[e], du) : du;      // (zero times an infinite y is not zero)
                }
                C::store(dx, c, tpr, cols, d);
                if (block) C::store(dy, c, tpr, cols, y);
            }
        }
        dx += a.d.ld_x;
        dy += a.d.ld_y;
        if (++s == r.stages) { s = 0; parity ^= 1u; }
    }
    if (group >= 0) ring_flush<T, W, VEC, NV>(a, chunk, begin, begin + n, group, gate, tpr, o, t, acc_a);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = C::first(i, tpr);
        if (c >= cols) continue;
        const bool straight = sums_go_straight(a);
        if (a.dw_after) C::put(straight ? a.dw_after : part_row(a, 0, chunk), c, tpr, cols, acc_a[i]);
        if (a.dw_before) C::put(straight ? a.dw_before : part_row(a, 1, chunk), c, tpr, cols, acc_b[i]);
    }
}

// whether a gate group lies in so few chunks that one warp sums them
__host__ __device__ __forceinline__ bool few_chunks(const NormArgs &a) { return a.d.group_rows <= 32 * a.chunk_rows; }

// Adds up the chunks' partial sums, always in the same order: blockIdx.y = 0 dW_after, 1 dW_before, from 2 on the gate
// groups that lie in more than one chunk.  CB columns a block, 512 / CB chunks at a time: the sums lie in L2, so it is loads
// in flight that count; few columns are taken eight (a 32-byte sector) a block, for more blocks.
template <typename T, int CB>
__global__ void __launch_bounds__(512) norm_backward_join_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float tile[16][CB];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * CB + lane % CB, turn = threadIdx.x / CB;
    asm volatile("griddepcontrol.wait;" ::: "memory");       // launched while the chunks are still at work
    const int64_t groups = (a.d.rows + a.d.group_rows - 1) / a.d.group_rows;
    const bool weights = blockIdx.y < 2;
    if (weights && !(blockIdx.y ? a.dw_before : a.dw_after)) return;
    const int64_t candidates = weights ? 1 : groups;
    int first = 0, last = a.n_chunks - 1;
    int64_t group = 0;
    const auto split = [&](int64_t k) {
        group = k;
        const int64_t g0 = group * a.d.group_rows, g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
        first = int(g0 / a.chunk_rows); last = int((g1 - 1) / a.chunk_rows);
        return first != last;
    };
    // A warp a group: with a block for each, most threads had no chunk (2,191 x 768 fp32 backward, 32 rows a group: 44 us,
    // 16 rows 62 us; 26 us both this way).
    if (!weights && few_chunks(a)) {
        for (int64_t k = int64_t(blockIdx.y - 2) * 16 + warp; k < candidates; k += int64_t(gridDim.y - 2) * 16) {
            if (!split(k)) continue;
            float v = 0.f;
            if (c < a.d.cols)
#pragma unroll 8
                for (int q = first + lane / CB; q <= last; q += 32 / CB) v += part_row(a, q == first ? 3 : 2, q)[c];
#pragma unroll
            for (int o = 16; o >= CB; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane < CB && c < a.d.cols) static_cast<T *>(a.dgate)[group * a.d.ld_gate + c] = from_f<T>(v);
        }
        return;
    }
    for (int64_t k = weights ? 0 : blockIdx.y - 2; k < candidates; k += weights ? 1 : gridDim.y - 2) {
        if (!weights && !split(k)) continue;
        float v = 0.f;
        if (c < a.d.cols)
#pragma unroll 8
            for (int q = first + turn; q <= last; q += 512 / CB) v += part_row(a, weights ? blockIdx.y : q == first ? 3 : 2, q)[c];
#pragma unroll
        for (int o = 16; o >= CB; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane < CB) tile[warp][lane] = v;
        __syncthreads();
        if (threadIdx.x < CB && c < a.d.cols) {
            v = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) v += tile[i][lane];
            if (!weights) static_cast<T *>(a.dgate)[group * a.d.ld_gate + c] = from_f<T>(v);
            else (blockIdx.y ? a.dw_before : a.dw_after)[c] = v;
        }
        __syncthreads();
    }
}

// Threads and vectors of a row: VE elements a vector, NV vectors a thread; for the ring its stages and blocks per SM.
struct Shape { int ve, nv, tpr, slots; bool ring, ring_vec; int blocks, smem; Ring r; };

int esize_of(int dtype) { return dtype == RUBICK_F32 ? 4 : 2; }

// 16-byte accesses where every row of every tensor starts on a 16-byte boundary
bool vectors_fit(const NormArgs &a, int esize)
{
    const void *rows[] = {a.x, a.y, a.x_out, a.h, a.dx_out, a.dh, a.dx, a.dy, a.gate, a.dgate, a.w_after, a.w_before};
    for (const void *p : rows) if (!aligned16(p)) return false;
    const bool blk = a.y != nullptr, bef = (a.d.flags & RUBICK_NORM_BEFORE) != 0;
    return a.d.ld_x * esize % 16 == 0 && (!blk || a.d.ld_y * esize % 16 == 0) && (!bef || a.d.ld_h * esize % 16 == 0)
        && (!a.gate || a.d.ld_gate * esize % 16 == 0);
}

// dynamic shared memory of one of n blocks on an SM: 228 KB, less what the system and the static part take of each
int ring_budget(int n) { return 228 * 1024 / n - 1792; }

// The ring's shape; false where a row does not fit: fewer than two stages, or more columns than 16 a thread cover.
bool ring_shape(const NormArgs &a, bool back, int num_sms, Shape &s)
{
    const int es = esize_of(a.d.dtype);
    const bool vec = s.ve > 1 && a.d.cols % s.ve == 0;
    const int unit = vec ? s.ve : 2, units = (a.d.cols + unit - 1) / unit, most = 16 / unit;
    int warps = (units + most * 32 - 1) / (most * 32);
    if (warps > 16) return false;
    // few rows: more warps a row, down to one set of columns a thread (backward, 64 x 4,096 bf16: 13.8 against 15.9 us, 300 x
    // 1,280 14.9 against 16.9; 1,000 x 1,280, where half the rows' threads do as well, 23.0 against 22.0)
    while (a.d.rows * warps < int64_t(num_sms) * 8 && warps * 2 <= 16 && warps * 32 < units) warps *= 2;
    Ring &r = s.r;
    const bool before = a.d.flags & RUBICK_NORM_BEFORE, after = a.d.flags & RUBICK_NORM_AFTER;
    int n = 0;
    r.i_x = !back || before ? n++ : -1;
    r.i_y = a.y && (!back || after || a.gate) ? n++ : -1;
    r.i_dxo = back && a.dx_out ? n++ : -1;
    r.i_dh = back && before ? n++ : -1;
    // Forward, a gate row that serves few rows travels with them; one that serves many is read when its group begins (16,384 x
    // 4,096 bf16, 1 row a group: 147 against 204 us, 7 rows: 106 against 110, 16: 103 against 102).  Backward there are more
    // tensors for the stages, and the gradients at a group's end take the gate once more: read at the group's beginning
    // always (8,192 x 4,096, 1 row: 188 against 159 us, 7 rows: 120 against 92).
    r.i_gate = !back && a.gate && a.d.group_rows < 8 ? n++ : -1;
    if (n == 0) return false;
    r.tensors = n;
    r.slot_bytes = vec ? uint32_t(a.d.cols * es) : uint32_t((a.d.cols * es + 15) / 16 + 1) * 16;
    s.tpr = warps * 32;
    s.nv = vec ? (units + s.tpr - 1) / s.tpr : 8;
    s.slots = 1;
    // 128 registers a thread backward, 96 forward (64 with one vector a thread)
    s.blocks = (back ? 512 : s.nv == 1 ? 1024 : 640) / s.tpr;
    if (s.blocks > 16) s.blocks = 16;
    for (;; --s.blocks) {
        if (s.blocks == 0) return false;
        r.stages = ring_budget(s.blocks) / (n * int(r.slot_bytes));
        if (r.stages >= 3 || (s.blocks == 1 && r.stages == 2)) break;
    }
    if (r.stages > RING_MOST) r.stages = RING_MOST;
    s.smem = r.stages * n * int(r.slot_bytes);
    s.ring_vec = vec;
    return true;
}

void cut_rows(const NormArgs &a, int64_t want, int64_t *chunk_rows, int *n_chunks)
{
    *chunk_rows = a.d.rows > want ? (a.d.rows + want - 1) / want : 1;
    *n_chunks = int((a.d.rows + *chunk_rows - 1) / *chunk_rows);
}

// Gate groups that are not longer than two chunks are kept whole, so that nothing of them is left to be joined (2,191 x 768
// fp32, four rows a group: chunks of two rows 169 us, of four 21 us).  Longer ones are cut: whole chunks of 8 rows
// would leave the SMs half empty (8 rows a chunk: 38 us where 2 a chunk take 30).
void keep_groups(const NormArgs &a, int64_t *chunk_rows, int *n_chunks)
{
    const int64_t g = a.d.group_rows;
    if (!a.gate || !a.dgate || g > 2 * *chunk_rows) return;
    *chunk_rows = (*chunk_rows + g - 1) / g * g;
    *n_chunks = int((a.d.rows + *chunk_rows - 1) / *chunk_rows);
}

// Forward rows that a resident block of the ring has to have, in halves: a ring has to be filled before it runs, and narrow rows do
// well in registers.  Ring against registers, bf16: 9,500 x 256 12.8 us and 11.7, 12,000 x 256 12.8 and 13.8; 4,800 x 512 12.8
// and 11.8, 6,000 x 512 12.8 and 13.8; 1,480 x 1,280 10.8 and 12.8; 2,400 x 4,096 22 and 46.  Rows at odd addresses:
// 20,000 x 125 28 and 17; 3,000 x 300 17 and 12, 4,800 x 300 21 and 42; 2,000 x 615 18 and 15, 3,000 x 615 22 and 50;
// 740 x 1,030 15 and 13, 1,480 x 1,030 19 and 45.
int64_t ring_halves(const NormArgs &a, const Shape &s)
{
    if (s.ring_vec) return s.tpr > 64 ? 2 : s.tpr == 32 && s.nv == 1 ? 8 : 4;
    return a.d.cols <= 128 ? int64_t(1) << 31 : s.tpr > 32 ? 3 : 4;
}

Shape forward_shape(const NormArgs &a, int num_sms)
{
    Shape s;
    const int es = esize_of(a.d.dtype);
    s.ve = vectors_fit(a, es) ? 16 / es : 1;
    s.ring = ring_shape(a, false, num_sms, s) && 2 * a.d.rows >= int64_t(num_sms) * s.blocks * ring_halves(a, s);
    if (s.ring) return s;
    const int most = 32 / s.ve, nvec = (a.d.cols + s.ve - 1) / s.ve;
    int warps = (nvec + most * 32 - 1) / (most * 32);
    // few rows: more warps a row while the rows do not fill the SMs' 64 warps (4 x 4,096 bf16: 6.7 us, 11.8 with the fewest warps
    // that hold a row; 1,000 x 777: 14.8 against 29.2, and 21.0 with 16 warps an SM for the limit)
    while (warps * 32 < nvec && a.d.rows * warps < int64_t(num_sms) * 64 && (warps <= 8 || (warps <= 16 && s.ve > 1 && warps * 64 >= nvec))) warps *= 2;
    s.tpr = warps * 32;
    s.nv = (nvec + s.tpr - 1) / s.tpr;
    s.slots = s.tpr >= 128 ? 1 : 128 / s.tpr;
    if (a.d.rows < int64_t(num_sms) * s.slots) s.slots = 1;
    return s;
}

Shape backward_shape(const NormArgs &a, int num_sms)
{
    Shape s;
    const int es = esize_of(a.d.dtype);
    s.ve = vectors_fit(a, es) ? 16 / es : 1;
    s.ring = ring_shape(a, true, num_sms, s);
    if (!s.ring) { s.tpr = 512; s.blocks = 1; }
    return s;
}

template <typename K> cudaError_t launch_ring(K kernel, const NormArgs &a, const Shape &s, cudaStream_t st)
{
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, s.smem);
    if (e != cudaSuccess) return e;
    kernel<<<unsigned(a.n_chunks), s.tpr, s.smem, st>>>(a, s.r);
    count_launch();
    return cudaGetLastError();
}

template <typename T, typename W, bool FULL> cudaError_t forward_ring(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    constexpr int MOST = 16 / Lanes<T>::N;
    if (!s.ring_vec) return launch_ring(norm_forward_ring_kernel<T, W, 8, FULL, false>, a, s, st);
    if (s.nv <= 1) return launch_ring(norm_forward_ring_kernel<T, W, 1, FULL, true>, a, s, st);
    if (s.nv <= 2) return launch_ring(norm_forward_ring_kernel<T, W, 2, FULL, true>, a, s, st);
    return launch_ring(norm_forward_ring_kernel<T, W, MOST, FULL, true>, a, s, st);
}
template <typename T, typename W, bool FULL> cudaError_t backward_ring(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    constexpr int MOST = 16 / Lanes<T>::N;
    if (!s.ring_vec) return launch_ring(norm_backward_ring_kernel<T, W, 8, FULL, false>, a, s, st);
    if (s.nv <= 1) return launch_ring(norm_backward_ring_kernel<T, W, 1, FULL, true>, a, s, st);
    if (s.nv <= 2) return launch_ring(norm_backward_ring_kernel<T, W, 2, FULL, true>, a, s, st);
    return launch_ring(norm_backward_ring_kernel<T, W, MOST, FULL, true>, a, s, st);
}

template <typename T, typename W, int VE> cudaError_t forward_nv(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    const dim3 block(s.tpr, s.slots);
    const unsigned grid = unsigned((a.d.rows + s.slots - 1) / s.slots);
    if constexpr (VE > 1) {
        if (s.nv <= 1) norm_forward_kernel<T, W, VE, 1><<<grid, block, 0, st>>>(a);
        else if (s.nv <= 2) norm_forward_kernel<T, W, VE, 2><<<grid, block, 0, st>>>(a);
        else if (s.nv <= 3) norm_forward_kernel<T, W, VE, 3><<<grid, block, 0, st>>>(a);
        else if (VE == 8 || s.nv <= 4) norm_forward_kernel<T, W, VE, 4><<<grid, block, 0, st>>>(a);
        else if constexpr (VE == 4) norm_forward_kernel<T, W, VE, 8><<<grid, block, 0, st>>>(a);
    } else {
        if (s.nv <= 4) norm_forward_kernel<T, W, VE, 4><<<grid, block, 0, st>>>(a);
        else if (s.nv <= 16) norm_forward_kernel<T, W, VE, 16><<<grid, block, 0, st>>>(a);
        else norm_forward_kernel<T, W, VE, 32><<<grid, block, 0, st>>>(a);
    }
    count_launch();
    return cudaGetLastError();
}

template <typename T, typename W> cudaError_t forward_any(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    if (s.ring) {
        const bool full = a.y && (a.d.flags & RUBICK_NORM_AFTER) && (a.d.flags & RUBICK_NORM_BEFORE);
        return full ? forward_ring<T, W, true>(a, s, st) : forward_ring<T, W, false>(a, s, st);
    }
    return s.ve > 1 ? forward_nv<T, W, Lanes<T>::N>(a, s, st) : forward_nv<T, W, 1>(a, s, st);
}

template <typename T, typename W, int VE> cudaError_t backward_wide(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    const int smem = 3 * a.d.cols * int(sizeof(float));
    const cudaError_t e = cudaFuncSetAttribute(norm_backward_wide_kernel<T, W, VE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    norm_backward_wide_kernel<T, W, VE><<<unsigned(a.n_chunks), s.tpr, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

template <typename T, typename W> cudaError_t backward_any(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    const bool full = a.y && (a.d.flags & RUBICK_NORM_AFTER) && (a.d.flags & RUBICK_NORM_BEFORE) && a.dx_out;
    const cudaError_t e = s.ring ? (full ? backward_ring<T, W, true>(a, s, st) : backward_ring<T, W, false>(a, s, st))
                                 : s.ve > 1 ? backward_wide<T, W, Lanes<T>::N>(a, s, st) : backward_wide<T, W, 1>(a, s, st);
    if (e != cudaSuccess) return e;
    if (s.ring && sums_go_straight(a)) return cudaSuccess;     // nothing is left to be joined
    const int64_t groups = (a.d.rows + a.d.group_rows - 1) / a.d.group_rows;
    const bool split = a.gate && a.dgate && a.chunk_rows % a.d.group_rows != 0;
    const int64_t blocks = few_chunks(a) ? (groups + 15) / 16 : groups;
    const unsigned more = split ? unsigned(blocks < 32 ? blocks : 32) : 0u;
    if (!a.dw_after && !a.dw_before && !more) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    // (2,000 x 512 bf16 backward: 8 columns a block 25.1 us, 32 36.3; 2,000 x 2,048 29.8 and 28.7; 2,000 x 4,096 42.4 and 34.8)
    const int cb = a.d.cols <= 2048 ? 8 : 32;
    cfg.gridDim = dim3((a.d.cols + cb - 1) / cb, 2 + more);
    cfg.blockDim = dim3(512);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    count_launch();
    return cb == 8 ? cudaLaunchKernelEx(&cfg, norm_backward_join_kernel<T, 8>, a) : cudaLaunchKernelEx(&cfg, norm_backward_join_kernel<T, 32>, a);
}

// by the element type and the weights' type
#define BY_TYPE(call)                                                                                                     \
    (a.d.dtype == RUBICK_BF16 ? (a.d.wtype == RUBICK_F32 ? call<bf16, float>(a, s, st) : call<bf16, bf16>(a, s, st))       \
     : a.d.dtype == RUBICK_F16 ? (a.d.wtype == RUBICK_F32 ? call<f16, float>(a, s, st) : call<f16, f16>(a, s, st))         \
                               : call<float, float>(a, s, st))

}  // namespace

cudaError_t launch_norm_forward(const NormArgs &args, int num_sms, cudaStream_t st)
{
    NormArgs a = args;
    const Shape s = forward_shape(a, num_sms);
    if (s.ring) cut_rows(a, int64_t(num_sms) * s.blocks, &a.chunk_rows, &a.n_chunks);
    return BY_TYPE(forward_any);
}

// floats of scratch; also fixes how the rows are cut into chunks: one chunk per row slot, as many blocks as the SMs
// hold at once
size_t norm_backward_scratch(const NormArgs &a, int num_sms, int64_t *chunk_rows, int *n_chunks)
{
    const Shape s = backward_shape(a, num_sms);
    cut_rows(a, int64_t(num_sms) * s.blocks, chunk_rows, n_chunks);
    keep_groups(a, chunk_rows, n_chunks);
    // two rows one after the other cost less than a second kernel, and the sums then go straight to their places (4 x 4,096 bf16 so
    // 13.8 us, with a join 12.8; 8 x 4,096 20.0 and 11.8)
    if (s.ring && a.d.rows <= 2 && aligned16(a.dw_after) && aligned16(a.dw_before)) { *chunk_rows = a.d.rows; *n_chunks = 1; }
    return size_t(4) * size_t(*n_chunks) * size_t(a.d.cols);
}

cudaError_t launch_norm_backward(const NormArgs &a, int num_sms, cudaStream_t st)
{
    const Shape s = backward_shape(a, num_sms);
    return BY_TYPE(backward_any);
}

}  // namespace rubick
