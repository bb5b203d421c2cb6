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
// All of it is bound by memory: 4 row elements move per column forward, 6 backward, for a dozen operations.  A row
// stays in the registers of one warp or one block between its loads and its stores.

#include "train_common.cuh"

namespace rubick {

using namespace train;

namespace {

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

// Writes the gate gradient of rows [first, last] of a chunk that starts at row `begin`, all in one gate group: final
// where the whole group is in the chunk, a partial sum otherwise.
template <typename T, int VE, int NV>
__device__ __forceinline__ void flush_gate(const NormArgs &a, int chunk, int64_t begin, int64_t end_row, int64_t group, int tpr,
                                           float (&acc)[NV][VE], const float (&g)[NV][VE])
{
    const int64_t g0 = group * a.d.group_rows;
    const int64_t g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
    if (a.d.flags & RUBICK_NORM_TANH_GATE) {      // g holds tanh(gate)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) acc[i][e] *= 1.f - g[i][e] * g[i][e];
    }
    if (!a.dgate) {
        // nobody asked for it
    } else if (g0 >= begin && g1 <= end_row) {
        T *dg = static_cast<T *>(a.dgate) + group * a.d.ld_gate;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float r[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) r[e] = acc[i][e];
            store_cols<T, VE>(dg, (i * tpr + int(threadIdx.x)) * VE, a.d.cols, r);
        }
    } else {
        float *p = part_row(a, g0 < begin ? 2 : 3, chunk);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const int c = (i * tpr + int(threadIdx.x)) * VE + e;
                if (c < a.d.cols) p[c] = acc[i][e];
            }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[i][e] = 0.f;
}

// One row slot (threadIdx.y) of a block works through one chunk of consecutive rows; the column sums stay in
// registers until the chunk ends.
template <typename T, typename W, int VE, int NV>
__global__ void __launch_bounds__(512) norm_backward_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float red[2][3 * 32];
    const int tpr = blockDim.x, warps = tpr >> 5, cols = a.d.cols;
    const int chunk = blockIdx.x * blockDim.y + threadIdx.y;
    const int64_t begin = chunk * a.chunk_rows;
    const int64_t stop = begin + a.chunk_rows < a.d.rows ? begin + a.chunk_rows : a.d.rows;
    const bool after = a.d.flags & RUBICK_NORM_AFTER, before = a.d.flags & RUBICK_NORM_BEFORE;
    const bool th = a.d.flags & RUBICK_NORM_TANH_GATE, need_y = a.y && (after || a.gate);
    const float o = a.d.flags & RUBICK_NORM_UNIT_OFFSET ? 1.f : 0.f;
    const float inv_cols = 1.f / float(cols);
    const int c0 = int(threadIdx.x) * VE;
    float acc_a[NV][VE], acc_b[NV][VE], acc_g[NV][VE], g[NV][VE];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) { acc_a[i][e] = acc_b[i][e] = acc_g[i][e] = 0.f; g[i][e] = 1.f; }
    int64_t group = -1, group_end = begin;        // the gate row in g[][]
    for (int64_t step = 0; step < a.chunk_rows; ++step) {          // the same count for every row slot of the block
        const int64_t row = begin + step;
        const bool live = row < stop;
        const int end = live ? cols : 0;
        Raw<T, VE> dxo[NV], xr[NV], dh[NV], yr[NV];
        const float ra = after && live ? a.rstd_in[2 * row] : 1.f;
        const float rb = before && live ? a.rstd_in[2 * row + 1] : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = i * tpr * VE + c0;
            dxo[i].zero(); xr[i].zero(); dh[i].zero(); yr[i].zero();
            if (a.dx_out) dxo[i].load(static_cast<const T *>(a.dx_out) + row * a.d.ld_x, c, end);
            if (before) xr[i].load(static_cast<const T *>(a.x) + row * a.d.ld_x, c, end);
            if (before) dh[i].load(static_cast<const T *>(a.dh) + row * a.d.ld_h, c, end);
            if (need_y) yr[i].load(static_cast<const T *>(a.y) + row * a.d.ld_y, c, end);
        }
        if (a.gate && live && row >= group_end) {
            if (group >= 0) flush_gate<T, VE, NV>(a, chunk, begin, stop, group, tpr, acc_g, g);
            group = row / a.d.group_rows;
            group_end = (group + 1) * a.d.group_rows;
            const T *gate = static_cast<const T *>(a.gate) + group * a.d.ld_gate;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                load_shared_cols<T, VE>(gate, i * tpr * VE + c0, cols, g[i], 0.f);
                if (th) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[i][e] = tanhf(g[i][e]);
                }
            }
        }
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = i * tpr * VE + c0;
            float wa[VE], wb[VE], d[VE], x[VE], e1[VE], y[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) wa[e] = wb[e] = 1.f - o;
            if (a.w_after) load_shared_cols<W, VE>(static_cast<const W *>(a.w_after), c, cols, wa, 0.f);
            if (a.w_before) load_shared_cols<W, VE>(static_cast<const W *>(a.w_before), c, cols, wb, 0.f);
            dxo[i].get(d); xr[i].get(x); dh[i].get(e1); yr[i].get(y);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float xh = x[e] * rb, ew = e1[e] * (wb[e] + o);
                acc_b[i][e] = fmaf(e1[e], xh, acc_b[i][e]);
                s[0] = fmaf(ew, xh, s[0]);
                const float q = a.d.alpha * g[i][e] * (wa[e] + o) * (y[e] * ra);
                s[1] = fmaf(q, fmaf(rb, ew, d[e]), s[1]);
                s[2] = fmaf(q, xh, s[2]);
            }
        }
        row_sum<3>(s, red[step & 1], warps, threadIdx.y);
        const float m1 = s[0] * inv_cols, m2 = after ? (s[1] - rb * m1 * s[2]) * inv_cols : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = i * tpr * VE + c0;
            float wa[VE], wb[VE], d[VE], x[VE], e1[VE], y[VE], dx[VE], dy[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) wa[e] = wb[e] = 1.f - o;
            if (a.w_after) load_shared_cols<W, VE>(static_cast<const W *>(a.w_after), c, cols, wa, 0.f);
            if (a.w_before) load_shared_cols<W, VE>(static_cast<const W *>(a.w_before), c, cols, wb, 0.f);
            dxo[i].get(d); xr[i].get(x); dh[i].get(e1); yr[i].get(y);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                dx[e] = fmaf(rb, e1[e] * (wb[e] + o) - x[e] * rb * m1, d[e]);
                const float f = a.d.alpha * dx[e], fg = f * g[i][e], yh = y[e] * ra, w = wa[e] + o;
                acc_g[i][e] = fmaf(f * w, yh, acc_g[i][e]);
                acc_a[i][e] = fmaf(fg, yh, acc_a[i][e]);
                dy[e] = after ? ra * (fg * w - yh * m2) : fg;
            }
            store_cols<T, VE>(static_cast<T *>(a.dx) + row * a.d.ld_x, c, end, dx);
            if (a.dy) store_cols<T, VE>(static_cast<T *>(a.dy) + row * a.d.ld_y, c, end, dy);
        }
    }
    if (chunk >= a.n_chunks) return;
    if (group >= 0) flush_gate<T, VE, NV>(a, chunk, begin, stop, group, tpr, acc_g, g);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const int c = i * tpr * VE + c0 + e;
            if (c < cols && a.dw_after) part_row(a, 0, chunk)[c] = acc_a[i][e];
            if (c < cols && a.dw_before) part_row(a, 1, chunk)[c] = acc_b[i][e];
        }
}

// The same for rows that are too wide for registers: the column sums are in shared memory, and a row is read twice
// (the second time from L2), once for its sums and once for its gradients.
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
                        if (th) { const float t = tanhf(to_f(gate[c + e])); v *= 1.f - t * t; }
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

// Adds up the chunks' partial sums, in chunk order: blockIdx.y = 0 dW_after, 1 dW_before, from 2 on the gate groups that
// lie in more than one chunk.  32 columns a block, one chunk a warp at a time.
template <typename T>
__global__ void __launch_bounds__(512) norm_backward_join_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float tile[16][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const int64_t groups = (a.d.rows + a.d.group_rows - 1) / a.d.group_rows;
    const bool weights = blockIdx.y < 2;
    if (weights && !(blockIdx.y ? a.dw_before : a.dw_after)) return;
    // a group that is split has a chunk in which it begins; no chunk holds the beginning of two such groups
    const bool by_group = groups <= a.n_chunks;
    const int64_t candidates = weights ? 1 : by_group ? groups : a.n_chunks;
    for (int64_t k = weights ? 0 : blockIdx.y - 2; k < candidates; k += weights ? 1 : gridDim.y - 2) {
        int first = 0, last = a.n_chunks - 1;
        int64_t group = k;
        if (!weights) {
            if (!by_group) {
                const int64_t end = (k + 1) * a.chunk_rows < a.d.rows ? (k + 1) * a.chunk_rows : a.d.rows;
                group = (end - 1) / a.d.group_rows;
            }
            const int64_t g0 = group * a.d.group_rows, g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
            first = int(g0 / a.chunk_rows); last = int((g1 - 1) / a.chunk_rows);
            if (first == last || (!by_group && first != k)) continue;
        }
        float v = 0.f;
        if (c < a.d.cols)
            for (int q = first + warp; q <= last; q += 16) v += part_row(a, weights ? blockIdx.y : q == first ? 3 : 2, q)[c];
        tile[warp][lane] = v;
        __syncthreads();
        if (warp == 0 && c < a.d.cols) {
            v = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) v += tile[i][lane];
            if (!weights) static_cast<T *>(a.dgate)[group * a.d.ld_gate + c] = from_f<T>(v);
            else (blockIdx.y ? a.dw_before : a.dw_after)[c] = v;
        }
        __syncthreads();
    }
}

// Threads and vectors of a row: VE elements a vector, NV vectors a thread.
struct Shape { int ve, nv, tpr, slots; bool wide; };

// 16-byte accesses where every row of every tensor starts on a 16-byte boundary
bool vectors_fit(const NormArgs &a, int esize, int wsize)
{
    const void *rows[] = {a.x, a.y, a.x_out, a.h, a.dx_out, a.dh, a.dx, a.dy, a.gate, a.dgate, a.w_after, a.w_before};
    for (const void *p : rows) if (!aligned16(p)) return false;
    (void)wsize;
    const bool blk = a.y != nullptr, bef = (a.d.flags & RUBICK_NORM_BEFORE) != 0;
    return a.d.ld_x * esize % 16 == 0 && (!blk || a.d.ld_y * esize % 16 == 0) && (!bef || a.d.ld_h * esize % 16 == 0)
        && (!a.gate || a.d.ld_gate * esize % 16 == 0);
}

int esize_of(int dtype) { return dtype == RUBICK_F32 ? 4 : 2; }

Shape forward_shape(const NormArgs &a, int num_sms)
{
    Shape s;
    const int es = esize_of(a.d.dtype);
    s.wide = false;
    s.ve = vectors_fit(a, es, 0) ? 16 / es : 1;
    const int most = 32 / s.ve, nvec = (a.d.cols + s.ve - 1) / s.ve;
    int warps = (nvec + most * 32 - 1) / (most * 32);
    // few rows: more warps a row while the rows do not fill the SMs' 64 warps
    while (warps * 32 < nvec && a.d.rows * warps < int64_t(num_sms) * 16 && (warps <= 8 || (warps <= 16 && s.ve > 1 && warps * 64 >= nvec))) warps *= 2;
    s.tpr = warps * 32;
    s.nv = (nvec + s.tpr - 1) / s.tpr;
    s.slots = s.tpr >= 128 ? 1 : 128 / s.tpr;
    if (a.d.rows < int64_t(num_sms) * s.slots) s.slots = 1;
    return s;
}

Shape backward_shape(const NormArgs &a)
{
    Shape s;
    const int es = esize_of(a.d.dtype);
    s.ve = vectors_fit(a, es, 0) ? 16 / es : 1;
    const int most = 16 / s.ve, nvec = (a.d.cols + s.ve - 1) / s.ve;   // 16 columns a thread
    const int warps = (nvec + most * 32 - 1) / (most * 32);
    s.wide = warps > 16;
    s.tpr = s.wide ? 512 : warps * 32;
    s.nv = (nvec + s.tpr - 1) / s.tpr;
    s.slots = s.wide || s.tpr >= 128 ? 1 : 128 / s.tpr;
    return s;
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

template <typename T, typename W, int VE> cudaError_t backward_nv(const NormArgs &a, const Shape &s, cudaStream_t st)
{
    const dim3 block(s.tpr, s.slots);
    const unsigned grid = unsigned((a.n_chunks + s.slots - 1) / s.slots);
    if (s.wide) {
        const int smem = 3 * a.d.cols * int(sizeof(float));
        const cudaError_t e = cudaFuncSetAttribute(norm_backward_wide_kernel<T, W, VE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        norm_backward_wide_kernel<T, W, VE><<<grid, block, smem, st>>>(a);
    } else if constexpr (VE == 8) {
        if (s.nv <= 1) norm_backward_kernel<T, W, VE, 1><<<grid, block, 0, st>>>(a);
        else norm_backward_kernel<T, W, VE, 2><<<grid, block, 0, st>>>(a);
    } else if constexpr (VE == 4) {
        if (s.nv <= 2) norm_backward_kernel<T, W, VE, 2><<<grid, block, 0, st>>>(a);
        else norm_backward_kernel<T, W, VE, 4><<<grid, block, 0, st>>>(a);
    } else {
        if (s.nv <= 4) norm_backward_kernel<T, W, VE, 4><<<grid, block, 0, st>>>(a);
        else norm_backward_kernel<T, W, VE, 16><<<grid, block, 0, st>>>(a);
    }
    count_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int64_t groups = (a.d.rows + a.d.group_rows - 1) / a.d.group_rows;
    const bool split = a.gate && a.dgate && a.chunk_rows % a.d.group_rows != 0;
    const unsigned more = split ? unsigned(groups < 32 ? groups : 32) : 0u;
    if (!a.dw_after && !a.dw_before && !more) return cudaSuccess;
    norm_backward_join_kernel<T><<<dim3((a.d.cols + 31) / 32, 2 + more), 512, 0, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

// calls f.template operator()<T, W, VE>() for the element type, the weights' type and the vector width at hand
template <typename F> cudaError_t by_type(const NormArgs &a, int ve, F f)
{
    const bool wide_w = a.d.wtype == RUBICK_F32;
    switch (a.d.dtype) {
    case RUBICK_BF16:
        if (wide_w) return ve > 1 ? f.template operator()<bf16, float, 8>() : f.template operator()<bf16, float, 1>();
        return ve > 1 ? f.template operator()<bf16, bf16, 8>() : f.template operator()<bf16, bf16, 1>();
    case RUBICK_F16:
        if (wide_w) return ve > 1 ? f.template operator()<f16, float, 8>() : f.template operator()<f16, float, 1>();
        return ve > 1 ? f.template operator()<f16, f16, 8>() : f.template operator()<f16, f16, 1>();
    default:
        return ve > 1 ? f.template operator()<float, float, 4>() : f.template operator()<float, float, 1>();
    }
}

struct Forward {
    const NormArgs &a; const Shape &s; cudaStream_t st;
    template <typename T, typename W, int VE> cudaError_t operator()() const { return forward_nv<T, W, VE>(a, s, st); }
};
struct Backward {
    const NormArgs &a; const Shape &s; cudaStream_t st;
    template <typename T, typename W, int VE> cudaError_t operator()() const { return backward_nv<T, W, VE>(a, s, st); }
};

}  // namespace

cudaError_t launch_norm_forward(const NormArgs &a, int num_sms, cudaStream_t st)
{
    const Shape s = forward_shape(a, num_sms);
    return by_type(a, s.ve, Forward{a, s, st});
}

// floats of scratch; also fixes how the rows are cut into chunks: one chunk per row slot, as many blocks as the SMs
// hold at once (16 warps an SM at the kernel's registers)
size_t norm_backward_scratch(const NormArgs &a, int num_sms, int64_t *chunk_rows, int *n_chunks)
{
    const Shape s = backward_shape(a);
    const int blocks = s.wide ? 1 : 512 / (s.tpr * s.slots) > 0 ? 512 / (s.tpr * s.slots) : 1;
    const int64_t want = int64_t(num_sms) * blocks * s.slots;
    *chunk_rows = a.d.rows > want ? (a.d.rows + want - 1) / want : 1;
    *n_chunks = int((a.d.rows + *chunk_rows - 1) / *chunk_rows);
    return size_t(4) * size_t(*n_chunks) * size_t(a.d.cols);
}

cudaError_t launch_norm_backward(const NormArgs &a, int num_sms, cudaStream_t st)
{
    (void)num_sms;
    const Shape s = backward_shape(a);
    return by_type(a, s.ve, Backward{a, s, st});
}

}  // namespace rubick
