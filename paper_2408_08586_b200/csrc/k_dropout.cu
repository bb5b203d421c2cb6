// Dropout from a counter-based generator, and the elementwise part of a linear layer's backward pass with its column sums.
//
// Both read and write every element once.  What bounds dropout is the generator: 15 products of 32 x 32 bits for every four
// elements, on a pipe that is 75 to 80 % busy (16,384 x 4,096 bf16 with residual 83 us, 74 % of the copy rate; fp32, twice the
// bytes an element, 3,001 x 1,537 at odd addresses 10.6 us).  dz of 4,096 x 8,192 gelu_tanh takes 48 us (4.2 TB/s): an exponential,
// a reciprocal and a dozen products an element, and memory.  Small calls are a launch and one trip to memory (4 x 4,096: 3.6 us).
#include "product.cuh"

namespace rubick {
namespace {

using namespace train;

// out = residual + drop(x), 16 bytes of columns a thread: a block takes a strip of columns of a run of rows, so that a thread
// keeps to its columns and to what the generator needs of them.
template <typename T, int LANES, bool RESIDUAL, bool WIDE> __global__ void __launch_bounds__(256, 3) dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    constexpr int VE = Lanes<T>::N, ROWS = WIDE ? 2 : 1, STEP = 256 / LANES, ACROSS = LANES * VE;
    chain_go();
    chain_wait();
    __shared__ uint4 staged[WIDE ? 1 : 256];
    const int cols = a.d.cols, lane = threadIdx.x & 31, first = blockIdx.x * ACROSS;
    const int c = first + (threadIdx.x & (LANES - 1)) * VE;
    const int per = int((a.d.rows + a.chunks - 1) / a.chunks);
    const int64_t from = int64_t(per) * blockIdx.y;
    const int high = int(a.d.rows - from < per ? a.d.rows - from : per);              // rows of this block
    const int64_t ld_x = a.d.ld_x, ld_res = a.d.ld_res, ld_out = a.d.ld_out;
    const T *const x = static_cast<const T *>(a.x) + from * ld_x, *const residual = RESIDUAL ? static_cast<const T *>(a.residual) + from * ld_res : nullptr;
    T *const out = static_cast<T *>(a.out) + from * ld_out;
    const bool inside = c < cols;
    Pieces<WIDE> p[ROWS], q[ROWS];
    auto fetch = [&](int row) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (row + i * STEP < high && inside) {
                p[i] = ask<WIDE>(x + (row + i * STEP) * ld_x, c, cols);
                if constexpr (RESIDUAL) q[i] = ask<WIDE>(residual + (row + i * STEP) * ld_res, c, cols);
            }
    };
    int row = threadIdx.x / LANES;
    const int ahead = lane / LANES;                    // rows from the warp's first one to this thread's
    fetch(row);
    const Drop drop(a.drop);                           // (behind the first loads: its seed is in memory too)
    const DropColumns<VE> columns(drop, c);
    const float scale = drop.scale;
    while (row - ahead < high) {
        // the next rows are asked for before these are worked on
        Pieces<WIDE> mine[ROWS], other[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            mine[i] = p[i];
            if constexpr (RESIDUAL) other[i] = q[i];
        }
        fetch(row + ROWS * STEP);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int here = row + i * STEP;
            const bool in = here < high && inside;
            uint4 result = {};
            if (in) {
                float v[VE];
                unpack16<T>(take<WIDE>(x + here * ld_x, c, cols, mine[i]), v);
                if (drop.on) columns.choose(uint32_t(from + here), v);
                if constexpr (RESIDUAL) {
                    float r[VE];
                    unpack16<T>(take<WIDE>(residual + here * ld_res, c, cols, other[i]), r);
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[e] = fmaf(v[e], scale, r[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[e] *= scale;
                }
                result = pack16<T>(v);
                if constexpr (WIDE) {
                    T *const to = out + here * ld_out;
                    if (c + VE <= cols) st_stream(to + c, result);
                    else {
                        const T *const part = reinterpret_cast<const T *>(&result);
#pragma unroll
                        for (int e = 0; e < VE; ++e) if (c + e < cols) to[c + e] = part[e];
                    }
                }
            }
            if constexpr (!WIDE) {
                // rows at any address: through shared memory, so that neighbouring lanes write neighbouring elements (16 bytes of
                // a lane one by one would touch every sector 16 times)
                staged[threadIdx.x] = result;
                __syncwarp();
                const T *const flat = reinterpret_cast<const T *>(staged + (threadIdx.x & ~31));
                T *const to = out + (here - ahead) * ld_out + first;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const int at = e * 32 + lane, col = at % ACROSS, line = at / ACROSS;
                    if (here - ahead + line < high && first + col < cols) to[line * ld_out + col] = flat[at];
                }
                __syncwarp();
            }
        }
        row += ROWS * STEP;
    }
}

constexpr int GRAD_WARPS = 8;

// dz = act'(pre) drop(dout), eight columns a thread, and the sums of its columns: a block takes a strip of columns of a run of
// rows and leaves its sums; the strip's last block adds the runs' sums in their order.
template <typename T, int ACT, bool WIDE> __global__ void __launch_bounds__(256, 3) linear_grad_kernel(const __grid_constant__ LinearGradArgs a)
{
    constexpr int ROWS = WIDE ? 2 : 1;                 // rows that a thread has under way, and as many asked for
    __shared__ float sums[GRAD_WARPS][32][9];
    __shared__ bool last;
    chain_go();
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cols = a.cols;
    const int lanes = a.lanes, c = (blockIdx.x * lanes + (lane & (lanes - 1))) * 8, sub = lane / lanes, abreast = 32 / lanes;
    const int64_t per = (a.rows + a.chunks - 1) / a.chunks, from = per * blockIdx.y, to = from + per < a.rows ? from + per : a.rows;
    const T *const dout = static_cast<const T *>(a.dout), *const pre = static_cast<const T *>(a.pre);
    T *const dz = static_cast<T *>(a.dz);
    const int64_t ld_dout = a.ld_dout, ld_pre = a.ld_pre, ld_dz = a.ld_dz, step = int64_t(GRAD_WARPS) * abreast;
    float total[8] = {};
    if (c < cols) {
        Pieces<WIDE> p[ROWS], q[ROWS];
        auto fetch = [&](int64_t row) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
                if (row + i * step < to) {
                    p[i] = ask<WIDE>(dout + (row + i * step) * ld_dout, c, cols);
                    if constexpr (ACT != RUBICK_ACT_NONE) q[i] = ask<WIDE>(pre + (row + i * step) * ld_pre, c, cols);
                }
        };
        int64_t row = from + warp * abreast + sub;
        fetch(row);
        const Drop drop(a.drop);                       // (behind the first loads: its seed is in memory too)
        const DropColumns<8> columns(drop, c);
        while (row < to) {
            // the next rows are asked for before these are worked on
            Pieces<WIDE> mine[ROWS], other[ROWS];
#pragma unroll
            for (int i = 0; i < ROWS; ++i) { mine[i] = p[i]; other[i] = q[i]; }
            fetch(row + ROWS * step);
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
                if (row + i * step < to) {
                    float v[8], z[8];
                    unpack16<T>(take<WIDE>(dout + (row + i * step) * ld_dout, c, cols, mine[i]), v);
                    if (drop.on) {
                        columns.choose(uint32_t(row + i * step), v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= drop.scale;
                    }
                    if constexpr (ACT != RUBICK_ACT_NONE) {
                        unpack16<T>(take<WIDE>(pre + (row + i * step) * ld_pre, c, cols, other[i]), z);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= act_slope(ACT, z[e]);
                    }
                    if (dz) *reinterpret_cast<uint4 *>(dz + (row + i * step) * ld_dz + c) = pack16<T>(v);     // (its padding too)
#pragma unroll
                    for (int e = 0; e < 8; ++e) total[e] += v[e];
                }
            row += ROWS * step;
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][lane][e] = total[e];
    __syncthreads();
    // column `at` of the strip: what its warps and the rows abreast have
    const int at = threadIdx.x, col = blockIdx.x * lanes * 8 + at;
    float s = 0.f;
    const bool mine = at < lanes * 8 && col < cols;
    if (mine) {
        for (int w = 0; w < GRAD_WARPS; ++w)
            for (int b = 0; b < abreast; ++b) s += sums[w][b * lanes + (at >> 3)][at & 7];
    }
    if (a.chunks == 1) {
        if (mine) a.dbias[col] = s;
        return;
    }
    if (mine) a.part[int64_t(blockIdx.y) * cols + col] = s;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        last = atomicAdd(a.tickets + blockIdx.x, 1u) == uint32_t(a.chunks) - 1;
        if (last) a.tickets[blockIdx.x] = 0;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    // all threads share the runs: 256 / width of them side by side
    const int width = lanes * 8, ways = 256 / width, way = threadIdx.x / width, column = threadIdx.x % width;
    const int col2 = blockIdx.x * width + column;
    float t = 0.f;
    if (col2 < cols) {
#pragma unroll 8
        for (int i = way; i < a.chunks; i += ways) t += __ldcg(a.part + int64_t(i) * cols + col2);
    }
    float *const flat = &sums[0][0][0];
    flat[threadIdx.x] = t;
    __syncthreads();
    if (threadIdx.x < width && col2 < cols) {
        for (int w = 1; w < ways; ++w) t += flat[w * width + column];
        a.dbias[col2] = t;
    }
}

// Runs of rows for so many strips of columns: as many as fill the card's places for blocks up to four times over, chosen so
// that the last filling is nearly whole (448 blocks where 444 have a place take twice a block's time: 110 us for 16,384 x
// 4,096 bf16 against 84), none shorter than what a block has under way.
int runs(int64_t rows, int64_t strips, int64_t least, int64_t places)
{
    const int64_t most = (rows + least - 1) / least;
    int64_t best = 1;
    double full = 0;
    for (int w = 1; w <= 4; ++w) {
        int64_t n = w * places / strips;
        n = n < 1 ? 1 : n < most ? n : most;
        const int64_t blocks = n * strips, waves = (blocks + places - 1) / places;
        const double share = double(blocks) / double(waves * places);
        if (share > full + 0.02) { full = share; best = n; }
    }
    return int(best > 65535 ? 65535 : best);
}

template <typename T, int LANES> cudaError_t dropout(DropoutArgs a, bool wide, int num_sms, cudaStream_t st)
{
    constexpr int across = LANES * Lanes<T>::N;
    const int strips = (a.d.cols + across - 1) / across;
    a.chunks = runs(a.d.rows, strips, 256 / LANES, int64_t(num_sms) * 3);
    const dim3 grid(strips, a.chunks);
    const auto kernel = a.residual ? (wide ? dropout_kernel<T, LANES, true, true> : dropout_kernel<T, LANES, true, false>)
                                   : (wide ? dropout_kernel<T, LANES, false, true> : dropout_kernel<T, LANES, false, false>);
    return launch_chained(kernel, grid, dim3(256), 0, 1, st, a);
}
// Eight threads a row, 128 bytes of it; one for rows of up to 16 bytes.
template <typename T> cudaError_t dropout(const DropoutArgs &a, int num_sms, cudaStream_t st)
{
    const int es = int(sizeof(T));
    const bool wide = aligned16(a.x) && aligned16(a.out) && aligned16(a.residual) && (a.d.ld_x * es) % 16 == 0 && (a.d.ld_out * es) % 16 == 0 &&
                      (!a.residual || (a.d.ld_res * es) % 16 == 0);
    return a.d.cols <= Lanes<T>::N ? dropout<T, 1>(a, wide, num_sms, st) : dropout<T, 8>(a, wide, num_sms, st);
}

template <typename T, int ACT> cudaError_t linear_grad(const LinearGradArgs &a, cudaStream_t st)
{
    const bool wide = aligned16(a.dout) && (a.ld_dout & 7) == 0 && (ACT == RUBICK_ACT_NONE || (aligned16(a.pre) && (a.ld_pre & 7) == 0));
    return launch_chained(wide ? linear_grad_kernel<T, ACT, true> : linear_grad_kernel<T, ACT, false>, dim3(a.strips, a.chunks), dim3(256), 0, 1, st, a);
}
template <typename T> cudaError_t linear_grad(const LinearGradArgs &a, cudaStream_t st)
{
    switch (a.act) {
    case RUBICK_ACT_RELU: return linear_grad<T, RUBICK_ACT_RELU>(a, st);
    case RUBICK_ACT_GELU: return linear_grad<T, RUBICK_ACT_GELU>(a, st);
    case RUBICK_ACT_GELU_TANH: return linear_grad<T, RUBICK_ACT_GELU_TANH>(a, st);
    case RUBICK_ACT_SILU: return linear_grad<T, RUBICK_ACT_SILU>(a, st);
    }
    return linear_grad<T, RUBICK_ACT_NONE>(a, st);
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

// Strips of up to 64 columns, 128 bytes of a row.  (Strips of 256 columns leave 768 columns three blocks that add 296 runs
// each at the end: 59 of 117 us for 16,384 rows.)
void plan_linear_grad(LinearGradArgs &a, int num_sms)
{
    a.lanes = 8;
    while (a.lanes > 1 && (a.lanes / 2) * 8 >= a.cols) a.lanes /= 2;
    a.strips = (a.cols + a.lanes * 8 - 1) / (a.lanes * 8);
    a.chunks = runs(a.rows, a.strips, int64_t(GRAD_WARPS) * (32 / a.lanes), int64_t(num_sms) * 3);
}

cudaError_t launch_linear_grad(const LinearGradArgs &a, int num_sms, cudaStream_t st)
{
    (void)num_sms;
    return a.dtype == RUBICK_BF16 ? linear_grad<train::bf16>(a, st) : linear_grad<train::f16>(a, st);
}

}  // namespace rubick
