// Matrix products of a training step with their epilogues, on the tensor cores.
//
// D[m][n] = sum_k A[m][k] B[n][k], operands of 16 bits, sums in single precision.  A persistent block (or a pair of blocks on
// neighbouring multiprocessors, which share the tile's columns of B) takes tile after tile.  One thread has the tensor-copy
// engine fetch 64 k of both operands into a ring of stages, one thread multiplies them into tensor memory, and eight warps
// take a finished tile out of it while the next one is multiplied into its other half.
#include <type_traits>

#include "product.cuh"
#include "tcgen.cuh"

namespace rubick {
namespace {

using namespace train;

constexpr int BM = 128, BK = 64;                     // rows a block, k a stage
constexpr int THREADS = 384;                         // fetch, multiply, allocate, -, and eight warps that read
constexpr int READERS = 8, FIRST_READER = 4;
constexpr int STAGING = READERS * 4096;              // 32 rows x 128 bytes a warp
constexpr int SHARED_LIMIT = 232448;

template <int BN, bool PAIR> struct Shape {
    static constexpr int CTAS = PAIR ? 2 : 1;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN / CTAS * BK * 2, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = (SHARED_LIMIT - STAGING - 2048) / STAGE > 8 ? 8 : (SHARED_LIMIT - STAGING - 2048) / STAGE;
    static constexpr int SHARED = STAGES * STAGE + STAGING + 1024 + 256;      // 1,024 to begin on such a boundary
    static constexpr uint32_t COLUMNS = 2 * BN;                               // of tensor memory: two tiles
};
struct Tiling { uint32_t tiles_m, tiles_n, each, all; int steps, per; };      // per: k stages of a split

// Tile number -> tile row, tile column, split: eight tile rows at a time, so that what runs at once shares operands in L2.
__device__ __forceinline__ void place(const Tiling &t, uint32_t i, int &m, int &n, int &split)
{
    const uint32_t s = t.all == t.each ? 0 : i / t.each, r = i - s * t.each, band = 8 * t.tiles_n, b = r / band, q = r - b * band;
    const uint32_t high = t.tiles_m - b * 8 < 8 ? t.tiles_m - b * 8 : 8;
    split = int(s);
    n = int(q / high);
    m = int(b * 8 + (q - n * high));
}

__device__ __forceinline__ float ninf() { return __uint_as_float(0xff800000u); }

template <typename T, ProductKind KIND, int ACT, int BN, bool PAIR>
__global__ void __launch_bounds__(THREADS, 1) product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                             const __grid_constant__ ProductArgs a, const __grid_constant__ Tiling t)
{
    using S = Shape<BN, PAIR>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    uint8_t *const shared = raw + (base - smem_addr(raw));
    const uint32_t stages = base, bars = base + S::STAGES * S::STAGE + STAGING;
    const uint32_t full = bars, empty = full + 8 * S::STAGES, done = empty + 8 * S::STAGES, taken = done + 16;
    volatile uint32_t *const words = reinterpret_cast<volatile uint32_t *>(shared + S::STAGES * S::STAGE + STAGING + 16 * S::STAGES + 32);
    volatile uint32_t *const given_up = words;       // [0] someone waited in vain; [1] where the tensor memory begins
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { barrier_init(done + 8 * i, 1); barrier_init(taken + 8 * i, READERS * S::CTAS); }
        barrier_init_done();
        *given_up = 0;
    }
    if (warp == 2) {
        tmem_alloc<PAIR>(smem_addr(const_cast<uint32_t *>(words + 1)), S::COLUMNS);
        tmem_alloc_done<PAIR>();
    }
    tcgen_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();
    tcgen_after_sync();
    const uint32_t tmem = words[1];
    const uint32_t first = blockIdx.x / S::CTAS, step = gridDim.x / S::CTAS;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t round = 0;                      // stages filled so far
            bool fine = true;
            for (uint32_t i = first; fine && i < t.all; i += step) {
                int tm, tn, split;
                place(t, i, tm, tn, split);
                const int m0 = (tm * S::CTAS + int(rank)) * BM, n0 = tn * BN + int(rank) * (BN / S::CTAS);
                const int k0 = split * t.per, k1 = k0 + t.per < t.steps ? k0 + t.per : t.steps;
                for (int k = k0; k < k1; ++k, ++round) {
                    const uint32_t s = round % S::STAGES, into = stages + s * S::STAGE;
                    if (!(fine = barrier_wait(empty + 8 * s, (round / S::STAGES & 1) ^ 1, given_up))) break;
                    if (rank == 0) barrier_expect(full + 8 * s, S::STAGE * S::CTAS);
                    const uint32_t bar = PAIR ? at_rank(full + 8 * s, 0) : full + 8 * s;
                    if (a.a.along_k) tensor_load<PAIR>(into, &map_a, k * BK, m0, bar);
                    else
                        for (int j = 0; j < BM / 64; ++j) tensor_load<PAIR>(into + j * BLOCK_BYTES, &map_a, m0 + 64 * j, k * BK, bar);
                    if (a.b.along_k) tensor_load<PAIR>(into + S::A_BYTES, &map_b, k * BK, n0, bar);
                    else
                        for (int j = 0; j < BN / S::CTAS / 64; ++j) tensor_load<PAIR>(into + S::A_BYTES + j * BLOCK_BYTES, &map_b, n0 + 64 * j, k * BK, bar);
                }
            }
            // given up: the copies in flight write into this block's memory, so they are waited for before it goes
            if (!fine && rank == 0) {
                volatile uint32_t never = 0;
                for (uint32_t r = round > S::STAGES ? round - S::STAGES : 0; r < round; ++r) barrier_wait(full + 8 * (r % S::STAGES), r / S::STAGES & 1, &never);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const bool ak = a.a.along_k, bk = a.b.along_k;
            const uint32_t desc = instruction_desc(std::is_same<T, bf16>::value, ak, bk, BM * S::CTAS, BN);
            const uint64_t da = operand_desc(stages, ak), db = operand_desc(stages + S::A_BYTES, bk);
            const uint32_t sa = operand_step(ak), sb = operand_step(bk);
            uint32_t round = 0, tile = 0;
            bool fine = true;
            for (uint32_t i = first; fine && i < t.all; i += step, ++tile) {
                const int k0 = t.all == t.each ? 0 : int(i / t.each) * t.per, k1 = k0 + t.per < t.steps ? k0 + t.per : t.steps;
                const uint32_t half = tile & 1, d = tmem + half * BN;
                if (!(fine = barrier_wait(taken + 8 * half, (tile / 2 & 1) ^ 1, given_up))) break;
                tcgen_after_sync();
                for (int k = k0; k < k1; ++k, ++round) {
                    const uint32_t s = round % S::STAGES, at = s * (S::STAGE >> 4);
                    if (!(fine = barrier_wait(full + 8 * s, round / S::STAGES & 1, given_up))) break;
                    tcgen_after_sync();
#pragma unroll
                    for (int q = 0; q < BK / 16; ++q) multiply<PAIR>(d, da + at + q * sa, db + at + q * sb, desc, k > k0 || q > 0);
                    multiplied<PAIR>(empty + 8 * s);
                }
                if (fine) multiplied<PAIR>(done + 8 * half);
            }
            if (!fine) {                             // what was multiplied is waited for before the tensor memory goes
                volatile uint32_t never = 0;
                for (uint32_t r = round > S::STAGES ? round - S::STAGES : 0; r < round; ++r) barrier_wait(empty + 8 * (r % S::STAGES), r / S::STAGES & 1, &never);
            }
        }
        __syncwarp();
    } else if (warp >= FIRST_READER) {
        const int quarter = warp & 3, side = (warp - FIRST_READER) >> 2;       // 32 rows, half of the columns
        uint8_t *const mine = shared + S::STAGES * S::STAGE + (warp - FIRST_READER) * 4096;
        const Finish<T, ACT> finish(a);
        const int64_t rows = a.m, cols = a.n;
        uint32_t tile = 0;
        for (uint32_t i = first; i < t.all; i += step, ++tile) {
            int tm, tn, split;
            place(t, i, tm, tn, split);
            const uint32_t half = tile & 1;
            const int64_t m0 = (int64_t(tm) * S::CTAS + rank) * BM + quarter * 32;
            const int64_t n0 = int64_t(tn) * BN + side * (BN / 2);
            if (!barrier_wait(done + 8 * half, tile / 2 & 1, given_up)) break;
            __syncwarp();
            tcgen_after_sync();
            const uint32_t at = tmem + half * BN + side * (BN / 2) + (uint32_t(quarter * 32) << 16);
            if constexpr (KIND == PRODUCT_OUT || KIND == PRODUCT_PART) {
                // 32 rows x 32 sums through shared memory, pieces of 16 bytes exchanged by the row, so that a warp then holds
                // eight neighbouring sums a lane and its accesses cover whole sectors of eight rows
                const int q = (lane & 3) * 2, above = lane >> 2;
                const bool quick = KIND == PRODUCT_OUT && m0 + 32 <= rows && finish.takes_four();
#pragma unroll 1
                for (int c = 0; c < BN / 2 && n0 + c < cols; c += 32) {
                    const int64_t col = n0 + c + q * 4;
                    float v[32], bias[8];
                    if constexpr (KIND == PRODUCT_OUT) finish.load_bias(col, bias);
                    tmem_load32(at + c, v);
#pragma unroll
                    for (int p = 0; p < 8; ++p)
                        *reinterpret_cast<float4 *>(mine + lane * 128 + ((p ^ (lane & 7)) << 4)) = make_float4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
                    __syncwarp();
                    float w[4][8];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint8_t *const line = mine + (r * 8 + above) * 128;
                        const float4 x = *reinterpret_cast<const float4 *>(line + ((q ^ above) << 4)), y = *reinterpret_cast<const float4 *>(line + (((q + 1) ^ above) << 4));
                        w[r][0] = x.x; w[r][1] = x.y; w[r][2] = x.z; w[r][3] = x.w; w[r][4] = y.x; w[r][5] = y.y; w[r][6] = y.z; w[r][7] = y.w;
                    }
                    if constexpr (KIND == PRODUCT_PART) {
                        float *const to = a.part + (int64_t(split) * rows + m0 + above) * finish.ld_acc + col;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if (m0 + above + 8 * r < rows && col < cols) {
                                *reinterpret_cast<float4 *>(to + 8 * r * finish.ld_acc) = make_float4(w[r][0], w[r][1], w[r][2], w[r][3]);
                                *reinterpret_cast<float4 *>(to + 8 * r * finish.ld_acc + 4) = make_float4(w[r][4], w[r][5], w[r][6], w[r][7]);
                            }
                        }
                    } else if (quick && n0 + c + 32 <= cols) {
                        finish.four(m0 + above, col, w, bias);
                    } else {
                        // Edges, and rows at any address: what is eight sums a lane goes back to where it was, and tensors are read and
                        // written a row at a time, a column a lane (eight 2-byte stores a lane would touch every sector 16 times).
                        const int64_t column = n0 + c + lane;
                        const int high = rows - m0 < 32 ? int(rows - m0) : 32;
                        auto cell = [&](int r) { return reinterpret_cast<float *>(mine + r * 128 + (((lane >> 2) ^ (r & 7)) << 4)) + (lane & 3); };
                        bool over = false;
                        for (int pass = 0; pass < 2 && !over; ++pass) {
                            if (pass == 1 && finish.pre) {
                                __syncwarp();
                                if (column < cols)
                                    for (int r = 0; r < high; ++r) finish.pre[(m0 + r) * finish.ld_pre + column] = from_f<T>(*cell(r));
                                __syncwarp();
                            }
#pragma unroll 1
                            for (int r = 0; r < 4; ++r) {
                                uint8_t *const line = mine + (r * 8 + above) * 128;
                                float4 *const fx = reinterpret_cast<float4 *>(line + ((q ^ above) << 4)), *const fy = reinterpret_cast<float4 *>(line + (((q + 1) ^ above) << 4));
                                float u[8] = {fx->x, fx->y, fx->z, fx->w, fy->x, fy->y, fy->z, fy->w};
                                const int64_t row = m0 + above + 8 * r;
                                if (pass == 0) {
                                    if (row < rows && col < cols) finish.accumulate(row, col, u);
#pragma unroll
                                    for (int e = 0; e < 8; ++e) u[e] += bias[e];
                                } else {
                                    finish.activate(row, col, u);
                                }
                                *fx = make_float4(u[0], u[1], u[2], u[3]);
                                *fy = make_float4(u[4], u[5], u[6], u[7]);
                            }
                            over = finish.acc_out != nullptr;
                        }
                        __syncwarp();
                        if (!over && column < cols) {
#pragma unroll 4
                            for (int r = 0; r < high; ++r) {
                                float u = *cell(r);
                                if (finish.residual) u += to_f(finish.residual[(m0 + r) * finish.ld_res + column]);
                                finish.out[(m0 + r) * finish.ld_out + column] = from_f<T>(u);
                            }
                        }
                    }
                    __syncwarp();
                }
            } else if constexpr (KIND == PRODUCT_STATS) {
                // a thread has a row: running maximum and sum of exponentials over its columns
                const int64_t row = m0 + lane;
                const int64_t label = row < rows ? int64_t(a.label[row]) - a.first - n0 : -1;
                float top = ninf(), sum = 0.f;
                for (int c = 0; c < BN / 2; c += 32) {
                    float v[32];
                    tmem_load32(at + c, v);
                    const int64_t left = cols - (n0 + c);
                    if (left <= 0) continue;
                    if (left < 32) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) if (e >= left) v[e] = ninf();
                    }
                    if (__any_sync(0xffffffffu, label >= c && label < c + 32 && label < c + left)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) if (label == c + e && e < left) a.at_label[row] = v[e];
                    }
                    float m = v[0];
#pragma unroll
                    for (int e = 1; e < 32; ++e) m = fmaxf(m, v[e]);
                    m = fmaxf(m, top);
                    const float from = m == ninf() ? 0.f : m;
                    float s0 = 0.f, s1 = 0.f;
#pragma unroll
                    for (int e = 0; e < 32; e += 2) { s0 += ex2((v[e] - from) * LOG2E); s1 += ex2((v[e + 1] - from) * LOG2E); }
                    sum = sum * ex2((top - from) * LOG2E) + (s0 + s1);
                    top = m;
                }
                if (row < rows && n0 < cols) a.stats[(int64_t(tn) * 2 + side) * rows + row] = make_float2(top, sum);
            } else {
                // a thread has a row; 64 columns become 128 bytes of it, written line by line
                const int64_t row = m0 + lane;
                const bool in = row < rows;
                const float from = in ? a.base[row] : 0.f, rest = in && a.rest ? a.rest[row] : 0.f, w = in ? a.weight[row] : 0.f;
                const uint32_t mask = w == 0.f ? 0u : 0xffffffffu;            // (rows that take no part, whatever their logits are)
                const int64_t label = in ? int64_t(a.label[row]) - a.first - n0 : -1;
                for (int c = 0; c < BN / 2; c += 64) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float v[32];
                        tmem_load32(at + c + 32 * h, v);
                        const int here = c + 32 * h;
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = w * ex2(((v[e] - from) - rest) * LOG2E);
                        if (__any_sync(0xffffffffu, label >= here && label < here + 32)) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) if (label == here + e) v[e] -= w;
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint4 p;
                            p.x = pack_pair(v[8 * q], v[8 * q + 1], T()) & mask; p.y = pack_pair(v[8 * q + 2], v[8 * q + 3], T()) & mask;
                            p.z = pack_pair(v[8 * q + 4], v[8 * q + 5], T()) & mask; p.w = pack_pair(v[8 * q + 6], v[8 * q + 7], T()) & mask;
                            *reinterpret_cast<uint4 *>(mine + lane * 128 + (((h * 4 + q) ^ (lane & 7)) << 4)) = p;
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int line = r * 4 + (lane >> 3), q = lane & 7;
                        const uint4 p = *reinterpret_cast<const uint4 *>(mine + line * 128 + ((q ^ (line & 7)) << 4));
                        const int64_t to = m0 + line, col = n0 + c + q * 8;
                        if (to < rows && col < finish.ld_out) *reinterpret_cast<uint4 *>(finish.out + to * finish.ld_out + col) = p;
                    }
                    __syncwarp();
                }
            }
            tcgen_before_sync();
            __syncwarp();
            if (lane == 0) barrier_arrive_at(PAIR ? at_rank(taken + 8 * half, 0) : taken + 8 * half);
        }
    }
    __syncthreads();
    if constexpr (PAIR) cluster_sync();              // the other block's copies, products and arrivals end here as well
    if (warp == 2) {
        tcgen_after_sync();
        tmem_free<PAIR>(tmem, S::COLUMNS);
    }
    if (threadIdx.x == 0 && *given_up && a.status) atomicOr(a.status, DS_COPY_LOST);
}

// The sums of the splits joined, and PRODUCT_OUT's epilogue.
template <typename T, int ACT> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ ProductArgs a)
{
    const Finish<T, ACT> finish(a);
    const int64_t units = (a.n + 7) / 8, all = a.m * units;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += int64_t(gridDim.x) * blockDim.x) {
        const int64_t row = i / units, c = (i - row * units) * 8;
        float v[8] = {}, bias[8];
        finish.load_bias(c, bias);
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
            float p[8];
            load8<float>(a.part + (int64_t(s) * a.m + row) * a.ld_acc, c, a.ld_acc, true, p);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += p[e];
        }
        finish(row, c, v, bias);
    }
}

// Rows laid out anew, on 16-byte boundaries (the copy engine takes no others); up to two matrices at once.
__global__ void __launch_bounds__(256) lay_out_kernel(const __grid_constant__ LayOutArgs a)
{
    const LayOutArgs::One &o = a.one[blockIdx.z];
    const uint16_t *const from = static_cast<const uint16_t *>(o.from);
    uint16_t *const to = static_cast<uint16_t *>(o.to);
    const int64_t units = (o.cols + 7) / 8;
    for (int64_t row = blockIdx.y * 4 + (threadIdx.x >> 6); row < o.rows; row += gridDim.y * 4)
#pragma unroll 2
        for (int64_t u = blockIdx.x * 64 + (threadIdx.x & 63); u < units; u += gridDim.x * 64)
            *reinterpret_cast<uint4 *>(to + row * o.ld_to + u * 8) = load_any(reinterpret_cast<const bf16 *>(from) + row * o.ld_from, u * 8, o.cols);
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static const EncodeTiled found = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult r = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return found;
}

// The copy engine's view of an operand with `dim` rows and k columns: boxes of 64 k x `high` rows, or 64 rows x 64 k.
bool operand_map(CUtensorMap *map, const Operand &o, int dtype, int64_t dim, int64_t k, int high)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {cuuint64_t(o.along_k ? k : dim), cuuint64_t(o.along_k ? dim : k)}, strides[1] = {cuuint64_t(o.ld) * 2};
    const cuuint32_t box[2] = {64, cuuint32_t(o.along_k ? high : 64)}, one[2] = {1, 1};
    return encode(map, dtype == RUBICK_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(o.p), dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, ProductKind KIND, int ACT, int BN, bool PAIR> cudaError_t launch(const ProductArgs &a, int num_sms, cudaStream_t st)
{
    using S = Shape<BN, PAIR>;
    CUtensorMap map_a, map_b;
    if (!operand_map(&map_a, a.a, a.dtype, a.m, a.k, BM) || !operand_map(&map_b, a.b, a.dtype, a.n, a.k, BN / S::CTAS)) return cudaErrorInvalidValue;
    const int64_t tiles_m = (a.m + BM * S::CTAS - 1) / (BM * S::CTAS), tiles_n = (a.n + BN - 1) / BN, steps = (a.k + BK - 1) / BK;
    const int64_t splits = KIND == PRODUCT_PART ? a.splits : 1, all = tiles_m * tiles_n * splits;
    if (all > 0x7fffffff || steps > 0x7fffffff / BK) return cudaErrorInvalidValue;
    const Tiling t = {uint32_t(tiles_m), uint32_t(tiles_n), uint32_t(tiles_m * tiles_n), uint32_t(all), int(steps), int((steps + splits - 1) / splits)};
    const auto kernel = product_kernel<T, KIND, ACT, BN, PAIR>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SHARED);
    if (e != cudaSuccess) return e;
    const int64_t most = num_sms / S::CTAS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned((all < most ? all : most) * S::CTAS));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = S::SHARED;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = S::CTAS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, a, t);
    count_launch();
    return e;
}

template <typename T, int ACT> cudaError_t join(const ProductArgs &a, int num_sms, cudaStream_t st)
{
    const int64_t blocks = (a.m * ((a.n + 7) / 8) + 255) / 256, most = int64_t(num_sms) * 8;
    join_kernel<T, ACT><<<int(blocks < most ? blocks : most), 256, 0, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

template <typename T, int BN, bool PAIR> cudaError_t product(ProductKind kind, const ProductArgs &a, int num_sms, cudaStream_t st)
{
    switch (kind) {
    case PRODUCT_STATS: return launch<T, PRODUCT_STATS, RUBICK_ACT_NONE, BN, PAIR>(a, num_sms, st);
    case PRODUCT_GRAD: return launch<T, PRODUCT_GRAD, RUBICK_ACT_NONE, BN, PAIR>(a, num_sms, st);
    case PRODUCT_OUT:
        switch (a.act) {
        case RUBICK_ACT_RELU: return launch<T, PRODUCT_OUT, RUBICK_ACT_RELU, BN, PAIR>(a, num_sms, st);
        case RUBICK_ACT_GELU: return launch<T, PRODUCT_OUT, RUBICK_ACT_GELU, BN, PAIR>(a, num_sms, st);
        case RUBICK_ACT_GELU_TANH: return launch<T, PRODUCT_OUT, RUBICK_ACT_GELU_TANH, BN, PAIR>(a, num_sms, st);
        case RUBICK_ACT_SILU: return launch<T, PRODUCT_OUT, RUBICK_ACT_SILU, BN, PAIR>(a, num_sms, st);
        }
        return launch<T, PRODUCT_OUT, RUBICK_ACT_NONE, BN, PAIR>(a, num_sms, st);
    case PRODUCT_PART: break;
    }
    const cudaError_t e = launch<T, PRODUCT_PART, RUBICK_ACT_NONE, BN, PAIR>(a, num_sms, st);
    if (e != cudaSuccess) return e;
    switch (a.act) {
    case RUBICK_ACT_RELU: return join<T, RUBICK_ACT_RELU>(a, num_sms, st);
    case RUBICK_ACT_GELU: return join<T, RUBICK_ACT_GELU>(a, num_sms, st);
    case RUBICK_ACT_GELU_TANH: return join<T, RUBICK_ACT_GELU_TANH>(a, num_sms, st);
    case RUBICK_ACT_SILU: return join<T, RUBICK_ACT_SILU>(a, num_sms, st);
    }
    return join<T, RUBICK_ACT_NONE>(a, num_sms, st);
}

// Pairs of blocks (tiles of 256 x 256) where there are enough such tiles for half of the card's pairs; else single blocks
// (128 x 128), with the k dealt out to several where there are fewer tiles than multiprocessors.
bool in_pairs(const ProductArgs &a, int num_sms) { return ((a.m + 255) / 256) * ((a.n + 255) / 256) >= num_sms / 4; }

}  // namespace

int product_splits(const ProductArgs &a, int num_sms)
{
    if (in_pairs(a, num_sms)) return 1;
    const int64_t tiles = ((a.m + BM - 1) / BM) * ((a.n + 127) / 128), steps = (a.k + BK - 1) / BK, most = (steps + 7) / 8;
    int64_t s = num_sms / (tiles < 1 ? 1 : tiles);
    s = s < 2 || most < 2 ? 1 : s < most ? s : most;
    const int64_t per = (steps + s - 1) / s;
    return int((steps + per - 1) / per);              // (no split is left without work)
}

int product_stats_cols(const ProductArgs &a, int num_sms) { return in_pairs(a, num_sms) ? 128 : 64; }

bool product_takes(const Operand &o) { return aligned16(o.p) && (o.ld & 7) == 0; }

cudaError_t launch_lay_out(const LayOutArgs &a, int num_sms, cudaStream_t st)
{
    if (a.n == 0) return cudaSuccess;
    int64_t across = 1, high = 1;
    for (int i = 0; i < a.n; ++i) {
        const int64_t x = (a.one[i].cols + 511) / 512, y = (a.one[i].rows + 3) / 4;
        across = x > across ? x : across;
        high = y > high ? y : high;
    }
    const int64_t places = int64_t(num_sms) * 8;
    across = across < places ? across : places;
    const int64_t most = (places + across - 1) / across;
    high = high < most ? high : most;
    lay_out_kernel<<<dim3(unsigned(across), unsigned(high), a.n), 256, 0, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_product(ProductKind kind, const ProductArgs &a, int num_sms, cudaStream_t st)
{
    if (in_pairs(a, num_sms)) return a.dtype == RUBICK_BF16 ? product<bf16, 256, true>(kind, a, num_sms, st) : product<f16, 256, true>(kind, a, num_sms, st);
    return a.dtype == RUBICK_BF16 ? product<bf16, 128, false>(kind, a, num_sms, st) : product<f16, 128, false>(kind, a, num_sms, st);
}

}  // namespace rubick
