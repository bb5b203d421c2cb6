// Matrix products of a training step with their epilogues, on the tensor cores.
//
// D[m][n] = sum_k A[m][k] B[n][k], operands of 16 bits, sums in single precision.  A persistent block (or a pair of blocks on
// neighbouring multiprocessors, which share the tile's columns of B) takes tile after tile.  Two warps have the tensor-copy
// engine fetch 64 k of an operand each into a ring of stages, one warp multiplies them into tensor memory, and eight warps
// take a finished tile out of it while the next one is multiplied into its other half.
//
// These warps go through their loops whole, and one elected thread issues: in a branch of a single lane the compiler moves
// every operand of a copy or product to a uniform register as if lanes could differ, which cost 0.35 us a stage of a pair
// whatever its width; now it is 0.32 with 256 columns, 0.25 with 192, 0.21 with 128.
//
// What bounds it: large products the tensor cores at the clock that the card's power allows (8,192 x 4,096 -> 16,384 bf16 with
// gelu and pre kept 724 us alone, 1.52 PFLOP/s, 843 between other work; 4,096 x 2,048 -> 8,192 90 us); products of fewer tiles
// than pairs the length of one tile and 5 us before and behind it (2,048 x 5,120 -> 1,280 fp16 56 tiles of 192 columns on 74
// pairs, 25 to 29 us); a few rows the weights' way from memory (32 x 768 -> 50,257 18.6 us, 4.1 TB/s with all that comes after
// it; 4 x 4,096 -> 4,096 9.1 us, of which 5 are a launch's); little depth the sums' way out (16,384 x 64 -> 16,384 136 us,
// 4 TB/s).  Half of the ring's stages do as well for a single tile; a large product lost 10 % with three.
#include <atomic>
#include <type_traits>

#include "product.cuh"
#include "tcgen.cuh"

namespace rubick {
namespace {

using namespace train;

constexpr int BM = 128, BK = 64;                     // rows a block, k a stage
constexpr int THREADS = 384;                         // fetch, multiply, allocate, -, and eight warps that read
constexpr int READERS = 8, FIRST_READER = 4;
constexpr int STAGES = 6, A_BYTES = BM * BK * 2, STAGE = 2 * A_BYTES;          // 128 rows of A, up to 128 of B
constexpr int STAGING = READERS * 4096;              // 32 rows x 128 bytes a warp
constexpr int SHARED = STAGES * STAGE + STAGING + 1024 + 256;                  // 1,024 to begin on such a boundary
constexpr int SINGLE_COLS = 128, PAIR_COLS = 256;    // most columns of a tile
constexpr int SHARE_LINE = SINGLE_COLS * 4 + 16;     // bytes of a row of sums that blocks share (16 apart in the banks)
static_assert(SHARED <= 232448 && BM * SHARE_LINE <= STAGES * STAGE, "what a block may have");

// A product cut into tiles of 128 (256 with a pair) rows and `cols` columns; `per` of the k stages go to each split.
struct Tiling {
    uint32_t tiles_m, tiles_n, each, all;
    int steps, per, cols;
    uint32_t bytes;                                  // of a stage, per block
    uint32_t band_part;                              // 2^32 / (8 tiles_n), rounded up
    uint32_t share, first;                           // blocks of a cluster that share a tile's k, and the first of them all
};
// Up to two products of one launch: the second one's tiles follow the first one's.  With a cluster of single blocks every
// block has one tile, or a share of the k of one.
struct Work { ProductArgs a[2]; Tiling t[2]; uint32_t all, cluster; };
struct Maps { CUtensorMap a[2], b[2]; };

// Pairs of blocks, single blocks, or single blocks for products of up to FEW_ROWS rows, which exchange the operands: a tile is
// 128 columns by all rows (16, 32, 48 or 64 of them), so that a stage is little more than the weights it is there for.
enum Shape : int { SHAPE_PAIR, SHAPE_SINGLE, SHAPE_FEW };
constexpr int FEW_ROWS = 64;

// Tile number -> tile row, tile column, split: eight tile rows at a time, so that what runs at once shares operands in L2.
__device__ __forceinline__ void place(const Tiling &t, uint32_t i, int &m, int &n, int &split)
{
    const uint32_t s = t.all == t.each ? 0 : i / t.each, r = i - s * t.each;
    split = int(s);
    if (t.tiles_m <= 8) {
        n = t.tiles_m == 1 ? int(r) : int(r / t.tiles_m);
        m = int(r - n * t.tiles_m);
        return;
    }
    // r / band by a multiplication: the quotient by the rounded-up reciprocal is never too small, and one too large at most
    const uint32_t band = 8 * t.tiles_n;
    uint32_t b = __umulhi(r, t.band_part);
    if (b * band > r) --b;
    const uint32_t q = r - b * band, high = t.tiles_m - b * 8;
    n = high >= 8 ? int(q >> 3) : int(q / high);
    m = int(b * 8 + (high >= 8 ? q & 7 : q - n * high));
}

__device__ __forceinline__ float ninf() { return __uint_as_float(0xff800000u); }

// 32 x 32 numbers of a warp, a lane a column, become a lane a row.
__device__ __forceinline__ void exchange(uint8_t *mine, int lane, float (&v)[32])
{
#pragma unroll
    for (int e = 0; e < 32; ++e) *reinterpret_cast<float *>(mine + e * 128 + (((lane >> 2) ^ (e & 7)) << 4) + (lane & 3) * 4) = v[e];
    __syncwarp();
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const float4 x = *reinterpret_cast<const float4 *>(mine + lane * 128 + ((p ^ (lane & 7)) << 4));
        v[4 * p] = x.x; v[4 * p + 1] = x.y; v[4 * p + 2] = x.z; v[4 * p + 3] = x.w;
    }
    __syncwarp();
}
// 32 rows of 128 bytes, 16-byte pieces exchanged by the row, to rows of 16-byte boundaries: whole lines at a time.
template <typename T> __device__ __forceinline__ void write_lines(const uint8_t *mine, int lane, T *to, int64_t m0, int64_t rows, int64_t ld, int64_t left)
{
    // (all read before any is written: the compiler cannot know that the two do not meet, and would wait for each in turn)
    const int line = lane >> 3, q = lane & 7;
    uint4 p[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) p[r] = *reinterpret_cast<const uint4 *>(mine + (r * 4 + line) * 128 + ((q ^ ((r * 4 + line) & 7)) << 4));
    if (q * 8 >= left) return;
    T *const first = to + (m0 + line) * ld + q * 8;
    const int64_t step = 4 * ld;
    if (m0 + 32 <= rows) {
#pragma unroll
        for (int r = 0; r < 8; ++r) *reinterpret_cast<uint4 *>(first + r * step) = p[r];
    } else {
#pragma unroll
        for (int r = 0; r < 8; ++r) if (m0 + r * 4 + line < rows) *reinterpret_cast<uint4 *>(first + r * step) = p[r];
    }
}

// Sums in tensor memory are cut off, not rounded, whenever 16 products join them, always towards zero: over 4,096 k that
// takes 2e-6 of a logit.  The loss is a difference of logits in single precision, so its logits are summed up in parts of
// SUM_STEPS x 64 k, which the reading warps add in registers (log-sums off by 1.3e-6 become 1.3e-7); gradients and layers,
// which are rounded to 16 bits, take their sums as they are.
constexpr int SUM_STEPS = 8;
// The reading warps of a pair need 128 registers for that, so they take some of the others': 64 x 128 + 216 x 256 threads' are
// less than the 168 x 384 the block has (checked before a launch).
constexpr int OTHERS_REGISTERS = 64, READERS_REGISTERS = 216;

template <typename T, ProductKind KIND, int ACT, Shape SHAPE>
__global__ void __launch_bounds__(THREADS, 1) product_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Work work)
{
    constexpr bool PAIR = SHAPE == SHAPE_PAIR, FEW = SHAPE == SHAPE_FEW;
    constexpr int CTAS = PAIR ? 2 : 1;
    constexpr bool TWO = KIND == PRODUCT_OUT && ACT == RUBICK_ACT_NONE && !PAIR;      // products there may be
    constexpr uint32_t HALF = PAIR ? PAIR_COLS : SINGLE_COLS, COLUMNS = 2 * HALF;      // of tensor memory: two tiles
    chain_go();
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    uint8_t *const shared = raw + (base - smem_addr(raw));
    const uint32_t stages = base, bars = base + STAGES * STAGE + STAGING;
    const uint32_t full = bars, empty = full + 8 * STAGES, done = empty + 8 * STAGES, taken = done + 16;
    volatile uint32_t *const words = reinterpret_cast<volatile uint32_t *>(shared + STAGES * STAGE + STAGING + 16 * STAGES + 32);
    volatile uint32_t *const given_up = words;       // [0] someone waited in vain; [1] where the tensor memory begins
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // a pair's rank in its cluster; a single block's among those that share its tile
    const bool shared_tiles = !PAIR && KIND == PRODUCT_OUT && (FEW || work.cluster > 1);
    const int mine_is = shared_tiles && blockIdx.x >= work.t[1].first;
    const uint32_t ranks = PAIR ? 2 : shared_tiles ? work.t[mine_is].share : 1;
    const uint32_t rank = PAIR ? cluster_rank() : shared_tiles ? (blockIdx.x - work.t[mine_is].first) % ranks : 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { barrier_init(done + 8 * i, 1); barrier_init(taken + 8 * i, READERS * CTAS); }
        barrier_init_done();
        *given_up = 0;
    }
    if (warp == 2) {
        tmem_alloc<PAIR>(smem_addr(const_cast<uint32_t *>(words + 1)), COLUMNS);
        tmem_alloc_done<PAIR>();
    } else if (threadIdx.x == 96) {
        tensor_prefetch(&maps.a[0]);
        tensor_prefetch(&maps.b[0]);
    }
    tcgen_before_sync();
    if constexpr (PAIR) {
        __syncthreads();
        cluster_sync();
    } else if (warp == 0) {
        // (the first warp fetches: it knows the barriers and does not wait for the tensor memory)
        __syncwarp();
        asm volatile("bar.arrive 1, %0;" ::"n"(THREADS) : "memory");
    } else {
        asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
    }
    tcgen_after_sync();
    const uint32_t tmem = !PAIR && warp == 0 ? 0 : words[1];
    const uint32_t first = !shared_tiles ? blockIdx.x / ranks : (mine_is ? work.t[0].all : 0) + (blockIdx.x - work.t[mine_is].first) / ranks;
    const uint32_t step = shared_tiles ? 0x80000000u : gridDim.x / ranks;
    const uint32_t end = shared_tiles && !mine_is ? work.t[0].all : work.all;     // (blocks that fill a cluster up have no tile)
    chain_wait();

    if (warp < FIRST_READER) {
        if constexpr (KIND == PRODUCT_STATS && PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHERS_REGISTERS));
        if (warp == 0 || warp == 3) {                // one fetches A, one B: a thread's copies go out one after the other
            const bool one = elected(), fetches_a = warp == 0;
            uint32_t round = 0, i = first;           // stages filled so far, tile
            bool fine = true;
            const uint32_t bar0 = PAIR ? at_rank(full, 0) : full;
            // (one loop for each product, so that its maps and sizes are at fixed places: chosen by a variable they cost a fifth of
            // the kernel's rate)
            auto fetch = [&](auto number) {
                constexpr int which = decltype(number)::value;
                const Tiling &t = work.t[which];
                const ProductArgs &a = work.a[which];
                const uint32_t to = which ? end : end < work.t[0].all ? end : work.t[0].all;
                for (; fine && i < to; i += step) {
                    int tm, tn, split;
                    place(t, which ? i - work.t[0].all : i, tm, tn, split);
                    if (!PAIR) split += rank;        // (a tile's blocks; there are no splits beside them)
                    const int m0 = FEW ? tn * BM : (tm * CTAS + (PAIR ? int(rank) : 0)) * BM, n0 = FEW ? 0 : tn * t.cols + (PAIR ? int(rank) * (t.cols / 2) : 0);
                    const int k0 = split * t.per, k1 = k0 + t.per < t.steps ? k0 + t.per : t.steps;
                    const bool ak = FEW ? a.b.along_k : a.a.along_k, bk = FEW || a.b.along_k;
                    const int blocks = (t.cols / CTAS + 63) / 64;
                    const uint32_t bytes = t.bytes * CTAS;
                    for (int k = k0; k < k1; ++k, ++round) {
                        const uint32_t s = round % STAGES, into = stages + s * STAGE, bar = bar0 + 8 * s;
                        if (!(fine = __all_sync(0xffffffffu, barrier_wait(empty + 8 * s, (round / STAGES & 1) ^ 1, given_up)))) break;
                        if (one && fetches_a) {
                            if (!PAIR || rank == 0) barrier_expect(full + 8 * s, bytes);
                            if (ak) tensor_load<PAIR>(into, &maps.a[which], k * BK, m0, bar);
                            else {
#pragma unroll
                                for (int j = 0; j < BM / 64; ++j) tensor_load<PAIR>(into + j * BLOCK_BYTES, &maps.a[which], m0 + 64 * j, k * BK, bar);
                            }
                        } else if (one) {
                            if (bk) tensor_load<PAIR>(into + A_BYTES, &maps.b[which], k * BK, n0, bar);
                            else {
                                tensor_load<PAIR>(into + A_BYTES, &maps.b[which], n0, k * BK, bar);
                                if (blocks > 1) tensor_load<PAIR>(into + A_BYTES + BLOCK_BYTES, &maps.b[which], n0 + 64, k * BK, bar);
                            }
                        }
                        __syncwarp();
                    }
                }
            };
            fetch(std::integral_constant<int, 0>());
            if constexpr (TWO) fetch(std::integral_constant<int, 1>());
            // given up: the copies in flight write into this block's memory, so they are waited for before it goes
            if (!fine && (!PAIR || rank == 0)) {
                volatile uint32_t never = 0;
                for (uint32_t r = round > STAGES ? round - STAGES : 0; r < round; ++r) barrier_wait(full + 8 * (r % STAGES), r / STAGES & 1, &never);
            }
        }
        if (warp == 1 && (!PAIR || rank == 0)) {
            const bool one = elected();
            uint32_t round = 0, tile = 0, i = first;
            bool fine = true;
            auto sum = [&](auto number) {
                constexpr int which = decltype(number)::value;
                const Tiling &t = work.t[which];
                const bool ak = FEW ? work.a[which].b.along_k : work.a[which].a.along_k, bk = FEW || work.a[which].b.along_k;
                const uint32_t desc = instruction_desc(std::is_same<T, bf16>::value, ak, bk, BM * CTAS, t.cols);
                const uint64_t da = operand_desc(stages, ak), db = operand_desc(stages + A_BYTES, bk);
                const uint32_t sa = operand_step(ak), sb = operand_step(bk);
                const uint32_t to = which ? end : end < work.t[0].all ? end : work.t[0].all;
                for (; fine && i < to; i += step) {
                    const int split = !PAIR ? int(rank) : t.all == t.each ? 0 : int((which ? i - work.t[0].all : i) / t.each);
                    const int k0 = split * t.per, k1 = k0 + t.per < t.steps ? k0 + t.per : t.steps;
                    for (int k = k0; fine && k < k1; ++tile) {
                        const int stop = KIND == PRODUCT_STATS && k + SUM_STEPS < k1 ? k + SUM_STEPS : k1;
                        const uint32_t half = tile & 1, d = tmem + half * HALF;
                        if (!(fine = __all_sync(0xffffffffu, barrier_wait(taken + 8 * half, (tile / 2 & 1) ^ 1, given_up)))) break;
                        tcgen_after_sync();
                        for (bool add = false; k < stop; ++k, ++round) {
                            const uint32_t s = round % STAGES, at = s * (STAGE >> 4);
                            if (!(fine = __all_sync(0xffffffffu, barrier_wait(full + 8 * s, round / STAGES & 1, given_up)))) break;
                            tcgen_after_sync();
                            if (one) {
#pragma unroll
                                for (int q = 0; q < BK / 16; ++q) multiply<PAIR>(d, da + at + q * sa, db + at + q * sb, desc, add || q);
                                multiplied<PAIR>(empty + 8 * s);
                            }
                            add = true;
                            __syncwarp();
                        }
                        if (fine && one) multiplied<PAIR>(done + 8 * half);
                        __syncwarp();
                    }
                }
            };
            sum(std::integral_constant<int, 0>());
            if constexpr (TWO) sum(std::integral_constant<int, 1>());
            if (!fine) {                             // what was multiplied is waited for before the tensor memory goes
                volatile uint32_t never = 0;
                for (uint32_t r = round > STAGES ? round - STAGES : 0; r < round; ++r) barrier_wait(empty + 8 * (r % STAGES), r / STAGES & 1, &never);
            }
        }
        __syncwarp();
        if (shared_tiles) cluster_sync();
    } else {
        if constexpr (KIND == PRODUCT_STATS && PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(READERS_REGISTERS));
        const int quarter = warp & 3, side = (warp - FIRST_READER) >> 2;       // 32 rows, half of the columns
        uint8_t *const mine = shared + STAGES * STAGE + (warp - FIRST_READER) * 4096;
        const int which = TWO && first >= work.t[0].all;           // (of two products every block has one tile)
        const Finish<T, ACT> finish(work.a[which]);
        uint32_t tile = 0;
        float running_top = ninf(), running_sum = 0.f;             // few rows: of all of the block's tiles
        // a cluster's tile: eight columns a lane, two rows a warp, every `ranks`-th row of them here
        const int share_row = ((warp - FIRST_READER) * 2 + (lane >> 4)) * int(ranks) + int(rank);
        int64_t share_m0 = 0, share_col = 0;
        float share_bias[8], share_residual[8];
        for (uint32_t i = first; i < end; i += step) {
            const ProductArgs &a = work.a[TWO ? which : 0];
            const Tiling &t = work.t[TWO ? which : 0];
            const int64_t rows = a.m, cols = a.n;
            int tm, tn, split;
            place(t, TWO && which ? i - work.t[0].all : i, tm, tn, split);
            const uint32_t half = tile & 1;
            const int width = KIND == PRODUCT_OUT ? t.cols / 2 : int(HALF) / 2;      // (only sums may be cut otherwise)
            const int64_t m0 = FEW ? side * 32 : (int64_t(tm) * CTAS + (PAIR ? rank : 0)) * BM + quarter * 32;
            const int64_t n0 = FEW ? int64_t(tn) * BM + quarter * 32 : int64_t(tn) * t.cols + side * width;
            if constexpr (KIND == PRODUCT_STATS) {
                // A thread has a row: its columns' logits, summed up a part of the k at a time, then their maximum and the sum of
                // their exponentials.
                constexpr int W = FEW ? 32 : int(HALF) / 2;
                float v[W];
#pragma unroll
                for (int e = 0; e < W; ++e) v[e] = 0.f;
                bool gone = false;
#pragma unroll 1
                for (int k = 0; k < t.steps && !gone; k += SUM_STEPS, ++tile) {
                    const uint32_t now = tile & 1;
                    if (!barrier_wait(done + 8 * now, tile / 2 & 1, given_up)) { gone = true; break; }
                    __syncwarp();
                    tcgen_after_sync();
                    if (!FEW || m0 < rows) {
                        const uint32_t at = tmem + now * HALF + side * W + (uint32_t(quarter * 32) << 16);
#pragma unroll
                        for (int c = 0; c < W; c += 32) {
                            float x[32];
                            tmem_load32(at + c, x);
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[c + e] += x[e];
                        }
                    }
                    tcgen_before_sync();
                    __syncwarp();
                    if (lane == 0) barrier_arrive_at(PAIR ? at_rank(taken + 8 * now, 0) : taken + 8 * now);
                }
                if (gone) break;
                if (FEW && m0 >= rows) continue;                   // (no rows for this half of the warps)
                if constexpr (FEW) exchange(mine, lane, v);
                const int64_t row = m0 + lane, left = cols - n0;
                const int64_t label = row < rows ? int64_t(a.label[row]) - a.first - n0 : -1;
                if (left < W) {
#pragma unroll
                    for (int e = 0; e < W; ++e) if (e >= left) v[e] = ninf();
                }
#pragma unroll
                for (int c = 0; c < W; c += 32)
                    if (__any_sync(0xffffffffu, label >= c && label < c + 32 && label < left)) {
#pragma unroll
                        for (int e = c; e < c + 32; ++e) if (label == e && e < left) a.at_label[row] = v[e];
                    }
                float top = FEW ? running_top : ninf(), s[4] = {};
#pragma unroll
                for (int e = 0; e < W; ++e) top = fmaxf(top, v[e]);
                const float from = top == ninf() ? 0.f : top;
#pragma unroll
                for (int c = 0; c < W; c += 64) {
#pragma unroll
                    for (int h = 0; h < (W < 64 ? 1 : 2); ++h) {
#pragma unroll
                        for (int e = c + 32 * h; e < c + 32 * h + 32; ++e) { v[e] = ex2((v[e] - from) * LOG2E); s[e & 3] += v[e]; }
                        if constexpr (!FEW) {
                            if (finish.out) {
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    const float *const x = v + c + 32 * h + 8 * q;
                                    uint4 p;
                                    p.x = pack_pair(KEPT * x[0], KEPT * x[1], T()); p.y = pack_pair(KEPT * x[2], KEPT * x[3], T());
                                    p.z = pack_pair(KEPT * x[4], KEPT * x[5], T()); p.w = pack_pair(KEPT * x[6], KEPT * x[7], T());
                                    *reinterpret_cast<uint4 *>(mine + lane * 128 + (((h * 4 + q) ^ (lane & 7)) << 4)) = p;
                                }
                            }
                        }
                    }
                    if constexpr (!FEW) {
                        if (finish.out) {
                            __syncwarp();
                            write_lines(mine, lane, finish.out + n0 + c, m0, rows, finish.ld_out, finish.ld_out - n0 - c);
                            __syncwarp();
                        }
                    }
                }
                const float sum = (s[0] + s[1]) + (s[2] + s[3]);
                if constexpr (FEW) {
                    running_sum = fmaf(running_sum, ex2((running_top - from) * LOG2E), sum);
                    running_top = top;
                } else if (row < rows && n0 < cols) {
                    a.stats[(int64_t(tn) * 2 + side) * rows + row] = make_float2(top, sum);
                }
                continue;
            }
            if (shared_tiles) {
                share_m0 = int64_t(tm) * BM;
                share_col = int64_t(tn) * SINGLE_COLS + (lane & 15) * 8;
                if (share_col < cols && share_m0 + share_row < (FEW && a.fold ? a.fold : rows)) {      // (asked for while the sums are still made)
                    finish.load_bias(share_col, share_bias);
                    finish.load_residual(share_m0 + share_row, share_col, share_residual);
                }
            }
            if (!barrier_wait(done + 8 * half, tile / 2 & 1, given_up)) break;
            __syncwarp();
            tcgen_after_sync();
            const uint32_t at = tmem + half * HALF + side * (FEW ? 32 : width) + (uint32_t(quarter * 32) << 16);
            if (FEW && m0 >= rows) {
                // (no rows for this half of the warps)
            } else if (KIND == PRODUCT_OUT && FEW) {
                float v[32];
                tmem_load32(at, v);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (m0 + e < rows) *reinterpret_cast<float *>(shared + (m0 + e) * SHARE_LINE + (quarter * 32 + lane) * 4) = v[e];
            } else if (ranks > 1 && shared_tiles) {
                // this block's share of the sums, for all of the cluster to read (nothing is copied or multiplied any more)
                if (m0 < rows)
#pragma unroll 1
                    for (int c = 0; c < SINGLE_COLS / 2; c += 32) {
                        float v[32];
                        tmem_load32(at + c, v);
                        float4 *const to = reinterpret_cast<float4 *>(shared + (quarter * 32 + lane) * SHARE_LINE + (side * (SINGLE_COLS / 2) + c) * 4);
#pragma unroll
                        for (int p = 0; p < 8; ++p) to[p] = make_float4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
                    }
            } else if constexpr (KIND == PRODUCT_OUT) {
                // 32 rows x 32 sums through shared memory, pieces of 16 bytes exchanged by the row, so that a warp then holds
                // eight neighbouring sums a lane and its accesses cover whole sectors of eight rows
                const int q = (lane & 3) * 2, above = lane >> 2;
                const bool quick = m0 + 32 <= rows && finish.takes_four();
                float *const part = t.all == t.each ? nullptr : a.part + (int64_t(split) * rows + m0 + above) * finish.ld_acc;
                int done_cols = 0;
                if (!part && finish.takes_rows()) {
                    // a thread has a row of 64 sums, which become 128 bytes of it, written line by line
#pragma unroll 1
                    for (; done_cols + 64 <= width && n0 + done_cols + 64 <= cols; done_cols += 64) {
                        float v[64];
                        tmem_load64(at + done_cols, v);
                        if (finish.bias) {
#pragma unroll
                            for (int p = 0; p < 8; ++p) {
                                float bias[8];
                                finish.load_bias(n0 + done_cols + 8 * p, bias);
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[8 * p + e] = fmaf(v[8 * p + e], finish.scale, bias[e]);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 64; ++e) v[e] *= finish.scale;
                        }
#pragma unroll
                        for (int p = 0; p < 8; ++p) {
                            float x[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] = act_value(ACT, v[8 * p + e]);
                            *reinterpret_cast<uint4 *>(mine + lane * 128 + ((p ^ (lane & 7)) << 4)) = pack16<T>(x);
                        }
                        __syncwarp();
                        write_lines(mine, lane, finish.out + n0 + done_cols, m0, rows, finish.ld_out, 64);
                        __syncwarp();
                    }
                }
#pragma unroll 1
                for (int c = done_cols; c < width && n0 + c < cols; c += 32) {
                    const int64_t col = n0 + c + q * 4;
                    float v[32], bias[8];
                    finish.load_bias(col, bias);
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
                    if (part) {
                        float *const to = part + col;
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
                        // (a gradient's sums have nothing but their factor to get)
                        const bool bare = ACT == RUBICK_ACT_NONE && !finish.acc_in && !finish.acc_out && !finish.bias && !finish.pre && !finish.drop.on;
                        bool over = false;
                        for (int pass = 0; pass < 2 && !over && !bare; ++pass) {
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
                            const float factor = bare ? finish.scale : 1.f;
                            T *to = finish.out + m0 * finish.ld_out + column;
                            const T *res = finish.residual ? finish.residual + m0 * finish.ld_res + column : nullptr;
                            // (eight read before they are written, as above)
#pragma unroll 1
                            for (int r = 0; r < high; r += 8) {
                                float u[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) u[e] = *cell(r + e) * factor;
                                if (r + 8 <= high && !res) {
#pragma unroll
                                    for (int e = 0; e < 8; ++e) { *to = from_f<T>(u[e]); to += finish.ld_out; }
                                    continue;
                                }
                                if (res) {
#pragma unroll
                                    for (int e = 0; e < 8; ++e) {
                                        if (r + e < high) u[e] += to_f(*res);
                                        res += finish.ld_res;
                                    }
                                }
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    if (r + e < high) *to = from_f<T>(u[e]);
                                    to += finish.ld_out;
                                }
                            }
                        }
                    }
                    __syncwarp();
                }
            } else {
                // a thread has a row; 64 columns become 128 bytes of it, written line by line
                const int64_t row = m0 + lane;
                const bool in = row < rows;
                const int is = in ? a.label[row] : -1;
                const bool live = is >= 0 && is < a.vocab;
                const float from = live ? a.base[row] : 0.f, rest = live && a.rest ? a.rest[row] : 0.f, w = live ? (a.dloss ? a.dloss[row] : 1.f) * *a.up : 0.f;
                const uint32_t mask = live ? 0xffffffffu : 0u;                // (rows that take no part, whatever their logits are)
                const int64_t label = live ? int64_t(is) - a.first - n0 : -1;
                for (int c = 0; c < (FEW ? 32 : width); c += 64) {
                    float all[FEW ? 32 : 64];
                    if constexpr (FEW) {
                        tmem_load32(at, all);
                        exchange(mine, lane, all);
                    } else {
                        tmem_load64(at + c, all);
                    }
#pragma unroll
                    for (int h = 0; h < (FEW ? 1 : 2); ++h) {
                        float v[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = all[32 * h + e];
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
                            if constexpr (!FEW) *reinterpret_cast<uint4 *>(mine + lane * 128 + (((h * 4 + q) ^ (lane & 7)) << 4)) = p;
                            else if (in && n0 + q * 8 < finish.ld_out) {
                                *reinterpret_cast<uint4 *>(finish.out + row * finish.ld_out + n0 + q * 8) = p;
                                if (a.in_two) {
                                    float high[8];
                                    unpack16<T>(p, high);
#pragma unroll
                                    for (int e = 0; e < 8; ++e) high[e] = v[8 * q + e] - high[e];
                                    uint4 low = pack16<T>(high);
                                    low.x &= mask; low.y &= mask; low.z &= mask; low.w &= mask;
                                    *reinterpret_cast<uint4 *>(finish.out + (rows + row) * finish.ld_out + n0 + q * 8) = low;
                                }
                            }
                        }
                    }
                    if constexpr (FEW) break;
                    __syncwarp();
                    write_lines(mine, lane, finish.out + n0 + c, m0, rows, finish.ld_out, finish.ld_out - n0 - c);
                    __syncwarp();
                }
            }
            tcgen_before_sync();
            __syncwarp();
            if (lane == 0) barrier_arrive_at(PAIR ? at_rank(taken + 8 * half, 0) : taken + 8 * half);
            ++tile;
        }
        if constexpr (KIND == PRODUCT_STATS && FEW) *reinterpret_cast<float2 *>(mine + lane * 8) = make_float2(running_top, running_sum);
        if (shared_tiles) {
            // the blocks' shares added up in their order
            cluster_sync();
            if ((FEW || ranks > 1) && first < end && !*given_up) {
                const int fold = FEW ? work.a[which].fold : 0;
                const int64_t rows = fold ? fold : work.a[which].m, cols = work.a[which].n;
                const uint32_t from_rank = cluster_rank() - rank;
                for (int r = share_row; r < BM && share_m0 + r < rows; r += READERS * 2 * int(ranks)) {
                    const uint32_t from = stages + r * SHARE_LINE + (lane & 15) * 32;
                    float v[8] = {};
                    for (uint32_t below = 0; below <= uint32_t(fold); below += fold ? fold : 1)
#pragma unroll
                    for (int g = 0; g < 8; g += 4) {               // four at a time
                        float4 x[4], y[4];
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            if (g + s < int(ranks)) {
                                const uint32_t there = at_rank(from + below * SHARE_LINE, from_rank + g + s);
                                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[s].x), "=f"(x[s].y), "=f"(x[s].z), "=f"(x[s].w) : "r"(there));
                                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(y[s].x), "=f"(y[s].y), "=f"(y[s].z), "=f"(y[s].w) : "r"(there + 16));
                            }
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            if (g + s < int(ranks)) {
                                v[0] += x[s].x; v[1] += x[s].y; v[2] += x[s].z; v[3] += x[s].w; v[4] += y[s].x; v[5] += y[s].y; v[6] += y[s].z; v[7] += y[s].w;
                            }
                    }
                    if (share_col >= cols) continue;
                    if (r != share_row) finish.load_residual(share_m0 + r, share_col, share_residual);
                    finish(share_m0 + r, share_col, v, share_bias, share_residual);
                }
            }
        }
    }
    __syncthreads();
    if constexpr (KIND == PRODUCT_STATS && FEW) {
        // a block's pair of a row: its warps' quarters joined
        const ProductArgs &a = work.a[0];
        if (threadIdx.x < a.m) {
            const uint8_t *const theirs = shared + STAGES * STAGE + (threadIdx.x >> 5) * 4 * 4096 + (threadIdx.x & 31) * 8;
            float2 p[4];
            float top = ninf(), sum = 0.f;
            for (int w = 0; w < 4; ++w) { p[w] = *reinterpret_cast<const float2 *>(theirs + w * 4096); top = fmaxf(top, p[w].x); }
            const float from = top == ninf() ? 0.f : top;
            for (int w = 0; w < 4; ++w) sum += p[w].y * ex2((p[w].x - from) * LOG2E);
            a.stats[int64_t(blockIdx.x) * a.m + threadIdx.x] = make_float2(top, sum);
        }
    }
    if (PAIR || shared_tiles) cluster_meet();        // (the other blocks' copies, products, arrivals and reads end here as well)
    if (warp == 2) {
        tcgen_after_sync();
        tmem_free<PAIR>(tmem, COLUMNS);
    }
    if (threadIdx.x == 0 && *given_up && work.a[0].status) atomicOr(work.a[0].status, DS_COPY_LOST);
}

// The sums of the splits joined, and PRODUCT_OUT's epilogue; of up to two products.
template <typename T, int ACT> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Work work)
{
    chain_go();
    chain_wait();
    const ProductArgs &a = work.a[blockIdx.y];
    const int splits = a.way.splits;
    if (splits == 1) return;
    const Finish<T, ACT> finish(a);
    const int64_t units = (a.n + 7) / 8, all = a.m * units;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += int64_t(gridDim.x) * blockDim.x) {
        const int64_t row = i / units, c = (i - row * units) * 8;
        float v[8] = {}, bias[8], residual[8];
        finish.load_bias(c, bias);
        finish.load_residual(row, c, residual);
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            float p[8];
            load8<float>(a.part + (int64_t(s) * a.m + row) * a.ld_acc, c, a.ld_acc, true, p);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += p[e];
        }
        finish(row, c, v, bias, residual);
    }
}

// Rows laid out anew, on 16-byte boundaries (the copy engine takes no others); up to two matrices at once.
__global__ void __launch_bounds__(256) lay_out_kernel(const __grid_constant__ LayOutArgs a)
{
    chain_go();
    chain_wait();
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

// Clusters of single blocks that are resident at once on this GPU, one block a multiprocessor: 74 of two, 33 of four, 15 of
// eight (a cluster lies within a group of multiprocessors, and those are not whole multiples).
int resident_clusters(int size)
{
    static std::atomic<int> known[64][4];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 0;
    std::atomic<int> &slot = known[device][size == 2 ? 1 : size == 4 ? 2 : 3];
    int n = slot.load(std::memory_order_relaxed);
    if (n) return n - 1;
    const auto kernel = product_kernel<bf16, PRODUCT_OUT, RUBICK_ACT_NONE, SHAPE_SINGLE>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(64 * size); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = SHARED;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        n = 0;
    }
    slot.store(n + 1, std::memory_order_relaxed);
    return n;
}

// Stages that are summed up in tensor memory at most.  What is cut off there grows with their number (sums of 2,000,000 positive
// products in one go are 0.5 % short, of 131,072 less than half a step of bfloat16), so longer sums are dealt out.
constexpr int64_t LONGEST = 2048;

// How a product is cut.  What a way takes is estimated in microseconds from measured times: a stage takes a pair 0.32 with 256
// columns, 0.25 with 192, 0.21 with 128, a single block of 128 x 128 sums 0.26, smaller ones as much less as they fetch, however
// the operands lie; what does not depend on the tiles is 6 for a pair and 4 for a single block.
ProductWay way_of(ProductKind kind, const ProductArgs &a, int num_sms)
{
    const int64_t steps = (a.k + BK - 1) / BK;
    ProductWay best = {SHAPE_SINGLE, SINGLE_COLS, 1, 1, 3e38f, 0};
    for (const int cols : {256, 192, 128}) {
        if (a.fold || a.in_two) break;
        if (kind != PRODUCT_OUT && cols != PAIR_COLS) continue;
        const int64_t tiles = ((a.m + 255) / 256) * ((a.n + cols - 1) / cols), places = num_sms / 2;
        // up to eight splits, or as many as make few tiles one for every pair (two 64-column operands of 262,144 rows: 198 us with
        // eight blocks of a cluster, 72 so)
        const int64_t whole = tiles < places ? places / tiles : 0;
        for (int64_t i = 1; i <= 9; ++i) {
            int64_t s = i <= 8 ? i : whole;
            if (s * LONGEST < steps && kind == PRODUCT_OUT) s = (steps + LONGEST - 1) / LONGEST;
            else if (s < 1 || (s > 1 && (kind != PRODUCT_OUT || steps < 8 * s || tiles > 64 * places))) continue;       // (what many tiles would gain is too little)
            const int64_t per = (steps + s - 1) / s, splits = (steps + per - 1) / per, waves = (tiles * splits + places - 1) / places;
            const float cost = float(waves) * float(per) * (0.1f + float(cols) * 0.00086f) + 6.f + (splits > 1 ? 4.f + float(splits) * (0.1f + float(a.m) * float(a.n) * 2e-6f) : 0.f);
            if (cost < best.cost) best = ProductWay{SHAPE_PAIR, cols, 1, int(splits), cost, 2 * tiles * splits};
        }
    }
    // single blocks: 128 x 128 sums, or few rows
    for (const Shape shape : {SHAPE_SINGLE, SHAPE_FEW}) {
        if (shape == SHAPE_FEW ? a.m > FEW_ROWS || !a.a.along_k : a.fold || a.in_two) continue;
        const int cols = shape == SHAPE_FEW ? int(a.m + 15) / 16 * 16 : SINGLE_COLS;
        const int64_t tiles = (shape == SHAPE_FEW ? 1 : (a.m + 127) / 128) * ((a.n + 127) / 128);
        const float each = (A_BYTES + cols * 128) * (0.26f / STAGE);
        for (int s = 1; s <= 8; s *= 2) {
            if (s > 1 && (kind != PRODUCT_OUT || steps < 2 * s || tiles > resident_clusters(s))) break;
            if (kind == PRODUCT_OUT && s * LONGEST < steps && !a.fold) continue;
            const int64_t per = (steps + s - 1) / s, waves = (tiles + num_sms - 1) / num_sms;
            if ((steps + per - 1) / per != s) continue;          // (no block is left without work)
            // (a gradient has another one beside it, which has no few rows: two launches instead of one)
            const float cost = float(waves) * float(per) * each + 4.f + (s > 1 ? 1.f : 0.f) + (shape == SHAPE_FEW && a.beside ? 3.f : 0.f);
            if (cost < best.cost) best = ProductWay{shape, cols, s, 1, cost, tiles * s};
        }
    }
    return best;
}

template <typename T, ProductKind KIND, int ACT, Shape SHAPE> cudaError_t launch(ProductArgs *a, int n, int num_sms, cudaStream_t st)
{
    constexpr bool PAIR = SHAPE == SHAPE_PAIR, FEW = SHAPE == SHAPE_FEW;
    constexpr int CTAS = PAIR ? 2 : 1;
    Maps maps;
    Work work = {};
    work.cluster = CTAS;
    for (int i = 0; i < n; ++i) if (uint32_t(a[i].way.share) > work.cluster) work.cluster = a[i].way.share;
    uint32_t blocks_of_shares = 0;
    bool joined = false;
    for (int i = 0; i < n; ++i) {
        const int cols = a[i].way.cols;
        if (!operand_map(&maps.a[i], FEW ? a[i].b : a[i].a, a[i].dtype, FEW ? a[i].n : a[i].m, a[i].k, BM) ||
            !operand_map(&maps.b[i], FEW ? a[i].a : a[i].b, a[i].dtype, FEW ? a[i].m : a[i].n, a[i].k, cols / CTAS)) return cudaErrorInvalidValue;
        if (FEW && !a[i].a.along_k) return cudaErrorInvalidValue;
        const int64_t tiles_m = FEW ? 1 : (a[i].m + BM * CTAS - 1) / (BM * CTAS), tiles_n = (a[i].n + (FEW ? BM : cols) - 1) / (FEW ? BM : cols), steps = (a[i].k + BK - 1) / BK;
        const int64_t parts = PAIR ? a[i].way.splits : a[i].way.share, all = tiles_m * tiles_n * (PAIR ? parts : 1);
        if (work.all + all > 0x7fffffff || steps > 0x7fffffff / BK) return cudaErrorInvalidValue;
        const uint32_t bytes = A_BYTES + (FEW || a[i].b.along_k ? cols / CTAS * 128 : (cols / CTAS + 63) / 64 * BLOCK_BYTES);
        work.a[i] = a[i];
        work.t[i] = Tiling{uint32_t(tiles_m), uint32_t(tiles_n), uint32_t(tiles_m * tiles_n), uint32_t(all), int(steps), int((steps + parts - 1) / parts), cols, bytes,
                           uint32_t(((uint64_t(1) << 32) + 8 * tiles_n - 1) / (8 * tiles_n)), uint32_t(a[i].way.share), blocks_of_shares};
        if (!PAIR && KIND == PRODUCT_OUT && (FEW || work.cluster > 1)) {
            if (all * a[i].way.share > 1 << 20) return cudaErrorInvalidValue;
            blocks_of_shares += (uint32_t(all) * a[i].way.share + work.cluster - 1) / work.cluster * work.cluster;
        }
        work.all += uint32_t(all);
        joined = joined || a[i].way.splits > 1;
    }
    for (int i = n; i < 2; ++i) { maps.a[i] = maps.a[0]; maps.b[i] = maps.b[0]; work.a[i].way.splits = 1; work.t[i].first = 0xffffffffu; }
    const auto kernel = product_kernel<T, KIND, ACT, SHAPE>;
    static std::atomic<uint64_t> ready{0};            // devices, by bits, on which the kernel has its shared memory
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device > 63 || !(ready.load(std::memory_order_relaxed) >> device & 1)) {
        if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED)) != cudaSuccess) return e;
        if constexpr (KIND == PRODUCT_STATS && PAIR) {
            // a block that lacks the registers its warps ask for would wait for them for ever
            cudaFuncAttributes has;
            if ((e = cudaFuncGetAttributes(&has, kernel)) != cudaSuccess) return e;
            if (has.numRegs * THREADS < OTHERS_REGISTERS * 128 + READERS_REGISTERS * 256) return cudaErrorInvalidConfiguration;
        }
        if (device <= 63) ready.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
    }
    const int64_t most = num_sms / CTAS;
    if (n == 2 && !blocks_of_shares && work.all > most) return cudaErrorInvalidValue;
    const unsigned grid = blocks_of_shares ? blocks_of_shares : unsigned((work.all < most ? work.all : most) * CTAS);
    e = launch_chained(kernel, dim3(grid), dim3(THREADS), SHARED, int(work.cluster), st, maps, work);
    if (e != cudaSuccess || !joined) return e;
    int64_t blocks = 1;
    for (int i = 0; i < n; ++i) {
        const int64_t b = (a[i].m * ((a[i].n + 7) / 8) + 255) / 256;
        if (a[i].way.splits > 1 && b > blocks) blocks = b;
    }
    const int64_t places = int64_t(num_sms) * 8;
    return launch_chained(join_kernel<T, ACT>, dim3(unsigned(blocks < places ? blocks : places), n), dim3(256), 0, 1, st, work);
}

template <typename T, ProductKind KIND, int ACT> cudaError_t launch(ProductArgs *a, int n, int num_sms, cudaStream_t st)
{
    switch (a[0].way.shape) {
    case SHAPE_PAIR: return launch<T, KIND, ACT, SHAPE_PAIR>(a, n, num_sms, st);
    case SHAPE_FEW: return launch<T, KIND, ACT, SHAPE_FEW>(a, n, num_sms, st);
    case SHAPE_SINGLE: break;
    }
    return launch<T, KIND, ACT, SHAPE_SINGLE>(a, n, num_sms, st);
}

template <typename T> cudaError_t product(ProductKind kind, ProductArgs *a, int n, int num_sms, cudaStream_t st)
{
    switch (kind) {
    case PRODUCT_STATS: return launch<T, PRODUCT_STATS, RUBICK_ACT_NONE>(a, n, num_sms, st);
    case PRODUCT_GRAD: return launch<T, PRODUCT_GRAD, RUBICK_ACT_NONE>(a, n, num_sms, st);
    case PRODUCT_OUT: break;
    }
    switch (a[0].act) {
    case RUBICK_ACT_RELU: return launch<T, PRODUCT_OUT, RUBICK_ACT_RELU>(a, n, num_sms, st);
    case RUBICK_ACT_GELU: return launch<T, PRODUCT_OUT, RUBICK_ACT_GELU>(a, n, num_sms, st);
    case RUBICK_ACT_GELU_TANH: return launch<T, PRODUCT_OUT, RUBICK_ACT_GELU_TANH>(a, n, num_sms, st);
    case RUBICK_ACT_SILU: return launch<T, PRODUCT_OUT, RUBICK_ACT_SILU>(a, n, num_sms, st);
    }
    return launch<T, PRODUCT_OUT, RUBICK_ACT_NONE>(a, n, num_sms, st);
}

}  // namespace

size_t plan_products(ProductKind kind, ProductArgs *a, int n, int num_sms)
{
    size_t floats = 0;
    for (int i = 0; i < n; ++i) {
        a[i].way = way_of(kind, a[i], num_sms);
        if (a[i].way.splits > 1) {
            if (!a[i].ld_acc) a[i].ld_acc = (a[i].n + 7) & ~int64_t(7);
            a[i].part_at = floats;
            floats += size_t(a[i].way.splits) * a[i].m * a[i].ld_acc;
        }
    }
    return floats;
}

bool product_few(int64_t rows) { return 2 * rows <= FEW_ROWS; }

bool product_keeps(const ProductArgs &a, int num_sms) { return way_of(PRODUCT_STATS, a, num_sms).shape != SHAPE_FEW; }

int64_t product_stats_pairs(const ProductArgs &a, int num_sms)
{
    const ProductWay w = way_of(PRODUCT_STATS, a, num_sms);
    if (w.shape == SHAPE_FEW) return w.blocks < num_sms ? w.blocks : num_sms;
    return (a.n + w.cols / 2 - 1) / (w.cols / 2);
}

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
    return launch_chained(lay_out_kernel, dim3(unsigned(across), unsigned(high), a.n), dim3(256), 0, 1, st, a);
}

cudaError_t launch_products(ProductKind kind, ProductArgs *a, int n, float *part, int num_sms, cudaStream_t st)
{
    // A product is cut by its own sizes, so that it is the same bits alone or with another.  Two share a launch where both are cut
    // into the same kind of tiles of single blocks and every block of theirs has a place at once (83 x 64 -> 704, both gradients:
    // 13.4 us, 23.9 in two launches with their joins); larger ones keep each other's operands out of L2 (4,096 x 2,048 -> 8,192:
    // 242 us together, 214 one after the other).
    for (int i = 0; i < n; ++i) a[i].part = part + a[i].part_at;
    bool together = n == 1;
    if (n == 2 && a[0].way.shape == a[1].way.shape && a[0].way.shape != SHAPE_PAIR) {
        const ProductWay &x = a[0].way, &y = a[1].way;
        const int share = x.share > y.share ? x.share : y.share;
        const int64_t blocks = (x.blocks + share - 1) / share + (y.blocks + share - 1) / share;
        together = blocks <= (share > 1 ? resident_clusters(share) : num_sms);
    }
    for (int i = 0; i < n; i += together ? n : 1) {
        const cudaError_t e = a[0].dtype == RUBICK_BF16 ? product<bf16>(kind, a + i, together ? n : 1, num_sms, st) : product<f16>(kind, a + i, together ? n : 1, num_sms, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace rubick
