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
//
// Measured on a B200: step over 2,048 x 128,000 bf16, 48 rows padding, 242 us = 4.3 TB/s (383 with a row a cluster and no
// ring), the pipe of the exponentials 53 % and the issue slots 51 % busy; gradient alone 1,000 x 32,000 fp16 33 us = 3.8
// TB/s, its warps waiting for copies (38 % of the warps an SM can hold, two stages a block); forward 2,048 x 128,000 bf16
// 153 us = 3.4 TB/s; 32 x 50,257 bf16 8.2 us, the time of the teacher's two dependent reads and a barrier.

#include <cooperative_groups.h>

#include <type_traits>

#include "train_common.cuh"

namespace rubick {

using namespace train;
namespace cg = cooperative_groups;

namespace {

constexpr int ROW_WARPS = 16, ROW_THREADS = ROW_WARPS * 32;      // a block of a row's cluster
constexpr int BACK_THREADS = 256;                                 // a block of the separate gradient
constexpr int STEP_NV = 8;                                        // vectors a thread of the step holds
constexpr int MAX_RANKS = 8;                                      // the portable cluster size
constexpr double LOG2E_D = 1.4426950408889634;
constexpr float LOG2E = 1.4426950408889634f;
constexpr double LN2_D = 0.6931471805599453;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The vectors of one row: vector v holds the elements v * VE - shift + e; those outside 0 .. vocab - 1 are other rows'.
// Only the first and the last vector can hold such elements (`head`, `tail`: their places, -1 if they do not); what is
// done element by element for those two is kept out of line, so that the loops stay short.
template <typename T> struct RowView {
    static constexpr int VE = Lanes<T>::N;
    const T *row;
    int shift, vocab, vectors, head, tail;
    __device__ RowView(const void *base, int64_t row_index, int64_t ld, int vocab_)
    {
        row = static_cast<const T *>(base) + row_index * ld;
        shift = int((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        vocab = vocab_;
        vectors = (vocab + shift + VE - 1) / VE;
        head = shift ? 0 : -1;
        tail = vectors * VE - shift > vocab ? vectors - 1 : -1;
    }
    __device__ __forceinline__ int first(int v) const { return v * VE - shift; }
    __device__ __forceinline__ bool whole(int v) const { return v != head && v != tail; }
    __device__ __forceinline__ uint4 load(int v) const { return whole(v) ? ld_stream(row + first(v)) : edge_load(row, first(v), vocab); }
    // vector v of a gradient row that may start elsewhere in its 16 bytes than z's (`same`: it does not)
    __device__ __forceinline__ void store(T *out, bool same, int v, const uint4 &r) const
    {
        if (same && whole(v)) st_stream(out + first(v), r);
        else edge_store(out, first(v), vocab, r);
    }
    // -inf in place of other rows' elements of vector v in shared memory
    __device__ __forceinline__ void mask(int v, T *at) const
    {
#pragma unroll 1
        for (int e = 0; e < VE; ++e) if (first(v) + e < 0 || first(v) + e >= vocab) at[e] = from_f<T>(-INFINITY);
    }
    // the elements of vector v that are this row's, from shared memory
    __device__ __forceinline__ void put(T *out, int v, const T *at) const
    {
#pragma unroll 1
        for (int e = 0; e < VE; ++e) if (first(v) + e >= 0 && first(v) + e < vocab) out[first(v) + e] = at[e];
    }

    static __device__ __noinline__ uint4 edge_load(const T *row, int c, int vocab)
    {
        float f[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = c + e >= 0 && c + e < vocab ? to_f(row[c + e]) : -INFINITY;
        return pack16<T>(f);
    }
    static __device__ __noinline__ void edge_store(T *out, int c, int vocab, uint4 r)
    {
        float f[VE];
        unpack16<T>(r, f);
#pragma unroll
        for (int e = 0; e < VE; ++e) if (c + e >= 0 && c + e < vocab) out[c + e] = from_f<T>(f[e]);
    }
};
// a vector of -inf: it changes neither a maximum nor a sum
template <typename T> __device__ __forceinline__ uint4 no_logits()
{
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
    return make_uint4(w, w, w, w);
}

// A row's teacher entries in shared memory.
struct Teacher {
    int32_t *index;               // -1: does not take part
    float *log_q;                 // log2 q
    float *z;                     // the student's logit there
    int32_t *live;                // whether the row has entries
};
struct TeacherSpace {
    int32_t index[RUBICK_MAX_TEACHER_LOGITS];
    float log_q[RUBICK_MAX_TEACHER_LOGITS], z[RUBICK_MAX_TEACHER_LOGITS];
    int32_t live;
    __device__ __forceinline__ Teacher view() { return Teacher{index, log_q, z, &live}; }
};

__device__ __forceinline__ float teacher_logit(const DistillArgs &a, int64_t at)
{
    if (a.d.ttype == RUBICK_BF16) return to_f(static_cast<const bf16 *>(a.teacher)[at]);
    if (a.d.ttype == RUBICK_F16) return to_f(static_cast<const f16 *>(a.teacher)[at]);
    return static_cast<const float *>(a.teacher)[at];
}

// Softmax over the entries of a row and the student's logits at the entries in elements c0 .. c1, by one warp; the
// others meet it at the next barrier.
template <typename T> __device__ __forceinline__ void read_teacher(const DistillArgs &a, int64_t row, const RowView<T> &z, int c0, int c1, const Teacher &t)
{
    const int k = a.d.k, lane = threadIdx.x & 31;
    const float c = LOG2E / a.d.temperature;
    float top = -INFINITY, total = 0.f;
    bool any = false;
    // the first entries' student logits are asked for as soon as their places are known, and awaited last
    constexpr int AHEAD = 4;
    float ahead[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ahead[u] = -INFINITY;
#pragma unroll 4
    for (int j = lane; j < k; j += 32) {
        const int i = a.index[row * k + j];
        const float l = teacher_logit(a, row * k + j);
        const bool in = i >= 0 && i < a.d.vocab && !(l == -INFINITY);
        t.index[j] = in ? i : -1;
        t.log_q[j] = l;
        if (in) { top = fmaxf(top, l); any = true; }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        const int j = lane + 32 * u, i = j < k ? t.index[j] : -1;
        if (i >= 0 && i >= c0 && i < c1) ahead[u] = to_f(z.row[i]);
    }
    any = __any_sync(0xffffffffu, any);
    top = warp_max(top);
    if (top == -INFINITY) top = 0.f;              // only NaN entries: they reach the sum
#pragma unroll 4
    for (int j = lane; j < k; j += 32) total += t.index[j] >= 0 ? ex2((t.log_q[j] - top) * c) : 0.f;
    total = warp_sum(total);
    const float log_total = log2f(total);
#pragma unroll 4
    for (int j = lane; j < k; j += 32) t.log_q[j] = t.index[j] >= 0 ? (t.log_q[j] - top) * c - log_total : -INFINITY;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) if (lane + 32 * u < k) t.z[lane + 32 * u] = ahead[u];
#pragma unroll 4
    for (int j = lane + 32 * AHEAD; j < k; j += 32) {
        const int i = t.index[j];
        t.z[j] = i >= 0 && i >= c0 && i < c1 ? to_f(z.row[i]) : -INFINITY;
    }
    if (lane == 0) *t.live = any;
    __syncwarp();
}

// q of vocabulary entry i: an index listed twice counts with the sum of its entries
__device__ __forceinline__ float teacher_mass(const Teacher &t, int k, int i)
{
    float s = 0.f;
    for (int j = 0; j < k; ++j) if (t.index[j] == i) s += ex2(t.log_q[j]);
    return s;
}

struct Pair { float m, s; };      // maximum of z, sum of 2^((z - m) c)

// maxima in the storage type: exact, and two at a time in 16 bits; NaN loses, and reaches the sum instead
template <typename T> struct Top;
template <> struct Top<float> {
    float m = -INFINITY;
    __device__ __forceinline__ void take(const uint4 &r)
    {
        m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w))));
    }
    __device__ __forceinline__ float get() const { return m; }
};
template <> struct Top<bf16> {
    __nv_bfloat162 m = __nv_bfloat162(__float2bfloat16_rn(-INFINITY), __float2bfloat16_rn(-INFINITY));
    static __device__ __forceinline__ __nv_bfloat162 as(const uint32_t &w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
    __device__ __forceinline__ void take(const uint4 &r) { m = __hmax2(m, __hmax2(__hmax2(as(r.x), as(r.y)), __hmax2(as(r.z), as(r.w)))); }
    __device__ __forceinline__ float get() const { return fmaxf(__low2float(m), __high2float(m)); }
};
template <> struct Top<f16> {
    __half2 m = __half2(__float2half_rn(-INFINITY), __float2half_rn(-INFINITY));
    static __device__ __forceinline__ __half2 as(const uint32_t &w) { return *reinterpret_cast<const __half2 *>(&w); }
    __device__ __forceinline__ void take(const uint4 &r) { m = __hmax2(m, __hmax2(__hmax2(as(r.x), as(r.y)), __hmax2(as(r.z), as(r.w)))); }
    __device__ __forceinline__ float get() const { return fmaxf(__low2float(m), __high2float(m)); }
};

// 2^((v - m) c) is taken as 2^(v c + off) with off = -m c: one instruction for the exponents of two logits.  The product is
// rounded, and every exponent is off by what that took (2^-20 of a row about 12, 2^-9 of one about 30,000); a fused
// product gives it whole, and this factor puts it right once for a sum.
__device__ __forceinline__ float give_back(float m, float c, float off) { return ex2(-fmaf(m, c, off)); }

// From FAR on |m c| has a remainder that moves exponents out of their range (and is infinite for the lowest values, masks of a
// whole stretch of the vocabulary): a warp then moves its part of the row to its maximum first, in the row's own type.
// That is exact for what lies within a factor of two of the maximum; what lies farther has no probability either way.  (The
// step over 2,048 rows of 128,000 bf16 takes 243.0 us with this and 241.3 without; 263 with the far sums out of line.)
// Beyond FARTHEST a remainder is no factor that single precision has.
constexpr float FAR = 1048576.f, FARTHEST = 1073741824.f;
// the same answer for the whole warp
__device__ __forceinline__ bool far_away(float m, float c) { return __any_sync(0xffffffffu, !(fabsf(m) * c < FAR)); }
template <typename T> __device__ __forceinline__ uint4 less(const uint4 &r, float m)
{
    float v[Lanes<T>::N];
    unpack16<T>(r, v);
#pragma unroll
    for (int e = 0; e < Lanes<T>::N; ++e) v[e] -= m;
    return pack16<T>(v);
}
// A part's exponents towards the row's maximum, z c + sub, and the factor for what sub's rounding took; `moved`: what the part
// was moved by.  Where the row is far and the part is not, the part has no probability (or is all -inf): sub stays a number then,
// and the factor one too.
struct Toward { float sub, back; };
__device__ __forceinline__ Toward toward(float shift, float c, float moved)
{
    const float d = shift - moved, sub = fminf(-d * c, FARTHEST);
    return Toward{sub, ex2(fminf(fmaxf(-fmaf(d, c, sub), -64.f), 64.f))};
}

// Of a log-sum given in two parts: the factor that 2^(z c + sub), sub = -lse log2(e), lacks by the rounding of lse, of c and
// of sub (near the row's largest logits; what is far below these has little of its own to lose).
__device__ __forceinline__ float give_back_lse(float lse, float low, float temperature, float c, float sub)
{
    return ex2(-float((double(lse) + double(low)) * double(temperature) * double(c) + double(sub)));
}

// s + sum of 2^(v c + off), pairwise
template <typename T> __device__ __forceinline__ f2 add_exps(const uint4 &r, f2 c, f2 off, f2 s)
{
    f2 v[Lanes<T>::N / 2];
    unpack16<T>(r, v);
#pragma unroll
    for (int e = 0; e < Lanes<T>::N / 2; ++e) {
        const f2 x = fma2(v[e], c, off);
        s = add2(s, pair(ex2(lo(x)), ex2(hi(x))));
    }
    return s;
}
// scale 2^(v c + off)
template <typename T> __device__ __forceinline__ uint4 scaled_exps(const uint4 &r, f2 c, f2 off, f2 scale)
{
    f2 v[Lanes<T>::N / 2];
    unpack16<T>(r, v);
#pragma unroll
    for (int e = 0; e < Lanes<T>::N / 2; ++e) {
        const f2 x = fma2(v[e], c, off);
        v[e] = mul2(scale, pair(ex2(lo(x)), ex2(hi(x))));
    }
    return pack16<T>(v);
}

// the cluster's barrier in its two halves; what was read and written before the arrival is done with by then
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Loss and log-sum of a row, by one warp.  log p is a difference of numbers of ten and more that may nearly meet log q: that
// difference alone is taken in double precision, the logarithm of the sum as exponent and logarithm of the mantissa.  LOW: where
// asked for, the log-sum in two parts (for a forward pass before another; compiled into the step, which has no use for it,
// it cost 14 of 254 us over 2,048 rows of 128,000).
template <bool LOW> __device__ __forceinline__ void write_loss(const DistillArgs &a, int64_t row, const Teacher &t, float shift, float total, bool live)
{
    const int lane = threadIdx.x & 31;
    float log_whole = 0.f, log_rest = log2f(total);
    if (total > 1e-30f && total < 1e30f) {
        const uint32_t bits = __float_as_uint(total);
        log_whole = float(int(bits >> 23) - 127);
        log_rest = log2f(__uint_as_float((bits & 0x007fffffu) | 0x3f800000u));
    }
    float loss = 0.f;
    // in the logits' own unit: the loss of an entry on the lowest value is a number, the same to the base of two at T = 1 is not
    const double unit = LN2_D * double(a.d.temperature), log_total = double(log_whole) + double(log_rest);
    for (int j = lane; live && j < a.d.k; j += 32) {
        const float lq = t.log_q[j], zj = t.z[j], q = ex2(lq);
        const double gap = unit * (double(lq) + log_total) + (double(shift) - double(zj));
        if (t.index[j] >= 0 && !(q == 0.f)) loss = fmaf(q, zj == -INFINITY ? INFINITY : float(gap), loss);
    }
    loss = warp_sum(loss);
    if (lane == 0) {
        a.loss[row] = live ? a.d.temperature * loss : 0.f;
        if (LOW && a.lse_low) {
            const double lse = live ? (double(shift) + unit * log_total) / double(a.d.temperature) : 0.0;
            a.lse[row] = float(lse);
            a.lse_low[row] = isfinite(float(lse)) ? float(lse - double(float(lse))) : 0.f;
        } else if (a.lse) {
            a.lse[row] = live ? fmaf(shift, 1.f / a.d.temperature, LN2 * (log_whole + log_rest)) : 0.f;
        }
    }
}

// One row per cluster.  STEP: the row's vectors stay in registers (NV a thread) and the gradient is written; otherwise
// any number of vectors is read in batches of NV.  Per warp a maximum, then a sum against it: the block's threads meet
// once, at the cluster's barrier, behind which every warp puts all warps' pairs together for itself.
template <typename T, int NV, bool STEP>
__global__ void __launch_bounds__(ROW_THREADS, 2) distill_row_kernel(const __grid_constant__ DistillArgs a)
{
    __shared__ TeacherSpace space;
    const Teacher teacher = space.view();
    __shared__ Pair pairs[ROW_WARPS];
    constexpr int VE = Lanes<T>::N;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = int(cluster.num_blocks()), rank = int(cluster.block_rank());
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = a.d.k;
    const int64_t row = blockIdx.x / ranks;
    const RowView<T> z(a.z, row, a.d.ld, a.d.vocab);
    const int per = (z.vectors + ranks - 1) / ranks;
    const int v0 = rank * per, v1 = v0 + per < z.vectors ? v0 + per : z.vectors, mine = v0 + int(threadIdx.x);
    const float c = LOG2E / a.d.temperature;
    const f2 c2 = both(c);

    uint4 r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) if (mine + i * ROW_THREADS < v1) r[i] = z.load(mine + i * ROW_THREADS);
    // the last warp, which has the fewest vectors, reads the teacher while the row is on its way; the first block
    // takes the loss and so every entry's logit, the others those that they will write
    if (warp == ROW_WARPS - 1) read_teacher<T>(a, row, z, rank ? z.first(v0) : 0, rank ? z.first(v1) : z.vocab, teacher);
    Pair p{-INFINITY, 0.f};
    float moved = 0.f;            // what this warp's part has been moved by
    {
        Top<T> top;
#pragma unroll
        for (int i = 0; i < NV; ++i) if (mine + i * ROW_THREADS < v1) top.take(r[i]);
        p.m = warp_max(top.get());
        float base = p.m == -INFINITY ? 0.f : p.m;
        if (far_away(base, c)) {
#pragma unroll
            for (int i = 0; i < NV; ++i) if (mine + i * ROW_THREADS < v1) r[i] = less<T>(r[i], base);
            moved = base;
            base = 0.f;
        }
        f2 s = 0ull;
#pragma unroll
        for (int i = 0; i < NV; ++i) if (mine + i * ROW_THREADS < v1) s = add_exps<T>(r[i], c2, both(-base * c), s);
        s = mul2(s, both(give_back(base, c, -base * c)));
        if constexpr (!STEP) {
            __syncthreads();
            // a row without entries is not read on
            for (int v = mine + NV * ROW_THREADS; *teacher.live && v - int(threadIdx.x) < v1; v += NV * ROW_THREADS) {
#pragma unroll
                for (int i = 0; i < NV; ++i) if (v + i * ROW_THREADS < v1) r[i] = z.load(v + i * ROW_THREADS);
                Top<T> more;
#pragma unroll
                for (int i = 0; i < NV; ++i) if (v + i * ROW_THREADS < v1) more.take(r[i]);
                const float m = fmaxf(p.m, warp_max(more.get()));
                base = m == -INFINITY ? 0.f : m;
                s = mul2(s, both(ex2((p.m - base) * c)));
                p.m = m;
                if (far_away(base, c)) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) if (v + i * ROW_THREADS < v1) r[i] = less<T>(r[i], base);
                    base = 0.f;
                }
                f2 t = 0ull;
#pragma unroll
                for (int i = 0; i < NV; ++i) if (v + i * ROW_THREADS < v1) t = add_exps<T>(r[i], c2, both(-base * c), t);
                s = fma2(t, both(give_back(base, c, -base * c)), s);
            }
        }
        p.s = warp_sum(lo(s) + hi(s));
    }
    if (lane == 0) pairs[warp] = p;
    cluster_arrive();
    cluster_wait();
    // all warps' pairs of all blocks, lane by lane
    Pair got[MAX_RANKS / 2];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < MAX_RANKS / 2; ++u) {
        const int q = 2 * u + (lane >> 4);        // half a warp per block
        got[u] = q < ranks ? *cluster.map_shared_rank(&pairs[lane & 15], q) : Pair{-INFINITY, 0.f};
        m = fmaxf(m, got[u].m);
    }
    m = warp_max(m);
    const float shift = m == -INFINITY ? 0.f : m;
    float total = 0.f;
#pragma unroll
    for (int u = 0; u < MAX_RANKS / 2; ++u) total = fmaf(got[u].s, ex2((got[u].m - shift) * c), total);
    cluster_arrive();                             // read: the others may go (awaited before this block goes itself)
    total = warp_sum(total);
    const bool live = *teacher.live;
    if (rank == 0 && warp == ROW_WARPS - 1) {
        write_loss<!STEP>(a, row, teacher, shift, total, live);
    }
    if constexpr (STEP) {
        const float up = (a.dloss ? a.dloss[row] : 1.f) * a.d.temperature, inv = total > 0.f || total != total ? 1.f / total : 0.f;
        T *dz = static_cast<T *>(a.dz) + row * a.d.ld;
        const bool same = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z.row) & 15);
        const Toward t = toward(shift, c, moved);
        const f2 off = both(t.sub), scale = both(up * inv * t.back);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = mine + i * ROW_THREADS;
            if (v < v1) z.store(dz, same, v, live ? scaled_exps<T>(r[i], c2, off, scale) : make_uint4(0u, 0u, 0u, 0u));
        }
        __syncthreads();
        for (int j = threadIdx.x; live && j < k; j += ROW_THREADS) {
            const int i = teacher.index[j], v = (i + z.shift) / VE;
            if (i >= 0 && v >= v0 && v < v1) {
                const float pj = ex2((teacher.z[j] - shift) * c) * inv;
                dz[i] = from_f<T>(up * (pj - teacher_mass(teacher, k, i)));
            }
        }
    }
    cluster_wait();
}

// Gradient from a saved log-sum: element-wise, so a row is cut into parts that need nothing of each other.
template <typename T>
__global__ void __launch_bounds__(BACK_THREADS, 4) distill_backward_kernel(const __grid_constant__ DistillArgs a, int parts)
{
    __shared__ TeacherSpace space;
    const Teacher teacher = space.view();
    constexpr int VE = Lanes<T>::N, NV = 4;
    const int64_t row = blockIdx.x / parts;
    const int part = blockIdx.x % parts, k = a.d.k;
    const RowView<T> z(a.z, row, a.d.ld, a.d.vocab);
    const int per = (z.vectors + parts - 1) / parts;
    const int v0 = part * per, v1 = v0 + per < z.vectors ? v0 + per : z.vectors;
    int v = v0 + int(threadIdx.x);
    uint4 r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) if (v + i * BACK_THREADS < v1) r[i] = z.load(v + i * BACK_THREADS);
    if (threadIdx.x >= BACK_THREADS - 32) read_teacher<T>(a, row, z, z.first(v0), z.first(v1), teacher);
    __syncthreads();                                         // the entries' logits are read before they are written over
    const bool live = *teacher.live;
    const float c = LOG2E / a.d.temperature, lse = a.lse_in[row] * LOG2E;
    // single-precision gradients: what the two factors lose by rounding shows in p, so it is added back
    const float given_low = a.lse_low ? a.lse_low[row] : 0.f;
    const float c_low = float(LOG2E_D / double(a.d.temperature) - double(c));
    const float lse_low = float((double(a.lse_in[row]) + double(given_low)) * LOG2E_D - double(lse));
    const float back = sizeof(T) == 2 && a.lse_low ? give_back_lse(a.lse_in[row], given_low, a.d.temperature, c, -lse) : 1.f;
    const auto prob = [&](float x) { return sizeof(T) == 4 ? ex2(fmaf(x, c, -lse) + fmaf(x, c_low, -lse_low)) : back * ex2(fmaf(x, c, -lse)); };
    // a row whose logits are all -inf has a log-sum of -inf and no probabilities
    const float up = (a.dloss ? a.dloss[row] : 1.f) * a.d.temperature;
    const bool none = a.lse_in[row] == -INFINITY;
    T *dz = static_cast<T *>(a.dz) + row * a.d.ld;
    const bool same = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z.row) & 15);
    while (v - int(threadIdx.x) < v1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int w = v + i * BACK_THREADS;
            if (w < v1) {
                uint4 g = make_uint4(0u, 0u, 0u, 0u);
                if (live && !none) {
                    if constexpr (sizeof(T) == 4) {
                        float f[VE];
                        unpack16<T>(r[i], f);
#pragma unroll
                        for (int e = 0; e < VE; ++e) f[e] = f[e] == -INFINITY ? 0.f : up * prob(f[e]);
                        g = pack16<T>(f);
                    } else {
                        g = scaled_exps<T>(r[i], both(c), both(-lse), both(up * back));
                    }
                }
                z.store(dz, same, w, g);
            }
        }
        v += NV * BACK_THREADS;
        if (live) {
#pragma unroll
            for (int i = 0; i < NV; ++i) if (v + i * BACK_THREADS < v1) r[i] = z.load(v + i * BACK_THREADS);
        }
    }
    if (!live) return;
    __syncthreads();
    for (int j = threadIdx.x; j < k; j += BACK_THREADS) {
        const int i = teacher.index[j], w = (i + z.shift) / VE;
        if (i >= 0 && w >= v0 && w < v1) {
            const float pj = none || teacher.z[j] == -INFINITY ? 0.f : prob(teacher.z[j]);
            dz[i] = from_f<T>(up * (pj - teacher_mass(teacher, k, i)));
        }
    }
}

// ---- many rows: clusters that stay, fed by the bulk-copy engine --------------------------------------------------
//
// A cluster takes every n-th row; a block holds its part of the row in registers and meanwhile the parts of the next
// rows are on their way into shared memory.  One more warp per block issues those copies and reads the next row's
// teacher entries, whose two dependent reads (index, then logit) would otherwise stand before every row, and takes the
// loss of the row before.  The blocks of
// a cluster send each other their warps' pairs with asynchronous stores that count towards the receiver's barrier:
// nobody waits for anything but the 8 bytes a warp that it needs.  The teacher's places are corrected by the warp that
// wrote them, so that the block's warps never meet.

enum { RING_STEP, RING_FORWARD, RING_BACKWARD };
constexpr int RING_NV = 8;        // vectors a thread holds
constexpr int RING_STAGES = 2;
constexpr int RING_CLAIMS = 1024; // slots in which the entries of a row find their doubles

struct RingSync {
    uint64_t full[RING_STAGES], empty[RING_STAGES], t_full[2], t_empty[2], x_full[2];
};

// the entries that lie in a block's own part, each place once, with all of its q
struct Own {
    int32_t *index;
    float *z, *mass;
    int32_t *count;
};

__device__ __forceinline__ void bar_init_n(uint64_t *bar, uint32_t n)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// 8 bytes into block `to`'s copy of `at`, counted by its copy of `bar`
__device__ __forceinline__ void send_pair(Pair *at, uint64_t *bar, Pair p, uint32_t to)
{
    uint32_t ra, rb;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(smem_addr(at)), "r"(to));
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rb) : "r"(smem_addr(bar)), "r"(to));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];"
                 ::"r"(ra), "r"(__float_as_uint(p.m)), "r"(__float_as_uint(p.s)), "r"(rb) : "memory");
}

// Lists the entries in elements c0 .. c1, by one warp.  Doubles are found by claiming: every entry writes its number into
// the slot of its index and looks who stayed; only one that lost its slot compares itself with all the others.  Where
// there are doubles, the first of a place takes the q of all of them.
__device__ __forceinline__ void list_own(const Teacher &t, int k, int c0, int c1, uint16_t *claims, const Own &own)
{
    const int lane = threadIdx.x & 31;
    for (int j = lane; j < k; j += 32) if (t.index[j] >= 0) claims[t.index[j] % RING_CLAIMS] = uint16_t(j);
    __syncwarp();
    bool doubles = false;
    for (int j = lane; j < k; j += 32) {
        const int i = t.index[j];
        if (i >= 0 && i >= c0 && i < c1 && claims[i % RING_CLAIMS] != j)
            for (int q = 0; q < k; ++q) doubles |= q != j && t.index[q] == i;
    }
    doubles = __any_sync(0xffffffffu, doubles);
    int n = 0;
    for (int j0 = 0; j0 < k; j0 += 32) {
        const int j = j0 + lane, i = j < k ? t.index[j] : -1;
        bool mine = i >= 0 && i >= c0 && i < c1;    // (a part may begin before its row does: c0 < 0)
        float mass = mine ? ex2(t.log_q[j]) : 0.f;
        if (mine && doubles)
            for (int q = 0; q < k; ++q)
                if (q != j && t.index[q] == i) { mass += ex2(t.log_q[q]); if (q < j) mine = false; }
        const uint32_t set = __ballot_sync(0xffffffffu, mine);
        if (mine) {
            const int at = n + __popc(set & ((1u << lane) - 1u));
            own.index[at] = i; own.z[at] = t.z[j]; own.mass[at] = mass;
        }
        n += __popc(set);
    }
    if (lane == 0) *own.count = n;
    __syncwarp();
}

// RAGGED: rows that do not begin and end on 16-byte boundaries
template <typename T, int M, int MODE, bool RAGGED>
__global__ void __launch_bounds__(M + 32, M == 256 ? 3 : 1) distill_ring_kernel(const __grid_constant__ DistillArgs a, int ranks, int per)
{
    constexpr int VE = Lanes<T>::N, NV = RING_NV, WARPS = M / 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) RingSync sync;
    __shared__ __align__(16) Pair pairs[2][MAX_RANKS * WARPS];
    __shared__ int32_t live_of[2], count_of[2];
    __shared__ float lse_of[2], up_of[2];
    __shared__ Pair sum_of[2];                    // what a row's logits came to: the largest and the sum against it
    __shared__ uint16_t claims[RING_CLAIMS];
    __shared__ uint4 edge[2];                     // gradients of the row's first and last vector where it shares them
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = a.d.k;
    const int rank = blockIdx.x % ranks, clusters = gridDim.x / ranks, first_row = blockIdx.x / ranks;
    const int v0 = rank * per, iters = (per + M - 1) / M, stage_bytes = per * 16;
    const float c = LOG2E / a.d.temperature;
    const auto entries = [&](int b) { return reinterpret_cast<int32_t *>(smem + RING_STAGES * stage_bytes) + b * 6 * k; };
    const auto teacher_at = [&](int b) {
        int32_t *base = entries(b);
        return Teacher{base, reinterpret_cast<float *>(base + k), reinterpret_cast<float *>(base + 2 * k), live_of + b};
    };
    const auto own_at = [&](int b) {
        int32_t *base = entries(b) + 3 * k;
        return Own{base, reinterpret_cast<float *>(base + k), reinterpret_cast<float *>(base + 2 * k), count_of + b};
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < RING_STAGES; ++i) { bar_init_n(sync.full + i, 1); bar_init_n(sync.empty + i, WARPS); }
        for (int i = 0; i < 2; ++i) { bar_init_n(sync.t_full + i, 1); bar_init_n(sync.t_empty + i, WARPS); bar_init_n(sync.x_full + i, 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (MODE == RING_BACKWARD) __syncthreads();
    else { cluster_arrive(); cluster_wait(); }               // no pair is sent to a barrier that is not there yet
    bool lost = false;
    const auto wait = [&](uint64_t *bar, uint32_t parity) {
        if (!lost && !bar_wait(bar, parity)) { lost = true; atomicOr(a.status, DS_COPY_LOST); }
    };

    if (warp == WARPS) {
        // the part of row n, rounded out to 16-byte units; units that may reach out of the tensor itself (of rows that begin or
        // end less than 16 bytes from its own ends) are put together element by element
        const auto issue = [&](int n) {
            const int64_t row = first_row + int64_t(n) * clusters;
            if (row >= a.d.rows) return;
            const RowView<T> z(a.z, row, a.d.ld, a.d.vocab);
            const int v1 = v0 + per < z.vectors ? v0 + per : z.vectors;
            uint8_t *stage = smem + (n % RING_STAGES) * stage_bytes;
            int b0 = v0, b1 = v1 > v0 ? v1 : v0;
            if (RAGGED) {
                if (row * a.d.ld < VE && b0 == 0 && b1 > 0 && !z.whole(0)) {
                    if (lane == 0) *reinterpret_cast<uint4 *>(stage) = z.load(0);
                    b0 = 1;
                }
                if ((a.d.rows - 1 - row) * a.d.ld < VE && b1 == z.vectors && b1 > b0 && !z.whole(b1 - 1)) {
                    if (lane == 0) *reinterpret_cast<uint4 *>(stage + size_t(b1 - 1 - v0) * 16) = z.load(b1 - 1);
                    --b1;
                }
            }
            if (lane == 0) {
                const uint32_t bytes = b1 > b0 ? uint32_t(b1 - b0) * 16 : 0;
                bar_expect(sync.full + n % RING_STAGES, bytes);
                if (bytes) bulk_load(stage + size_t(b0 - v0) * 16, z.row + z.first(b0), bytes, sync.full + n % RING_STAGES);
            }
            __syncwarp();
        };
        // row n is done with: its loss is taken here, where nothing waits for it (in the warps that hold the row it cost
        // 15 of 254 us over 2,048 rows of 128,000)
        const auto finish = [&](int n) {
            const int b = n & 1;
            wait(sync.t_empty + b, (n >> 1) & 1);
            if (MODE != RING_BACKWARD && rank == 0)
                write_loss<MODE == RING_FORWARD>(a, first_row + int64_t(n) * clusters, teacher_at(b), sum_of[b].m, sum_of[b].s, live_of[b]);
            __syncwarp();
        };
        for (int n = 0; n < RING_STAGES; ++n) issue(n);
        int n = 0;
        for (int64_t row = first_row; row < a.d.rows; row += clusters, ++n) {
            const int b = n & 1;
            if (n >= 2) finish(n - 2);
            const RowView<T> z(a.z, row, a.d.ld, a.d.vocab);
            const int v1 = v0 + per < z.vectors ? v0 + per : z.vectors, c0 = z.first(v0), c1 = z.first(v1);
            const bool all = MODE != RING_BACKWARD && rank == 0;         // the loss is this block's
            if (lane == 0) {
                if (MODE == RING_BACKWARD) lse_of[b] = a.lse_in[row];
                if (MODE != RING_FORWARD) up_of[b] = (a.dloss ? a.dloss[row] : 1.f) * a.d.temperature;
            }
            read_teacher<T>(a, row, z, all ? 0 : c0, all ? z.vocab : c1, teacher_at(b));
            if (MODE != RING_FORWARD) list_own(teacher_at(b), k, c0, c1, claims, own_at(b));
            if (lane == 0) bar_arrive(sync.t_full + b);
            wait(sync.empty + n % RING_STAGES, (n / RING_STAGES) & 1);   // the row is in the other warps' registers
            issue(n + RING_STAGES);
        }
        if (MODE != RING_BACKWARD) for (int done = n > 2 ? n - 2 : 0; done < n; ++done) finish(done);
    } else {
        const f2 c2 = both(c);
        int n = 0;
        RowView<T> z(a.z, first_row, a.d.ld, a.d.vocab);
        for (int64_t row = first_row; row < a.d.rows; row += clusters, ++n) {
            const int b = n & 1, st = n % RING_STAGES;
            if (RAGGED) z = RowView<T>(a.z, row, a.d.ld, a.d.vocab);
            const int v1 = v0 + per < z.vectors ? v0 + per : z.vectors, mine = v0 + int(threadIdx.x);
            if (MODE != RING_BACKWARD && threadIdx.x == 0) bar_expect(sync.x_full + b, uint32_t(ranks * WARPS * sizeof(Pair)));
            wait(sync.full + st, (n / RING_STAGES) & 1);
            uint4 r[NV];
            uint8_t *stage = smem + st * stage_bytes;
            // the thread that holds the row's first or last vector clears what is not the row's
            const bool has_head = RAGGED && v0 <= z.head && z.head < v1 && threadIdx.x == 0;
            const bool has_tail = RAGGED && v0 <= z.tail && z.tail < v1 && int(threadIdx.x) == (z.tail - v0) % M;
            if (has_head) z.mask(z.head, reinterpret_cast<T *>(stage));
            if (has_tail) z.mask(z.tail, reinterpret_cast<T *>(stage + size_t(z.tail - v0) * 16));
            // the next copy into this stage comes behind these stores
            if (has_head || has_tail) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i >= iters) continue;                    // (the same for all threads)
                r[i] = no_logits<T>();                       // so that the arithmetic below need not ask
                if (mine + i * M < v1) r[i] = *reinterpret_cast<const uint4 *>(stage + (i * M + int(threadIdx.x)) * 16);
            }
            __syncwarp();
            if (lane == 0) bar_arrive(sync.empty + st);
            float shift = 0.f, total = 0.f, moved = 0.f;     // moved: what this warp's part of the row has been moved by
            if constexpr (MODE != RING_BACKWARD) {
                Top<T> top;
#pragma unroll
                for (int i = 0; i < NV; ++i) if (i < iters) top.take(r[i]);
                Pair p;
                p.m = warp_max(top.get());
                float base = p.m == -INFINITY ? 0.f : p.m;
                if (far_away(base, c)) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) if (i < iters) r[i] = less<T>(r[i], base);
                    moved = base;
                    base = 0.f;
                }
                const f2 off = both(-base * c);
                f2 s = 0ull;
#pragma unroll
                for (int i = 0; i < NV; ++i) if (i < iters) s = add_exps<T>(r[i], c2, off, s);
                p.s = warp_sum(lo(s) + hi(s)) * give_back(base, c, -base * c);
                // the first block has read every logit that it needs before another block may write over it
                wait(sync.t_full + b, (n >> 1) & 1);
                if (lane < ranks) send_pair(&pairs[b][rank * WARPS + warp], sync.x_full + b, p, uint32_t(lane));
                wait(sync.x_full + b, (n >> 1) & 1);
                Pair got[MAX_RANKS * WARPS / 32];
                float m = -INFINITY;
#pragma unroll
                for (int u = 0; u < MAX_RANKS * WARPS / 32; ++u) {
                    const int q = u * 32 + lane;
                    got[u] = q < ranks * WARPS ? pairs[b][q] : Pair{-INFINITY, 0.f};
                    m = fmaxf(m, got[u].m);
                }
                m = warp_max(m);
                shift = m == -INFINITY ? 0.f : m;
#pragma unroll
                for (int u = 0; u < MAX_RANKS * WARPS / 32; ++u) total = fmaf(got[u].s, ex2((got[u].m - shift) * c), total);
                total = warp_sum(total);
            } else {
                wait(sync.t_full + b, (n >> 1) & 1);
            }
            const bool live = live_of[b];
            if (MODE != RING_BACKWARD && threadIdx.x == 0) sum_of[b] = Pair{shift, total};
            if constexpr (MODE != RING_FORWARD) {
                const float up = up_of[b];
                float inv = 1.f, sub = -shift * c, back = 1.f;           // p = inv back 2^(z c + sub)
                bool none = false;
                if (MODE == RING_STEP) {
                    inv = total > 0.f || total != total ? __fdividef(1.f, total) : 0.f;
                    const Toward t = toward(shift, c, moved);
                    sub = t.sub;
                    back = t.back;
                } else {
                    sub = -lse_of[b] * LOG2E;
                    none = lse_of[b] == -INFINITY;
                }
                // single-precision gradients from a saved log-sum: what the factors lose by rounding is added back
                constexpr bool FINE = MODE == RING_BACKWARD && sizeof(T) == 4;
                const float c_low = FINE ? float(LOG2E_D / double(a.d.temperature) - double(c)) : 0.f;
                const float sub_low = FINE ? float(-double(lse_of[b]) * LOG2E_D - double(sub)) : 0.f;
                const auto prob = [&](float x) {
                    if (MODE == RING_STEP) return inv * ex2((x - shift) * c);
                    return x == -INFINITY || none ? 0.f : ex2(FINE ? fmaf(x, c, sub) + fmaf(x, c_low, sub_low) : fmaf(x, c, sub));
                };
                T *dz = static_cast<T *>(a.dz) + row * a.d.ld, *to = dz + z.first(mine);
                const bool some = live && !none;
                // unpacked anew: kept since the sum they would fill the registers
#pragma unroll
                for (int i = 0; i < NV; ++i) asm volatile("" : "+r"(r[i].x), "+r"(r[i].y), "+r"(r[i].z), "+r"(r[i].w));
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (i >= iters) continue;
                    uint4 g = make_uint4(0u, 0u, 0u, 0u);
                    if (some) {
                        if constexpr (FINE) {
                            float f[VE];
                            unpack16<T>(r[i], f);
#pragma unroll
                            for (int e = 0; e < VE; ++e) f[e] = up * prob(f[e]);
                            g = pack16<T>(f);
                        } else {
                            g = scaled_exps<T>(r[i], c2, both(sub), both(up * inv * back));
                        }
                    }
                    if (mine + i * M < v1) {
                        if (!RAGGED || z.whole(mine + i * M)) st_stream(to + i * M * VE, g);
                        else edge[mine + i * M == z.tail] = g;
                    }
                }
                if (has_head) z.put(dz, z.head, reinterpret_cast<const T *>(edge + (z.head == z.tail)));
                if (has_tail && z.tail != z.head) z.put(dz, z.tail, reinterpret_cast<const T *>(edge + 1));
                __syncwarp();                                // this warp's vectors are written
                const Own own = own_at(b);
                const int count = live && !lost ? count_of[b] : 0;
                for (int j = lane; j < count; j += 32) {
                    const int i = own.index[j], u = (i + z.shift) / VE - v0;
                    if (u % M / 32 == warp) dz[i] = from_f<T>(up * (prob(own.z[j]) - own.mass[j]));
                }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(sync.t_empty + b);
        }
    }
    if (MODE != RING_BACKWARD) { cluster_arrive(); cluster_wait(); }
}

template <typename T, int NV, bool STEP> cudaError_t launch_rows(const DistillArgs &a, int ranks, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(a.d.rows * ranks));
    cfg.blockDim = dim3(ROW_THREADS);
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

// How many clusters of `ranks` blocks the current GPU holds at once, asked once per GPU, kernel and shape.
template <typename K> int resident_clusters(K kernel, int threads, int smem, int ranks, int num_sms)
{
    struct Known { const void *kernel; int device, smem, ranks, n; };
    static thread_local Known known[16];
    static thread_local unsigned turn = 0;
    int device = 0, n = 0;
    if (cudaGetDevice(&device) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
    for (const Known &e : known) if (e.kernel == reinterpret_cast<const void *>(kernel) && e.device == device && e.smem == smem && e.ranks == ranks) return e.n;
    if (ranks > 1) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(unsigned(num_sms / ranks * ranks));
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { (void)cudaGetLastError(); n = 0; }
    } else {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess) { (void)cudaGetLastError(); n = 0; }
        n *= num_sms;
    }
    known[turn++ % 16] = Known{reinterpret_cast<const void *>(kernel), device, smem, ranks, n};
    return n;
}

// The ring, where a row fits the registers of up to eight blocks and there is a row for every other resident cluster (step over
// 40 x 128,000 bf16, 48 clusters: 12.8 us against 15.8 by a cluster a row; 100 x 128,000: 20 against 25; 900 x 5,000: 19
// against 27; 24 x 128,000 and 120 x 32,000: 11.8 both).  The gradient alone of rows that one block holds, whose parts need
// nothing of each other, wants three rows a block (900 x 5,000: 17.5 against 12.8; longer rows, 100 x 128,000: 14.9 against
// 17.9, 250 x 32,000: 14.9 against 13.2).  Otherwise *done stays false and nothing is launched.
template <typename T, int M, int MODE, bool RAGGED> cudaError_t launch_ring(const DistillArgs &a, int vectors, int num_sms, cudaStream_t st, bool *done)
{
    const int ranks = (vectors + M * RING_NV - 1) / (M * RING_NV), per = (vectors + ranks - 1) / ranks;
    const int smem = RING_STAGES * per * 16 + 2 * 6 * a.d.k * 4;
    auto kernel = distill_ring_kernel<T, M, MODE, RAGGED>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    // the separate gradient needs no cluster: its parts are blocks that know nothing of each other
    int n = resident_clusters(kernel, M + 32, smem, MODE == RING_BACKWARD ? 1 : ranks, num_sms);
    if (MODE == RING_BACKWARD) n /= ranks;
    if (n < 1 || (MODE == RING_BACKWARD && ranks == 1 ? a.d.rows < 3 * int64_t(n) : a.d.rows * 2 < n)) return cudaSuccess;
    // the gradient's vectors are stored as z's are read: its rows have to lie in their 16 bytes as z's do
    if (MODE != RING_FORWARD && ((reinterpret_cast<uintptr_t>(a.dz) ^ reinterpret_cast<uintptr_t>(a.z)) & 15)) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(n * ranks));
    cfg.blockDim = dim3(M + 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = MODE == RING_BACKWARD ? 1 : ranks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, a, ranks, per);
    count_launch();
    *done = true;
    return e;
}
template <typename T, int MODE> cudaError_t try_ring(const DistillArgs &a, int num_sms, cudaStream_t st, bool *done)
{
    const int vectors = (a.d.vocab + 2 * Lanes<T>::N - 2) / Lanes<T>::N;       // of a row at the worst shift
    *done = false;
    const bool ragged = a.d.ld * int64_t(sizeof(T)) % 16 || reinterpret_cast<uintptr_t>(a.z) % 16 || a.d.vocab % Lanes<T>::N;
    if (vectors <= 256 * RING_NV * MAX_RANKS) return ragged ? launch_ring<T, 256, MODE, true>(a, vectors, num_sms, st, done) : launch_ring<T, 256, MODE, false>(a, vectors, num_sms, st, done);
    if (vectors <= 512 * RING_NV * MAX_RANKS) return ragged ? launch_ring<T, 512, MODE, true>(a, vectors, num_sms, st, done) : launch_ring<T, 512, MODE, false>(a, vectors, num_sms, st, done);
    return cudaSuccess;
}

// Blocks of a row: a power of two up to 8, more while they leave half of the SMs without one (step over 60 x 32,000 bf16: 10.8 us,
// 22.0 with two blocks an SM for the limit; 32 x 50,257 11.8 and 13.8; 8 x 128,000 11.8 both).
constexpr int cluster_limit(int num_sms) { return num_sms / 2; }

template <typename T> cudaError_t forward_of(const DistillArgs &a, int num_sms, cudaStream_t st)
{
    bool done;
    const cudaError_t e = try_ring<T, RING_FORWARD>(a, num_sms, st, &done);
    if (done || e != cudaSuccess) return e;
    const int vectors = a.d.vocab / Lanes<T>::N + 2;
    int ranks = 1;
    while (ranks < MAX_RANKS && a.d.rows * ranks < cluster_limit(num_sms) && vectors > ranks * ROW_THREADS) ranks *= 2;
    return launch_rows<T, 4, false>(a, ranks, st);
}

template <typename T> cudaError_t backward_of(const DistillArgs &a, int num_sms, cudaStream_t st)
{
    bool done;
    const cudaError_t e = try_ring<T, RING_BACKWARD>(a, num_sms, st, &done);
    if (done || e != cudaSuccess) return e;
    const int64_t vectors = a.d.vocab / Lanes<T>::N + 2;
    // up to 32 KB of z a block; less where that leaves SMs without a block (20 x 128,000 bf16: 9.7 us, 12.8 with eight blocks an SM
    // for the limit, each of which reads the teacher; 60 x 32,000 7.7 and 10.8)
    int64_t parts = (vectors + 8 * BACK_THREADS - 1) / (8 * BACK_THREADS);
    while (parts * a.d.rows < int64_t(num_sms) && parts * BACK_THREADS < vectors) parts *= 2;
    if (parts * a.d.rows > 0x7fffffff) parts = 0x7fffffff / a.d.rows;
    distill_backward_kernel<T><<<unsigned(a.d.rows * parts), BACK_THREADS, 0, st>>>(a, int(parts));
    count_launch();
    return cudaGetLastError();
}

template <typename T> cudaError_t step_of(const DistillArgs &a, int num_sms, cudaStream_t st)
{
    bool done;
    cudaError_t e = try_ring<T, RING_STEP>(a, num_sms, st, &done);
    if (done || e != cudaSuccess) return e;
    constexpr int NV = STEP_NV;
    const int vectors = (a.d.vocab + 2 * Lanes<T>::N - 2) / Lanes<T>::N;       // of a row at the worst shift
    int ranks = 1;
    while (ranks < MAX_RANKS && ranks * NV * ROW_THREADS < vectors) ranks *= 2;
    while (ranks < MAX_RANKS && a.d.rows * ranks < cluster_limit(num_sms) && vectors > ranks * ROW_THREADS) ranks *= 2;
    if (ranks * NV * ROW_THREADS >= vectors) return launch_rows<T, NV, true>(a, ranks, st);
    // longer than a cluster's registers: two passes, with the log-sum between them in two parts (one float has ulps of 2^-9
    // about 30,000, and every probability would be off by as much)
    e = forward_of<T>(a, num_sms, st);
    if (e != cudaSuccess) return e;
    DistillArgs b = a;
    b.lse_in = a.lse;
    return backward_of<T>(b, num_sms, st);
}

}  // namespace

#define BY_TYPE(call) (a.d.dtype == RUBICK_BF16 ? call<bf16>(a, num_sms, st) : a.d.dtype == RUBICK_F16 ? call<f16>(a, num_sms, st) : call<float>(a, num_sms, st))
size_t distill_step_scratch(const DistillArgs &a)
{
    const int lanes = a.d.dtype == RUBICK_F32 ? 4 : 8;
    return (a.d.vocab + 2 * lanes - 2) / lanes > MAX_RANKS * STEP_NV * ROW_THREADS ? size_t(a.d.rows) : 0;
}
cudaError_t launch_distill_forward(const DistillArgs &a, int num_sms, cudaStream_t st) { return BY_TYPE(forward_of); }
cudaError_t launch_distill_backward(const DistillArgs &a, int num_sms, cudaStream_t st) { return BY_TYPE(backward_of); }
cudaError_t launch_distill_step(const DistillArgs &a, int num_sms, cudaStream_t st) { return BY_TYPE(step_of); }
#undef BY_TYPE

}  // namespace rubick
