// Router of a mixture of experts with its balance loss: softmax over the experts, the k largest logits, their
// weights, and per group of rows the assignments and probability sums that the loss is made of; and its gradient.
//
//   loss = coef / groups * sum_g E / (k n_g^2) sum_e counts_ge S_ge,   S_ge = sum over the group's rows of p_e
//   dlogit_e = p_e (a_e - sum_j a_j p_j),  a_e = dloss coef E counts_ge / (groups k n_g^2),
//   and from the weights' gradients  + w_j (d_j - sum_i w_i d_i) at the chosen (weights that sum to one), or
//   + w_j d_j at the chosen and - p_e sum_i w_i d_i everywhere (raw weights).
//
// A row is spread over a power of two of lanes, EPL elements a lane, so that a warp works on 32 / lanes rows at once
// and nothing of a row leaves the registers.
//
// The choice works on 32-bit keys: the upper bits of the logit, in unsigned order, and in the lower ones the expert's
// number from the top, so that no two keys are equal and the lowest index wins among equal logits.  Sixteen-bit
// logits fit the upper bits whole.  Of single-precision ones some bits are cut off: where two neighbours among the
// first k + 1 keys differ in nothing but these, or a larger logit with the upper bits of the last place was left out, the
// row is chosen again with whole keys.  Every lane sorts its own keys
// once, in two halves, and puts the two lists into shared memory; after that one of the k is a maximum over the lanes'
// first keys and one lane's step down one list, some fifteen instructions for all rows of the warp together.  (Two lists of
// eight take 38 comparators, one of sixteen 63: 800 against 1,020 instructions for four rows of 128, 39 against 43 us for
// 65,536 of them.)  Sixteen elements a lane: fewer leave the steps that a warp's rows share to fewer rows, more make the
// sort dear.
//
// Bound by the latency of one chain, not by memory: four rows of 128 experts are 2 KB and some 800 instructions of a warp, half
// of them for keys, sort and choice, and the choice is k steps of shuffles, a comparison and a load from shared memory that
// wait for one another.  3.7 warps a scheduler, as their registers allow, fill 47 % of the issue slots.  65,536 x 128 fp32, 8
// chosen: 33 us = 1.1 TB/s; three blocks an SM instead of two spill and take as long.  Backward, 131,072 x 256 bf16: 39 us =
// 3.8 TB/s, 65 % of the issue slots.  512 x 8 bf16: 6 us, most of it the joins' waiting for one another.
//
// Probability sums stay in the lane that owns the column until its chunk of rows ends, then go chunk by chunk, in order,
// into the group's sum: the last block of a group to arrive adds them up, the last of all the loss.  Where groups are
// many, each belongs to one warp alone.

#include "train_common.cuh"

namespace rubick {

using namespace train;

namespace {

constexpr int ROUTER_THREADS = 256;
constexpr int ROUTER_WARPS = ROUTER_THREADS / 32;
constexpr int FORWARD_BLOCKS = 2, BACKWARD_BLOCKS = 3;      // blocks an SM holds, by their registers

// unsigned keys in the order of the values: -inf gets 0x007fffff, NaN of either sign 0 (never chosen)
__device__ __forceinline__ uint32_t order_key(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);          // -0 and 0 are equal
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0u;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_NINF = 0x007fffffu;

// column of element i of lane `sub` of a row
template <bool VEC, int VE, int LANES> __device__ __forceinline__ int column(int i, int sub)
{
    return VEC ? ((i / VE) * LANES + sub) * VE + i % VE : i * LANES + sub;
}

// A row's elements of one lane as they come from memory: nothing looks at them before the row's turn, so that the load
// is under way during the row before.
template <typename T, int EPL, bool VEC, int LANES> struct RawRow {
    static constexpr int VE = Lanes<T>::N;
    uint4 v[VEC ? EPL / VE : 1];
    T s[VEC ? 1 : EPL];
    __device__ __forceinline__ void load(const T *row, int sub, int experts)
    {
        if (VEC && experts == LANES * EPL) {
#pragma unroll
            for (int i = 0; i < EPL / VE; ++i) v[i] = ld_stream(row + (i * LANES + sub) * VE);
        } else if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < EPL / VE; ++i) {
                const int c = (i * LANES + sub) * VE;
                if (c + VE <= experts) v[i] = ld_stream(row + c);
                else {
                    float f[VE];
#pragma unroll
                    for (int e = 0; e < VE; ++e) f[e] = c + e < experts ? to_f(row[c + e]) : -INFINITY;
                    v[i] = pack16<T>(f);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < EPL; ++i) s[i] = i * LANES + sub < experts ? row[i * LANES + sub] : from_f<T>(-INFINITY);
        }
    }
    __device__ __forceinline__ void get(f2 (&f)[EPL / 2]) const
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < EPL / VE; ++i) {
                f2 part[VE / 2];
                unpack16<T>(v[i], part);
#pragma unroll
                for (int e = 0; e < VE / 2; ++e) f[i * VE / 2 + e] = part[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < EPL; i += 2) f[i / 2] = pair(to_f(s[i]), to_f(s[i + 1]));
        }
    }
    __device__ __forceinline__ void get(float (&f)[EPL]) const
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < EPL / VE; ++i) {
                float part[VE];
                unpack16<T>(v[i], part);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[i * VE + e] = part[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < EPL; ++i) f[i] = to_f(s[i]);
        }
    }
};

template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int LANES> __device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    if constexpr (LANES == 32) {
        return __reduce_max_sync(0xffffffffu, v);
    } else {
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    }
}

// Descending sort of a lane's keys by Batcher's odd-even merge network (K. E. Batcher, 1968)
template <int N> __device__ __forceinline__ void sort_keys(uint32_t *s)
{
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const uint32_t x = s[i + j], y = s[i + j + k];
                        s[i + j] = max(x, y); s[i + j + k] = min(x, y);
                    }
}

// The state of a warp's rows while it goes through a chunk
template <int EPL> struct Tally { f2 acc[EPL / 2]; int valid; };

// One row per group of lanes: index, weight and histogram are written, probabilities added to the tally.
template <typename T, int EPL, bool VEC, int LANES>
__device__ __forceinline__ void route_rows(const RouterArgs &a, int64_t row, bool here, const f2 (&z)[EPL / 2], int sub,
                                           uint32_t *sorted, uint32_t *list, float *kept, int32_t *hist, Tally<EPL> &tally)
{
    constexpr int VE = Lanes<T>::N, lanes = LANES;
    constexpr bool WARP = LANES == 32;
    constexpr uint32_t low = LANES * EPL - 1;     // a power of two less one
    const int k = a.d.k;
    // keys; -0 counts as 0 (a NaN may be anywhere: the row's sum shows it)
    uint32_t key[EPL];
#pragma unroll
    for (int i = 0; i < EPL; i += 2) {
        const f2 v = add2(z[i / 2], 0ull);
        const uint32_t b0 = uint32_t(v), b1 = uint32_t(v >> 32);
        key[i] = ((b0 ^ (uint32_t(int32_t(b0) >> 31) | 0x80000000u)) & ~low) | (low - uint32_t(column<VEC, VE, LANES>(i, sub)));
        key[i + 1] = ((b1 ^ (uint32_t(int32_t(b1) >> 31) | 0x80000000u)) & ~low) | (low - uint32_t(column<VEC, VE, LANES>(i + 1, sub)));
    }
    if constexpr (sizeof(T) == 4) {
        // the chosen logits are looked up whole
#pragma unroll
        for (int i = 0; i < EPL; i += VEC ? 4 : 2) {
            if constexpr (VEC) {
                *reinterpret_cast<float4 *>(kept + column<VEC, VE, LANES>(i, sub)) = make_float4(lo(z[i / 2]), hi(z[i / 2]), lo(z[i / 2 + 1]), hi(z[i / 2 + 1]));
            } else {
                kept[column<VEC, VE, LANES>(i, sub)] = lo(z[i / 2]);
                kept[column<VEC, VE, LANES>(i + 1, sub)] = hi(z[i / 2]);
            }
        }
    }
    sort_keys<EPL / 2>(key);
    sort_keys<EPL / 2>(key + EPL / 2);
    // this lane's two lists, 32 words from one key to the next; behind each a 0 (written once, at the start)
#pragma unroll
    for (int i = 1; i < EPL / 2; ++i) { sorted[i * 32] = key[i]; sorted[(EPL / 2 + 1 + i) * 32] = key[EPL / 2 + i]; }
    uint32_t mine = 0u, head0 = key[0], head1 = key[EPL / 2];
    const uint32_t *next0 = sorted + 32, *next1 = sorted + (EPL / 2 + 2) * 32;
    uint32_t next = lanes_max<LANES>(max(head0, head1));
    const uint32_t first = next, none = KEY_NINF | low;      // up to `none`: closed, or not a column
    bool near = false;                            // two neighbours that only the cut-off bits may tell apart
#pragma unroll 2
    for (int j = 0; j < k; ++j) {
        // keys are never 0 before the lists end, and k places do not reach that end
        if (LANES >= RUBICK_MAX_CHOSEN) mine = sub == j ? next : mine;
        else if (sub == (j & (lanes - 1))) list[j] = next;
        if (head0 == next) { head0 = *next0; next0 += 32; }
        if (head1 == next) { head1 = *next1; next1 += 32; }
        const uint32_t above = next;
        next = lanes_max<LANES>(max(head0, head1));
        if (sizeof(T) == 4) near |= (above ^ next) <= low && next > none;
    }
    const bool some = first > none;
    // The exponents are taken against what the keys leave of the largest logit, times log2(e) and rounded: both are off by a
    // share of the logit, the same for the whole row, which divides out again.  From FAR on that share could move an exponent
    // out of its range (of a few million, and infinite for the lowest values): then against the largest logit itself, the
    // differences before the product.  (Always so: 2 to 4 % more for 65,536 x 128 fp32, 33 us; this costs nothing.)
    constexpr float FAR = 1024.f;
    const uint32_t cut = first & ~low;
    float shift = some ? __uint_as_float(cut & 0x80000000u ? cut & 0x7fffffffu : ~(cut | low)) : 0.f;
    const float off = -shift * 1.4426950408889634f;
    const bool far = __any_sync(0xffffffffu, fabsf(shift) >= FAR);
    f2 e[EPL / 2], sums = 0ull;
#pragma unroll
    for (int i = 0; i < EPL / 2; ++i) e[i] = fma2(z[i], both(1.4426950408889634f), both(off));
    if (far) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < EPL / 2; ++i) top = fmaxf(top, fmaxf(lo(z[i]), hi(z[i])));
        top = lanes_max<LANES>(top);
        shift = some ? top : 0.f;
#pragma unroll
        for (int i = 0; i < EPL / 2; ++i) e[i] = mul2(add2(z[i], both(-shift)), both(1.4426950408889634f));
    }
#pragma unroll
    for (int i = 0; i < EPL / 2; ++i) {
        float e0, e1;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(lo(e[i])));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(hi(e[i])));
        e[i] = pair(e0, e1);
        sums = add2(sums, e[i]);
    }
    const float total = lanes_sum<LANES>(lo(sums) + hi(sums));
    const float inv = some ? __fdividef(1.f, total) : 0.f;
#pragma unroll
    for (int i = 0; i < EPL / 2; ++i) tally.acc[i] = fma2(e[i], both(inv), tally.acc[i]);
    tally.valid += (some || total != total) && sub == 0 ? 1 : 0;      // (a NaN counts as above -inf)
    if (!WARP || sizeof(T) == 4) __syncwarp();
    // A NaN, or neighbours that only the cut-off bits tell apart: once more, with whole keys.
    bool unsure = total != total;
    if constexpr (sizeof(T) == 4) {
        if (__any_sync(0xffffffffu, near)) {
            const uint32_t below = WARP ? __shfl_down_sync(0xffffffffu, mine, 1) : 0u;
            for (int j = sub; j < k; j += lanes) {
                const uint32_t x = WARP ? mine : list[j], y = j + 1 == k ? next : WARP ? below : list[j + 1];
                unsure |= (x ^ y) <= low && x > none && kept[low - (x & low)] != kept[low - (y & low)];
            }
            // Behind the last place and an equal next one there may be a larger logit of the same upper bits: every lane looks
            // among its own.  (Logits that are all equal, as those of weights that begin at zero, cost no second choice:
            // 65,536 x 128 take 33 us instead of 72.)
            const uint32_t last = WARP ? __shfl_sync(0xffffffffu, mine, k - 1) : list[k - 1];
            if ((last ^ next) <= low && next > none) {
                const float v = kept[low - (last & low)] + 0.f;
#pragma unroll
                for (int i = 0; i < EPL / 2; ++i) {
                    const float z0 = lo(z[i]), z1 = hi(z[i]);
                    unsure |= z0 > v && (__float_as_uint(z0) ^ __float_as_uint(v)) <= low;
                    unsure |= z1 > v && (__float_as_uint(z1) ^ __float_as_uint(v)) <= low;
                }
            }
        }
    }
    if (__any_sync(0xffffffffu, unsure)) {
        uint32_t whole[EPL];
#pragma unroll
        for (int i = 0; i < EPL; i += 2) { whole[i] = order_key(lo(z[i / 2])); whole[i + 1] = order_key(hi(z[i / 2])); }
        __syncwarp();
#pragma unroll 1
        for (int j = 0; j < k; ++j) {
            uint32_t best = 0u;
            int col = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                const int c = column<VEC, VE, LANES>(i, sub);
                if (whole[i] > best || (whole[i] == best && c < col && best)) { best = whole[i]; col = c; }
            }
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) {
                const uint32_t kb = __shfl_xor_sync(0xffffffffu, best, o);
                const int cb = __shfl_xor_sync(0xffffffffu, col, o);
                if (kb > best || (kb == best && cb < col)) { best = kb; col = cb; }
            }
            // the key of that column as above; 0 where nothing is open
            const uint32_t m = best > KEY_NINF ? (best & ~low) | (low - uint32_t(col)) : 0u;
            if (LANES >= RUBICK_MAX_CHOSEN) mine = sub == j ? m : mine;
            else if (sub == (j & (lanes - 1))) list[j] = m;
#pragma unroll
            for (int i = 0; i < EPL; ++i) if (column<VEC, VE, LANES>(i, sub) == col) whole[i] = 0u;
        }
        __syncwarp();
    }
    // places: lane j of the row has the j-th (and the j + lanes-th ...)
    float sum = 0.f;
    for (int j = sub; j < k; j += lanes) {
        const uint32_t m = WARP ? mine : list[j];
        const int col = int(low - (m & low));
        const bool ok = m > none;
        const uint32_t b = m & ~low;
        const float logit = sizeof(T) == 4 ? (ok ? kept[col] : 0.f) : __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~(b | low));
        float w;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(far ? (logit - shift) * 1.4426950408889634f : fmaf(logit, 1.4426950408889634f, off)));
        w = ok ? w * inv : 0.f;
        sum += w;
        if (here) {
            a.index[row * k + j] = ok ? col : -1;
            if (!(a.d.flags & RUBICK_ROUTER_RENORM)) a.weight[row * k + j] = w;
            else if (!WARP) list[j] = __float_as_uint(w);     // (this lane's own place)
            else mine = __float_as_uint(w);
            if (ok) atomicAdd(hist + col, 1);
        }
    }
    if (a.d.flags & RUBICK_ROUTER_RENORM) {
        sum = lanes_sum<LANES>(sum);
        const float share = sum > 0.f || sum != sum ? __fdividef(1.f, sum) : 0.f;
        for (int j = sub; here && j < k; j += lanes) a.weight[row * k + j] = __uint_as_float(WARP ? mine : list[j]) * share;
    }
    if (!WARP || sizeof(T) == 4) __syncwarp();    // list and kept are free again
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
        const float loss = valid > 0 ? dot * float(a.d.experts) / (float(a.d.k) * n * n) : 0.f;
        a.valid[g] = valid;
        a.group_loss[g] = loss;
        if (a.groups == 1) *a.loss = a.d.coef * loss;
    }
}

// What the last block of a group does: the chunks' sums, every warp a run of them, then the warps' sums in order (a block
// that joins takes no further group: there are chunks only where groups are fewer than blocks).  JOIN columns at a time,
// all their loads under way together.  `red`: 2 x [warps][JOIN] words.
constexpr int JOIN = 128;
__device__ void join_group(const RouterArgs &a, int64_t g, float *red)
{
    __shared__ int32_t valid_rows;
    const int E = a.d.experts, C = a.chunks, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t *pc = a.part_counts + g * C * (E + 1);
    const float *ps = a.part + g * C * E;
    int32_t *red_n = reinterpret_cast<int32_t *>(red + ROUTER_WARPS * JOIN);
    if (threadIdx.x == 0) valid_rows = 0;
    __syncthreads();
    int valid = 0;
    for (int q = threadIdx.x; q < C; q += ROUTER_THREADS) valid += __ldcg(pc + int64_t(q) * (E + 1) + E);
    const int run = (C + ROUTER_WARPS - 1) / ROUTER_WARPS, q0 = warp * run, q1 = q0 + run < C ? q0 + run : C;
    float dot = 0.f;
    for (int e0 = 0; e0 < E; e0 += JOIN) {
        int n[JOIN / 32];
        float s[JOIN / 32];
#pragma unroll
        for (int u = 0; u < JOIN / 32; ++u) { n[u] = 0; s[u] = 0.f; }
#pragma unroll 2
        for (int q = q0; q < q1; ++q)
#pragma unroll
            for (int u = 0; u < JOIN / 32; ++u) {
                const int e = e0 + u * 32 + lane;
                if (e < E) { n[u] += __ldcg(pc + int64_t(q) * (E + 1) + e); s[u] += __ldcg(ps + int64_t(q) * E + e); }
            }
        if (e0) __syncthreads();                  // the columns before are read
        else {
            valid = __reduce_add_sync(0xffffffffu, valid);
            if (lane == 0 && valid) atomicAdd(&valid_rows, valid);
        }
#pragma unroll
        for (int u = 0; u < JOIN / 32; ++u) { red[warp * JOIN + u * 32 + lane] = s[u]; red_n[warp * JOIN + u * 32 + lane] = n[u]; }
        __syncthreads();
        const int e = e0 + int(threadIdx.x);
        if (threadIdx.x < JOIN && e < E) {
            int m = 0;
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < ROUTER_WARPS; ++w) { m += red_n[w * JOIN + threadIdx.x]; t += red[w * JOIN + threadIdx.x]; }
            a.counts[g * E + e] = m;
            a.prob_sum[g * E + e] = t;
            dot = fmaf(float(m), t, dot);
        }
    }
    finish_group(a, g, dot, valid_rows);
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

// Goes through rows first, first + stride, ... below end, 32 / LANES at a time, with the next ones on their way.
template <typename T, int EPL, bool VEC, int LANES>
__device__ __forceinline__ void route_chunk(const RouterArgs &a, int64_t first, int64_t end, int64_t stride, int sub, int slot,
                                            uint32_t *sorted, uint32_t *list, float *kept, int32_t *hist, Tally<EPL> &tally)
{
    RawRow<T, EPL, VEC, LANES> next;
    uint8_t mask = 1;
    const auto fetch = [&](int64_t row) {
        const int64_t at = row < end ? row : first;      // (a row that is there)
        if (a.mask) mask = a.mask[at];
        next.load(static_cast<const T *>(a.logits) + at * a.d.ld, sub, a.d.experts);
    };
    if (first < end) fetch(first + slot);
    for (int64_t row = first; row < end; row += stride) {
        f2 z[EPL / 2];
        next.get(z);
        const bool out = !mask || row + slot >= end;
        if (__any_sync(0xffffffffu, out)) {       // what stands in a masked row is not looked at
#pragma unroll
            for (int i = 0; i < EPL / 2; ++i) z[i] = out ? both(-INFINITY) : z[i];
        }
        if (row + stride < end) fetch(row + stride + slot);
        route_rows<T, EPL, VEC, LANES>(a, row + slot, row + slot < end, z, sub, sorted, list, kept, hist, tally);
    }
}

// the sums of a warp's rows, at the lanes of its first row
template <int EPL, int LANES> __device__ __forceinline__ void fold_rows(const Tally<EPL> &t, float (&acc)[EPL], int &valid)
{
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        acc[i] = i & 1 ? hi(t.acc[i / 2]) : lo(t.acc[i / 2]);
#pragma unroll
        for (int o = 16; o >= LANES; o >>= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
    }
    valid = __reduce_add_sync(0xffffffffu, t.valid);
}

// Shared memory of the forward kernel, in words: per warp its 32 EPL logits (single precision), the lanes' sorted lists
// and a list of k keys per row; then [1 or warps][E] assignments and [warps][E] probability sums.
template <typename T, int EPL> __host__ __device__ __forceinline__ int kept_words() { return sizeof(T) == 4 ? 32 * EPL : 0; }
template <typename T, int EPL, int LANES> __host__ __device__ __forceinline__ int warp_words(int k)
{
    return kept_words<T, EPL>() + 32 * (EPL + 2) + (LANES == 32 ? 0 : (32 / LANES * k + 3) / 4 * 4);
}

// blockIdx.x = chunk of rows within the group, blockIdx.y = group; by_warp: a warp takes whole groups
template <typename T, int EPL, bool VEC, int LANES>
__global__ void __launch_bounds__(ROUTER_THREADS, EPL > 16 ? 1 : FORWARD_BLOCKS) router_forward_kernel(const __grid_constant__ RouterArgs a, bool by_warp)
{
    constexpr int VE = Lanes<T>::N, lanes = LANES, per_warp = 32 / LANES;
    extern __shared__ __align__(16) int32_t smem[];
    __shared__ int32_t valid_rows;
    __shared__ bool last;
    const int E = a.d.experts, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane & (lanes - 1), slot = lane / lanes;
    const int own_words = warp_words<T, EPL, LANES>(a.d.k);
    int32_t *own = smem + warp * own_words, *tables = smem + ROUTER_WARPS * own_words;
    float *kept = reinterpret_cast<float *>(own) + slot * lanes * EPL;
    uint32_t *sorted = reinterpret_cast<uint32_t *>(own + kept_words<T, EPL>()) + lane;
    uint32_t *list = reinterpret_cast<uint32_t *>(own + kept_words<T, EPL>() + 32 * (EPL + 2)) + slot * a.d.k;
    int32_t *hist = tables + (by_warp ? warp * E : 0);
    float *psum = reinterpret_cast<float *>(tables + E);
    sorted[EPL / 2 * 32] = sorted[(EPL + 1) * 32] = 0u;
    for (int e = threadIdx.x; e < E * (by_warp ? ROUTER_WARPS : 1); e += ROUTER_THREADS) tables[e] = 0;
    if (threadIdx.x == 0) valid_rows = 0;
    __syncthreads();
    if (by_warp) {
        for (int64_t g = int64_t(blockIdx.x) * ROUTER_WARPS + warp; g < a.groups; g += int64_t(gridDim.x) * ROUTER_WARPS) {
            const int64_t g0 = g * a.d.group_rows, g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
            Tally<EPL> t;
#pragma unroll
            for (int i = 0; i < EPL / 2; ++i) t.acc[i] = 0ull;
            t.valid = 0;
            route_chunk<T, EPL, VEC, LANES>(a, g0, g1, per_warp, sub, slot, sorted, list, kept, hist, t);
            float acc[EPL];
            int valid;
            fold_rows<EPL, LANES>(t, acc, valid);
            __syncwarp();
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                const int c = column<VEC, VE, LANES>(i, sub);
                if (lane < lanes && c < E) {
                    const int n = hist[c];
                    hist[c] = 0;
                    a.counts[g * E + c] = n;
                    a.prob_sum[g * E + c] = acc[i];
                    dot = fmaf(float(n), acc[i], dot);
                }
            }
            dot = warp_sum(dot);
            __syncwarp();
            if (lane == 0) {
                const float n = float(valid);
                a.valid[g] = valid;
                a.group_loss[g] = valid > 0 ? dot * float(E) / (float(a.d.k) * n * n) : 0.f;
            }
        }
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(a.tickets + a.groups, 1u) == gridDim.x - 1;
        __syncthreads();
        if (last) {
            __threadfence();
            join_loss(a);
            if (threadIdx.x == 0) a.tickets[a.groups] = 0u;
        }
        return;
    }
    for (int64_t g = blockIdx.y; g < a.groups; g += gridDim.y) {
        const int64_t g0 = g * a.d.group_rows;
        const int64_t g1 = g0 + a.d.group_rows < a.d.rows ? g0 + a.d.group_rows : a.d.rows;
        Tally<EPL> t;
#pragma unroll
        for (int i = 0; i < EPL / 2; ++i) t.acc[i] = 0ull;
        t.valid = 0;
        route_chunk<T, EPL, VEC, LANES>(a, g0 + (int64_t(blockIdx.x) * ROUTER_WARPS + warp) * per_warp, g1, int64_t(a.chunks) * ROUTER_WARPS * per_warp,
                                          sub, slot, sorted, list, kept, hist, t);
        // rows of a warp, then warps of the block
        float acc[EPL];
        int valid;
        fold_rows<EPL, LANES>(t, acc, valid);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const int c = column<VEC, VE, LANES>(i, sub);
            if (lane < lanes && c < E) psum[warp * E + c] = acc[i];
        }
        if (lane == 0 && valid) atomicAdd(&valid_rows, valid);
        __syncthreads();
        const int64_t place = g * a.chunks + blockIdx.x;
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
                __stcg(a.part + place * E + e, s);
                __stcg(a.part_counts + place * (E + 1) + e, n);
            }
        }
        const int rows_here = valid_rows;
        if (threadIdx.x == 0 && !alone) __stcg(a.part_counts + place * (E + 1) + E, rows_here);
        if (!alone) __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            valid_rows = 0;
            last = alone || atomicAdd(a.tickets + g, 1u) == uint32_t(a.chunks - 1);
        }
        __syncthreads();
        if (last) {                                // every chunk of the group has arrived
            if (alone) finish_group(a, g, dot, rows_here);
            else { __threadfence(); join_group(a, g, reinterpret_cast<float *>(smem)); }
            if (!alone && threadIdx.x == 0) a.tickets[g] = 0u;
            if (a.groups == 1) return;             // finish_group has written the loss
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) last = atomicAdd(a.tickets + a.groups, 1u) == uint32_t(a.groups - 1);
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

// A warp takes a run of consecutive rows, so that a group's factors a_e stay in registers from row to row.
template <typename T, int EPL, bool VEC, int LANES>
__global__ void __launch_bounds__(ROUTER_THREADS, EPL > 16 ? 1 : BACKWARD_BLOCKS) router_backward_kernel(const __grid_constant__ RouterArgs a, int run)
{
    constexpr int VE = Lanes<T>::N, lanes = LANES, per_warp = 32 / LANES;
    extern __shared__ float add[];                // [warps][rows of a warp][lanes * EPL]: what the weights' gradients add
    const int E = a.d.experts, k = a.d.k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane & (lanes - 1), slot = lane / lanes;
    float *mine = add + (warp * 32 + slot * lanes) * EPL;
#pragma unroll
    for (int i = 0; i < EPL; ++i) mine[i * lanes + sub] = 0.f;
    __syncwarp();                                 // one lane clears what others add to
    __shared__ float red[ROUTER_WARPS];
    float n = 0.f;                                // groups that take part in the loss
    if (a.some) n = *a.some;
    else {
        for (int64_t g = threadIdx.x; g < a.groups; g += ROUTER_THREADS) n += a.valid_in[g] > 0 ? 1.f : 0.f;
        n = warp_sum(n);
        if (lane == 0) red[warp] = n;
        __syncthreads();
        n = 0.f;
        for (int w = 0; w < ROUTER_WARPS; ++w) n += red[w];
    }
    const float pull = (a.dloss ? *a.dloss : 1.f) * a.d.coef * float(E) / (float(k) * fmaxf(n, 1.f));
    const bool renorm = a.d.flags & RUBICK_ROUTER_RENORM;
    const int64_t begin = (int64_t(blockIdx.x) * ROUTER_WARPS + warp) * run * per_warp;
    const int64_t end = begin + int64_t(run) * per_warp < a.d.rows ? begin + int64_t(run) * per_warp : a.d.rows;
    RawRow<T, EPL, VEC, LANES> next;
    int lead = -1, col = -1;                      // the row's first index; this lane's (the first of them if it has more)
    float w = 0.f, d = 0.f;
    const bool weights = a.dweight != nullptr;
    const auto fetch = [&](int64_t row) {
        const bool here = row < end;
        next.load(static_cast<const T *>(a.logits) + (here ? row : begin) * a.d.ld, sub, E);
        lead = col = -1;
        if (here) lead = a.index_in[row * k];
        if (here && sub < k && weights) {
            col = a.index_in[row * k + sub];
            w = a.weight_in[row * k + sub];
            d = a.dweight[row * k + sub];
        }
    };
    int64_t group = -1, group_end = -1;
    f2 f[EPL / 2];
#pragma unroll
    for (int i = 0; i < EPL / 2; ++i) f[i] = 0ull;
    if (begin < end) fetch(begin + slot);
    for (int64_t first = begin; first < end; first += per_warp) {
        const int64_t row = first + slot;
        const bool h = row < end, l = lead >= 0;
        const int c0 = col;
        const float w0 = w, d0 = d;
        f2 z[EPL / 2];
        next.get(z);
        if (first + per_warp < end) fetch(row + per_warp);
        if (h && row >= group_end) {
            group = row / a.d.group_rows;
            group_end = (group + 1) * a.d.group_rows;
            const float m = fmaxf(float(a.valid_in[group]), 1.f), scale = pull / (m * m);
#pragma unroll
            for (int i = 0; i < EPL; i += 2) {
                const int c = column<VEC, VE, LANES>(i, sub), c1 = column<VEC, VE, LANES>(i + 1, sub);
                f[i / 2] = pair(c < E ? scale * float(__ldg(a.counts_in + group * E + c)) : 0.f, c1 < E ? scale * float(__ldg(a.counts_in + group * E + c1)) : 0.f);
            }
        }
        // the chosen: w_j d_j, their sum over the row, and what goes to their columns
        float wd = 0.f;
        if (weights) {
            wd = l && c0 >= 0 ? w0 * d0 : 0.f;
            for (int j = sub + lanes; j < k; j += lanes)
                if (l && a.index_in[row * k + j] >= 0) wd = fmaf(a.weight_in[row * k + j], a.dweight[row * k + j], wd);
            wd = lanes_sum<LANES>(wd);
            const float mean = renorm ? wd : 0.f;
            if (l && c0 >= 0 && c0 < E) atomicAdd(mine + c0, w0 * (d0 - mean));
            for (int j = sub + lanes; j < k; j += lanes) {
                const int e = l ? a.index_in[row * k + j] : -1;
                if (e >= 0 && e < E) atomicAdd(mine + e, a.weight_in[row * k + j] * (a.dweight[row * k + j] - mean));
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < EPL / 2; ++i) top = fmaxf(top, fmaxf(lo(z[i]), hi(z[i])));
        top = lanes_max<LANES>(top);
        const f2 less_top = both(top > -INFINITY ? -top : 0.f);       // (a difference first, as in the forward pass)
        f2 sums = 0ull, dots = 0ull;
#pragma unroll
        for (int i = 0; i < EPL / 2; ++i) {
            const f2 x = mul2(add2(z[i], less_top), both(1.4426950408889634f));
            float e0, e1;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(lo(x)));
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(hi(x)));
            z[i] = pair(e0, e1);
            sums = add2(sums, z[i]);
            dots = fma2(f[i], z[i], dots);
        }
        const float total = lanes_sum<LANES>(lo(sums) + hi(sums));
        float dot = lanes_sum<LANES>(lo(dots) + hi(dots));
        const float inv = __fdividef(1.f, total);
        dot = fmaf(dot, inv, renorm ? 0.f : wd);
        if (weights) __syncwarp();
        T *out = static_cast<T *>(a.dlogits) + (h ? row : begin) * a.d.ld;
        const f2 inv2 = both(inv), less = both(-dot);
#pragma unroll
        for (int i = 0; i < EPL; i += VEC ? VE : 2) {
            const int c = column<VEC, VE, LANES>(i, sub);
            if constexpr (VEC) {
                f2 r[VE / 2];
#pragma unroll
                for (int e = 0; e < VE; e += 4) {
                    const ulonglong2 q = weights ? *reinterpret_cast<const ulonglong2 *>(mine + c + e) : make_ulonglong2(0ull, 0ull);
                    r[e / 2] = fma2(mul2(z[(i + e) / 2], inv2), add2(f[(i + e) / 2], less), q.x);
                    r[e / 2 + 1] = fma2(mul2(z[(i + e) / 2 + 1], inv2), add2(f[(i + e) / 2 + 1], less), q.y);
                }
                uint4 v = pack16<T>(r);
                if (!l) v = make_uint4(0u, 0u, 0u, 0u);
                if (h && c + VE <= E) st_stream(out + c, v);
                else if (h && c < E) {
                    float t[VE];
                    unpack16<T>(v, t);
#pragma unroll
                    for (int e = 0; e < VE; ++e) if (c + e < E) out[c + e] = from_f<T>(t[e]);
                }
            } else {
                const int c1 = column<VEC, VE, LANES>(i + 1, sub);
                const f2 q = weights ? pair(mine[c], mine[c1]) : 0ull;
                const f2 r = fma2(mul2(z[i / 2], inv2), add2(f[i / 2], less), q);
                if (h && c < E) out[c] = from_f<T>(l ? lo(r) : 0.f);
                if (h && c1 < E) out[c1] = from_f<T>(l ? hi(r) : 0.f);
            }
        }
        if (weights) {
            __syncwarp();
            if (l && c0 >= 0 && c0 < E) mine[c0] = 0.f;
            for (int j = sub + lanes; j < k; j += lanes) {
                const int e = l ? a.index_in[row * k + j] : -1;
                if (e >= 0 && e < E) mine[e] = 0.f;
            }
            __syncwarp();
        }
    }
}

// how many groups take part in the loss, where they are too many for every block to count them
__global__ void __launch_bounds__(1024) count_groups_kernel(const int32_t *valid, int64_t groups, float *some)
{
    __shared__ float red[32];
    float n = 0.f;
    for (int64_t g = threadIdx.x; g < groups; g += 1024) n += valid[g] > 0 ? 1.f : 0.f;
    n = warp_sum(n);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = n;
    __syncthreads();
    n = warp_sum(red[threadIdx.x & 31]);
    if (threadIdx.x == 0) *some = n;
}

struct RouterShape { int epl, lanes; bool vec; };

RouterShape router_shape(const RouterArgs &a)
{
    RouterShape s;
    const int es = a.d.dtype == RUBICK_F32 ? 4 : 2;
    s.vec = aligned16(a.logits) && (!a.dlogits || aligned16(a.dlogits)) && a.d.ld * es % 16 == 0;
    s.epl = a.d.experts > 512 ? 32 : a.d.experts > 8 ? 16 : 8;
    s.lanes = 1;
    while (s.lanes * s.epl < a.d.experts) s.lanes *= 2;
    return s;
}

// Groups so many that a warp each does: four to sixteen an SM, more the longer a warp would be at one (a warp against a
// block each, bf16: 600 groups of 4 x 64 9.7 against 15.4 us, 2,300 of them 11.3 against 37.9; 600 of 40 x 128 23.6
// against 21.5, 900 28.2 against 27.6, 1,800 29.7 against 44; 600 of 200 x 128 82 against 44, 2,300 104 against 124).
bool by_warp(const RouterArgs &a, int num_sms)
{
    const RouterShape s = router_shape(a);
    const int64_t passes = (a.d.group_rows * s.lanes + 31) / 32, an_sm = passes / 2;
    return a.groups >= int64_t(num_sms) * (an_sm < 4 ? 4 : an_sm > 16 ? 16 : an_sm);
}

template <typename T, bool BACK, int EPL, bool VEC, int LANES> cudaError_t launch_shape(const RouterArgs &a, int num_sms, cudaStream_t st)
{
    constexpr int per_warp = 32 / LANES;
    if constexpr (BACK) {
        const int smem = ROUTER_THREADS * EPL * int(sizeof(float));
        // a run of rows a warp, so long that all blocks are resident at once
        const int64_t slots = int64_t(num_sms) * BACKWARD_BLOCKS * ROUTER_WARPS * per_warp;
        const int run = int((a.d.rows + slots - 1) / slots);
        const int64_t per_block = int64_t(run) * ROUTER_WARPS * per_warp;
        if (a.some) {
            count_groups_kernel<<<1, 1024, 0, st>>>(a.valid_in, a.groups, const_cast<float *>(a.some));
            count_launch();
        }
        router_backward_kernel<T, EPL, VEC, LANES><<<unsigned((a.d.rows + per_block - 1) / per_block), ROUTER_THREADS, smem, st>>>(a, run);
    } else {
        const bool one = by_warp(a, num_sms);
        const int words = a.d.experts * (one ? ROUTER_WARPS : ROUTER_WARPS + 1) + ROUTER_WARPS * warp_words<T, EPL, LANES>(a.d.k);
        // 48 KB come without asking, the kernel's static variables (some hundred bytes) included
        if (words * 4 > 47 * 1024) {
            const cudaError_t e = cudaFuncSetAttribute(router_forward_kernel<T, EPL, VEC, LANES>, cudaFuncAttributeMaxDynamicSharedMemorySize, words * 4);
            if (e != cudaSuccess) return e;
        }
        const dim3 grid = one ? dim3(unsigned(num_sms) * FORWARD_BLOCKS) : dim3(a.chunks, unsigned(a.groups < 32768 ? a.groups : 32768));
        router_forward_kernel<T, EPL, VEC, LANES><<<grid, ROUTER_THREADS, words * 4, st>>>(a, one);
    }
    count_launch();
    return cudaGetLastError();
}

template <typename T, bool BACK, bool VEC> cudaError_t launch_vec(const RouterArgs &a, const RouterShape &s, int num_sms, cudaStream_t st)
{
    if (s.epl == 8) return launch_shape<T, BACK, 8, VEC, 1>(a, num_sms, st);
    if (s.epl == 32) return launch_shape<T, BACK, 32, VEC, 32>(a, num_sms, st);
    switch (s.lanes) {
    case 1: return launch_shape<T, BACK, 16, VEC, 1>(a, num_sms, st);
    case 2: return launch_shape<T, BACK, 16, VEC, 2>(a, num_sms, st);
    case 4: return launch_shape<T, BACK, 16, VEC, 4>(a, num_sms, st);
    case 8: return launch_shape<T, BACK, 16, VEC, 8>(a, num_sms, st);
    case 16: return launch_shape<T, BACK, 16, VEC, 16>(a, num_sms, st);
    default: return launch_shape<T, BACK, 16, VEC, 32>(a, num_sms, st);
    }
}
template <typename T, bool BACK> cudaError_t router_epl(const RouterArgs &a, int num_sms, cudaStream_t st)
{
    const RouterShape s = router_shape(a);
    return s.vec ? launch_vec<T, BACK, true>(a, s, num_sms, st) : launch_vec<T, BACK, false>(a, s, num_sms, st);
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

// blocks per group: as many as are resident at once, at least one pass of a block's warps each
int router_chunks(const RouterArgs &a, int num_sms)
{
    const RouterShape s = router_shape(a);
    const int64_t rows = a.d.group_rows < a.d.rows ? a.d.group_rows : a.d.rows;
    const int64_t most = (rows + ROUTER_WARPS * (32 / s.lanes) - 1) / (ROUTER_WARPS * (32 / s.lanes));
    const int64_t want = int64_t(num_sms) * FORWARD_BLOCKS / a.groups;
    // up to two passes by one block cost no more than a join (30 groups of 300 x 16 bf16: 9.7 against 11.8 us; 512 x 8: 7.7
    // both), four do (128 x 128: 11.8 against 9.7; 16 groups of 256 x 64: 15 against 11.8)
    if (most <= 2) return 1;
    return int(most < want ? most : want > 1 ? want : 1);
}

cudaError_t launch_router_forward(const RouterArgs &a, int num_sms, cudaStream_t st) { return router_type<false>(a, num_sms, st); }
cudaError_t launch_router_backward(const RouterArgs &a, int num_sms, cudaStream_t st) { return router_type<true>(a, num_sms, st); }

}  // namespace rubick
