// bsm_beam_select.cu -- the best continuations of every request's beams: the
// log-softmax of each beam's logits, its score added, and the `keep` largest of
// all of them in order, without the probabilities ever being written.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "bsm_beam.h"
#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kGroups = kBeamThreads / 4;       // groups of four neighbouring threads
constexpr int kGroupSize = 4 * kBeamLoads;      // pieces of 16 bytes of a group
constexpr int kWarps = kBeamThreads / 32;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

// The values of a 32-bit word of logits.
template <int kType> struct Word {
    static constexpr int kN = kType == BSM_F32 ? 1 : 2;         // values of a word
    static constexpr int kW = 4 * kN;                           // of a piece
    static constexpr int kEs = 4 / kN;
    static constexpr uint32_t kNone = kType == BSM_F32 ? 0xff800000u : kType == BSM_BF16 ? 0xff80ff80u : 0xfc00fc00u;
    static __device__ __forceinline__ void get(uint32_t w, float (&x)[kN])
    {
        if (kType == BSM_F32) {
            x[0] = __uint_as_float(w);
        } else if (kType == BSM_BF16) {
            x[0] = __uint_as_float(w << 16);
            x[kN - 1] = __uint_as_float(w & 0xffff0000u);
        } else {
            const __half2 h = *reinterpret_cast<const __half2 *>(&w);
            x[0] = __low2float(h);
            x[kN - 1] = __high2float(h);
        }
    }
    // (a NaN loses against any number)
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        if (kType == BSM_F32)
            return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        if (kType == BSM_BF16) {
            const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a),
                                             *reinterpret_cast<const __nv_bfloat162 *>(&b));
            return *reinterpret_cast<const uint32_t *>(&m);
        }
        const __half2 m = __hmax2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
};

// Logits [i, i + W) of a row of n that starts `off` bytes past a 16-byte boundary, -inf
// past its end: one aligned load, or two neighbouring ones shifted into place (the second
// is the next lane's first and comes from the first-level cache); at a row's ends value by
// value.  Which values a thread gets depends on their index alone, so equal rows give
// equal sums wherever they lie.
template <int kType> __device__ __forceinline__ uint4 load_piece(const unsigned char *row, int32_t i, int32_t n, uint32_t off)
{
    using T = Word<kType>;
    uint4 v = make_uint4(T::kNone, T::kNone, T::kNone, T::kNone);
    if (i >= n)
        return v;
    const unsigned char *p = row + static_cast<int64_t>(i) * T::kEs;
    if (off == 0 && i + T::kW <= n)
        return *reinterpret_cast<const uint4 *>(p);
    if (off != 0 && i > 0 && i + 2 * T::kW <= n) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p - off), b = *reinterpret_cast<const uint4 *>(p - off + 16);
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (off & 8) {
#pragma unroll
            for (int k = 0; k < 6; ++k)
                w[k] = w[k + 2];
        }
        if (off & 4) {
#pragma unroll
            for (int k = 0; k < 5; ++k)
                w[k] = w[k + 1];
        }
        const uint32_t bits = (off & 3) * 8;
        return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                          __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
    }
    uint32_t w[4] = {T::kNone, T::kNone, T::kNone, T::kNone};
#pragma unroll
    for (int k = 0; k < T::kW; ++k) {
        if (i + k >= n)
            continue;
        if (T::kN == 1) {
            w[k % 4] = reinterpret_cast<const uint32_t *>(p)[k];
        } else {
            const uint32_t h = reinterpret_cast<const uint16_t *>(p)[k];
            w[k / 2 % 4] = k % 2 ? (w[k / 2 % 4] & 0xffffu) | h << 16 : (w[k / 2 % 4] & 0xffff0000u) | h;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct PartSmem {
    float group[kGroups];               // the largest value of each group
    int32_t first[kGroups];             // where a group's value ties with the bound: its lowest token
    float warp_top[kWarps], warp_sum[kWarps], warp_bound[kGroups / 32];
    int32_t above, count, last;
};

// One part of a row: its values stay in registers while the largest is found, the sum of
// exponentials taken and the list made.  The keep-th largest of 128 group maxima is a
// bound that at least `keep` values reach, and values above it can lie in fewer than
// `keep` groups, so what reaches it fits a list of keep x 128 values whatever the row
// holds; where groups tie at the bound only the first of them, by token, count.  The list is then
// ordered by counting for each entry how many are better.
template <int kType> __global__ void __launch_bounds__(kBeamThreads, 2) select_rows(const BeamSelectArgs a)
{
    using T = Word<kType>;
    constexpr int W = T::kW;
    __shared__ PartSmem s;
    extern __shared__ __align__(16) unsigned char raw_list[];
    BeamEntry *list = reinterpret_cast<BeamEntry *>(raw_list);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    const int32_t row = static_cast<int32_t>(blockIdx.x / static_cast<uint32_t>(a.parts));
    const int32_t part = static_cast<int32_t>(blockIdx.x - static_cast<uint32_t>(row) * a.parts);
    const float score = a.scores[row];
    if (!(fabsf(score) < __int_as_float(0x7f800000)) || (a.ended && a.ended[row]))
        return;                         // no candidate, or one that needs no logits
    const int32_t request = row / a.beams, beam = row - request * a.beams;
    const unsigned char *base = a.logits + request * a.stride_request + beam * a.stride_beam;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) & 15u;
    const int32_t lo = part * a.part, hi = min(lo + a.part, a.vocab);
    uint4 v[kBeamLoads];
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j) {
        const int32_t i = lo + (j * kBeamThreads + tid) * W;
        // (parts are whole pieces: only the row's end cuts one)
        v[j] = i < hi ? load_piece<kType>(base, i, a.vocab, off) : make_uint4(T::kNone, T::kNone, T::kNone, T::kNone);
    }
    uint32_t most = T::kNone;
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j)
        most = T::larger(most, T::larger(T::larger(v[j].x, v[j].y), T::larger(v[j].z, v[j].w)));
    float ends[T::kN];
    T::get(most, ends);
    const float mine = fmaxf(fmaxf(ends[0], ends[T::kN - 1]), neg_inf());      // (not NaN)
    float best = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
    best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 2));
    if (lane % 4 == 0)
        s.group[tid / 4] = best;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1)
        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0)
        s.warp_top[warp] = best;
    if (tid == 0) {
        s.above = 0;
        s.count = 0;
        s.last = INT_MAX;
    }
    __syncthreads();
    // the bound: the smallest of the group maxima that fewer than `keep` exceed
    if (tid < kGroups) {
        const float g = s.group[tid];
        int over = 0;
#pragma unroll 8
        for (int k = 0; k < kGroups / 4; ++k) {
            const float4 o = reinterpret_cast<const float4 *>(s.group)[k];
            over += (o.x > g) + (o.y > g) + (o.z > g) + (o.w > g);
        }
        float b = over < a.keep ? g : __int_as_float(0x7f800000);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
            b = fminf(b, __shfl_xor_sync(0xffffffffu, b, o));
        if (lane == 0)
            s.warp_bound[warp] = b;
    }
    float top = s.warp_top[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w)
        top = fmaxf(top, s.warp_top[w]);
    // exp(x - top) = 2^((x - top) log2(e)); an empty part sums up to 0
    const float from = top == neg_inf() ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j) {
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x[T::kN];
            T::get(w[k], x);
#pragma unroll
            for (int e = 0; e < T::kN; ++e)
                sum += pg_exp2((x[e] - from) * 1.4426950408889634f);
        }
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0)
        s.warp_sum[warp] = sum;
    __syncthreads();
    float bound = s.warp_bound[0];
#pragma unroll
    for (int w = 1; w < kGroups / 32; ++w)
        bound = fminf(bound, s.warp_bound[w]);
    // groups that reach the bound: where more than `keep` do, the last ones tie there
    const float group = s.group[tid / 4];
    int32_t last = INT_MAX;
    const int reach = __syncthreads_count(lane % 4 == 0 && group >= bound);
    if (bound > neg_inf() && reach > a.keep) {
        const int above = __syncthreads_count(lane % 4 == 0 && group > bound);
        int32_t first = INT_MAX;
        if (mine == bound) {
#pragma unroll
            for (int j = kBeamLoads - 1; j >= 0; --j) {
                const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int k = 3; k >= 0; --k) {
                    float x[T::kN];
                    T::get(w[k], x);
#pragma unroll
                    for (int e = T::kN - 1; e >= 0; --e)
                        if (x[e] == bound)
                            first = lo + (j * kBeamThreads + tid) * W + k * T::kN + e;
                }
            }
        }
        first = min(first, __shfl_xor_sync(0xffffffffu, first, 1));
        first = min(first, __shfl_xor_sync(0xffffffffu, first, 2));
        if (lane % 4 == 0)
            s.first[tid / 4] = group == bound ? first : INT_MAX;
        __syncthreads();
        if (tid < kGroups) {
            const int32_t f = s.first[tid];
            int before = 0;
            for (int k = 0; k < kGroups; ++k)
                before += s.first[k] < f;
            // of the tied groups the last one that is still needed
            if (f != INT_MAX && before == a.keep - above - 1)
                s.last = f;
        }
        __syncthreads();
        last = s.last;
    }
    if (mine >= bound && mine > neg_inf()) {
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j) {
            const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x[T::kN];
                T::get(w[k], x);
#pragma unroll
                for (int e = 0; e < T::kN; ++e) {
                    const int32_t token = lo + (j * kBeamThreads + tid) * W + k * T::kN + e;
                    if (x[e] >= bound && x[e] > neg_inf() && (x[e] > bound || token <= last))
                        list[atomicAdd(&s.count, 1)] = BeamEntry{x[e], token};
                }
            }
        }
    }
    __syncthreads();
    const int count = s.count;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * a.keep;
    for (int i = tid; i < count; i += kBeamThreads) {
        const BeamEntry e = list[i];
        int better = 0;
        for (int k = 0; k < count; ++k) {
            const BeamEntry o = list[k];
            better += o.x > e.x || (o.x == e.x && o.token < e.token);
        }
        if (better < a.keep)
            a.entries[at + better] = e;
    }
    if (tid == 0) {
        double all = 0.0;
        for (int w = 0; w < kWarps; ++w)
            all += s.warp_sum[w];
        a.meta[blockIdx.x] = BeamPart{all, top, min(count, a.keep)};
    }
}

// Two fp32 numbers whose sum stands for a value of 48 bits.
struct Pair {
    float hi, lo;
};
__device__ __forceinline__ Pair two_sum(float a, float b)
{
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return Pair{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Pair add(const Pair &x, const Pair &y)
{
    const Pair s = two_sum(x.hi, y.hi), t = two_sum(x.lo, y.lo);
    const Pair u = two_sum(s.hi, __fadd_rn(s.lo, t.hi));
    return two_sum(u.hi, __fadd_rn(u.lo, t.lo));
}

// A candidate: its value as a whole number of the same order, and its place among the
// request's (beam * vocab + token), the lower one first where values are equal.
struct Cand {
    uint64_t key;                       // 0: none
    int32_t at;
};
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);               // (-0 becomes 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float disordered(uint32_t u)
{
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ bool better(const Cand &a, const Cand &b) { return a.key > b.key || (a.key == b.key && a.at < b.at); }
__device__ __forceinline__ Cand other(const Cand &c, int mask)
{
    Cand o;
    o.key = __shfl_xor_sync(0xffffffffu, c.key, mask);
    o.at = __shfl_xor_sync(0xffffffffu, c.at, mask);
    return o;
}

// A warp's sorted list of 32 R candidates (lane l holds ranks l, l + 32), best first.
template <int R> struct Best {
    Cand c[R];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int r = 0; r < R; ++r)
            c[r] = Cand{0, INT_MAX};
    }
    // The best of this list and another sorted one: rank i against the other's rank from the
    // end leaves the best half as a sequence that rises once and falls once, which log2
    // exchanges sort.
    __device__ __forceinline__ void merge(const Best &o, int lane)
    {
        Cand m[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Cand x = other(o.c[R - 1 - r], 31);
            m[r] = better(c[r], x) ? c[r] : x;
        }
        if (R == 2 && better(m[R - 1], m[0])) {
            const Cand x = m[0];
            m[0] = m[R - 1];
            m[R - 1] = x;
        }
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const Cand x = other(m[r], k);
                const bool want = (lane & k) == 0;
                m[r] = better(m[r], x) == want ? m[r] : x;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            c[r] = m[r];
    }
};

struct JoinSmem {
    float top[kBeamMost];
    double sum[kBeamMost];
    Pair shift[kBeamMost];              // score - log(sum): what a row adds to x - top
    int32_t kind[kBeamMost];            // 0: no candidate, 1: one (an ended beam), 2: its parts' lists
    Cand best[kWarps][kBeamMost];
};

// The lists of all parts of all beams of a request, in order by value: score + (x - top) -
// log(sum), held in two fp32 numbers.  Every warp merges its share of the lists,
// skipping those whose first entry does not get in, then pairs of warps join.
template <int R> __global__ void __launch_bounds__(kBeamThreads) select_join(const BeamSelectArgs a)
{
    __shared__ JoinSmem s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t request = blockIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    for (int b = warp; b < a.beams; b += kWarps) {
        const int64_t row = static_cast<int64_t>(request) * a.beams + b;
        const float score = a.scores[row];
        int32_t kind = 2;
        if (!(fabsf(score) < __int_as_float(0x7f800000)))
            kind = 0;
        else if (a.ended && a.ended[row])
            kind = 1;
        float top = neg_inf();
        double sum = 0.0;
        if (kind == 2) {
            float m[kBeamMostParts / 32];
            double z[kBeamMostParts / 32];
#pragma unroll
            for (int i = 0; i < kBeamMostParts / 32; ++i) {
                const int p = lane + 32 * i;
                m[i] = neg_inf();
                z[i] = 0.0;
                if (p < a.parts) {
                    const BeamPart &part = a.meta[row * a.parts + p];
                    m[i] = part.top;
                    z[i] = part.sum;
                }
                top = fmaxf(top, m[i]);
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
            for (int i = 0; i < kBeamMostParts / 32; ++i)
                if (z[i] != 0.0)        // (an empty part: -inf - -inf)
                    sum += z[i] * expf(m[i] - top);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1)
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        if (lane == 0) {
            s.top[b] = top;
            s.sum[b] = sum;
            s.kind[b] = kind;
        }
    }
    __syncthreads();
    if (tid < a.beams) {
        const float score = a.scores[static_cast<int64_t>(request) * a.beams + tid];
        double shift = score;
        if (s.kind[tid] == 2) {
            // NaN or +inf among the logits, or none above -inf: the row's softmax is NaN
            if (!(s.sum[tid] > 0.0))
                s.kind[tid] = 0;
            shift -= log(s.sum[tid]);
        }
        const float hi = static_cast<float>(shift);
        s.shift[tid] = Pair{hi, static_cast<float>(shift - hi)};
    }
    __syncthreads();
    Best<R> best;
    best.clear();
    const int lists = a.beams * a.parts;
    for (int l = warp; l < lists; l += kWarps) {
        const int b = l / a.parts, p = l - b * a.parts;
        const int kind = s.kind[b];
        if (kind == 0 || (kind == 1 && p > 0))
            continue;
        Best<R> next;
        next.clear();
        if (kind == 1) {
            if (lane == 0)
                next.c[0] = Cand{static_cast<uint64_t>(ordered(s.shift[b].hi)) << 32 | ordered(s.shift[b].lo),
                                 b * a.vocab + a.end_token};
        } else {
            const int64_t at = (static_cast<int64_t>(request) * a.beams + b) * a.parts + p;
            const int count = a.meta[at].count;
            const Pair shift = s.shift[b];
            const float top = s.top[b];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = lane + 32 * r;
                if (i < count) {
                    const BeamEntry e = a.entries[at * a.keep + i];
                    const Pair x = add(two_sum(e.x, -top), shift);
                    if (x.hi > neg_inf())           // (not beyond fp32's range)
                        next.c[r] = Cand{static_cast<uint64_t>(ordered(x.hi)) << 32 | ordered(x.lo), b * a.vocab + e.token};
                }
            }
        }
        // a list whose first does not beat the last kept one has nothing to add
        const int worst = a.keep - 1;
        Cand first, least = best.c[R - 1];         // (keep is above 32 where R is 2)
        first.key = __shfl_sync(0xffffffffu, next.c[0].key, 0);
        first.at = __shfl_sync(0xffffffffu, next.c[0].at, 0);
        least.key = __shfl_sync(0xffffffffu, least.key, worst % 32);
        least.at = __shfl_sync(0xffffffffu, least.at, worst % 32);
        if (better(first, least))
            best.merge(next, lane);
    }
    for (int half = kWarps / 2; half > 0; half >>= 1) {
        if (warp >= half && warp < 2 * half) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                s.best[warp][lane + 32 * r] = best.c[r];
        }
        __syncthreads();
        if (warp < half) {
            Best<R> next;
#pragma unroll
            for (int r = 0; r < R; ++r)
                next.c[r] = s.best[warp + half][lane + 32 * r];
            best.merge(next, lane);
        }
    }
    if (warp == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = lane + 32 * r;
            if (i < a.keep) {
                const int64_t to = static_cast<int64_t>(request) * a.keep + i;
                const Cand c = best.c[r];
                const bool there = c.key != 0;
                const int32_t parent = there ? c.at / a.vocab : -1;
                // (the larger of the two numbers is the value rounded to fp32)
                a.out_scores[to] = there ? disordered(static_cast<uint32_t>(c.key >> 32)) : neg_inf();
                a.parents[to] = parent;
                a.tokens[to] = there ? c.at - parent * a.vocab : -1;
            }
        }
    }
}

}  // namespace

void beam_parts(int64_t rows, int32_t vocab, int es, int n_sm, int32_t *parts, int32_t *part)
{
    const int64_t piece = 16 / es, most = kBeamThreads * kBeamLoads * piece, least = kBeamThreads * piece;
    auto up = [](int64_t x, int64_t d) { return (x + d - 1) / d; };
    // as many as there are SMs, of one piece a thread at least
    int64_t n = up(n_sm, rows < 1 ? 1 : rows);
    n = n < up(vocab, least) ? n : up(vocab, least);
    n = n > up(vocab, most) ? n : up(vocab, most);
    n = n < kBeamMostParts ? n : kBeamMostParts;
    const int64_t each = up(up(vocab, n), piece) * piece;
    *part = static_cast<int32_t>(each);
    *parts = static_cast<int32_t>(up(vocab, each));
}

int launch_beam_select(const BeamSelectArgs &a, int dtype, void *stream)
{
    const unsigned rows = static_cast<unsigned>(a.n) * a.beams;
    const size_t list = static_cast<size_t>(a.keep) * kGroupSize * (dtype == BSM_F32 ? 4 : 8) * sizeof(BeamEntry);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 grid(rows * a.parts);
    int e = dtype == BSM_F32    ? launch_early(select_rows<BSM_F32>, grid, kBeamThreads, list, st, a)
            : dtype == BSM_BF16 ? launch_early(select_rows<BSM_BF16>, grid, kBeamThreads, list, st, a)
                                : launch_early(select_rows<BSM_F16>, grid, kBeamThreads, list, st, a);
    if (e)
        return e;
    return a.keep <= 32 ? launch_early(select_join<1>, dim3(a.n), kBeamThreads, 0, st, a)
                        : launch_early(select_join<2>, dim3(a.n), kBeamThreads, 0, st, a);
}

int beam_set_smem_limit()
{
    int e = 0;
    auto set = [&](const void *f, int piece) {
        if (!e)
            e = static_cast<int>(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                      static_cast<int>(kBeamMost * kGroupSize * piece * sizeof(BeamEntry))));
    };
    set(reinterpret_cast<const void *>(&select_rows<BSM_F32>), 4);
    set(reinterpret_cast<const void *>(&select_rows<BSM_BF16>), 8);
    set(reinterpret_cast<const void *>(&select_rows<BSM_F16>), 8);
    return e;
}

}  // namespace bsm
