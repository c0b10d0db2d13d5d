// bsm_beam_select.cu -- the best continuations of every request's beams: the
// log-softmax of each beam's logits, its score added, and the `keep` largest of
// all of them in order, without the probabilities ever being written.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "bsm_beam.h"
#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kGroups = 128;                    // groups of neighbouring threads, more than are ever kept
constexpr int kGroupLanes = kBeamThreads / kGroups;
constexpr int kWarps = kBeamThreads / 32;
constexpr int kRowCtas = 3;                      // of select_rows on an SM

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

// The 16 bytes that start `off` bytes into a.
__device__ __forceinline__ uint4 shifted(const uint4 &a, const uint4 &b, uint32_t off)
{
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

// A thread's pieces of the block that starts at `first`, -inf from hi on (the end of the part, or
// of the row of n).  A row may start `off` bytes past a 16-byte boundary: its pieces are put
// together from two neighbouring aligned ones (the second is the next lane's first and comes
// from the first-level cache), at the row's ends from single values.  Which values a
// thread gets depends on their index alone, so equal rows give equal sums wherever they lie.
template <int kType>
__device__ __forceinline__ void load_block(uint4 (&v)[kBeamLoads], const unsigned char *row, uint32_t off, int32_t first,
                                           int32_t hi, int32_t n)
{
    using T = Word<kType>;
    constexpr int W = T::kW, kStep = kBeamThreads * W;          // values between a thread's pieces
    const int32_t mine = first + static_cast<int32_t>(threadIdx.x) * W;
    const unsigned char *p = row + static_cast<int64_t>(mine) * T::kEs - off;
    if (first + kBeamLoads * kStep <= hi && (off == 0 || (first > 0 && first + kBeamLoads * kStep + W <= n))) {
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j)
            v[j] = *reinterpret_cast<const uint4 *>(p + j * kStep * T::kEs);
        if (off != 0) {
#pragma unroll
            for (int j = 0; j < kBeamLoads; ++j)
                v[j] = shifted(v[j], *reinterpret_cast<const uint4 *>(p + j * kStep * T::kEs + 16), off);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j) {
        const int32_t i = mine + j * kStep;
        const unsigned char *q = p + j * kStep * T::kEs;
        v[j] = make_uint4(T::kNone, T::kNone, T::kNone, T::kNone);
        if (i >= hi)
            continue;
        if (off == 0 ? i + W <= n : i > 0 && i + 2 * W <= n) {
            v[j] = *reinterpret_cast<const uint4 *>(q);
            if (off != 0)
                v[j] = shifted(v[j], *reinterpret_cast<const uint4 *>(q + 16), off);
            continue;
        }
        uint32_t w[4] = {T::kNone, T::kNone, T::kNone, T::kNone};
#pragma unroll
        for (int k = 0; k < W; ++k) {
            if (i + k >= n)
                continue;
            if (T::kN == 1) {
                w[k % 4] = reinterpret_cast<const uint32_t *>(q + off)[k];
            } else {
                const uint32_t h = reinterpret_cast<const uint16_t *>(q + off)[k];
                w[k / 2 % 4] = k % 2 ? (w[k / 2 % 4] & 0xffffu) | h << 16 : (w[k / 2 % 4] & 0xffff0000u) | h;
            }
        }
        v[j] = make_uint4(w[0], w[1], w[2], w[3]);
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

struct PartSmem {
    float group[kGroups];               // the largest value of each group
    int32_t first[kGroups];             // where a group's value ties with the bound: its lowest token
    float warp_top[kWarps], warp_sum[kWarps], warp_bound[kWarps];
    uint4 hit[kWarps][kBeamLoads];      // the pieces of a lane that has something for the list
    int32_t count, last;
};

// Two fp32 numbers at once.
__device__ __forceinline__ uint64_t pack2(float a, float b)
{
    return static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float low2(uint64_t a) { return __uint_as_float(static_cast<uint32_t>(a)); }
__device__ __forceinline__ float high2(uint64_t a) { return __uint_as_float(static_cast<uint32_t>(a >> 32)); }

// Calls f(value, token) for every value of a thread's pieces of a block that starts at `first`.
template <int kType, typename F> __device__ __forceinline__ void each_value(const uint4 (&v)[kBeamLoads], int32_t first, F &&f)
{
    using T = Word<kType>;
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j) {
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        const int32_t token = first + (j * kBeamThreads + static_cast<int>(threadIdx.x)) * T::kW;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x[T::kN];
            T::get(w[k], x);
#pragma unroll
            for (int e = 0; e < T::kN; ++e)
                f(x[e], token + k * T::kN + e);
        }
    }
}

// The list's best `keep` in order to `to`: four threads count for each entry how many are better.
__device__ __forceinline__ void rank_list(const BeamEntry *list, int count, int keep, BeamEntry *to)
{
    const int lane = threadIdx.x & 31, quarter = lane & 3;
    for (int i0 = (threadIdx.x >> 5) * 8; i0 < count; i0 += kWarps * 8) {
        const int i = i0 + lane / 4;
        const BeamEntry e = list[i < count ? i : 0];
        int better = 0;
        for (int k = quarter; k < count; k += 4) {
            const BeamEntry o = list[k];
            better += o.x > e.x || (o.x == e.x && o.token < e.token);
        }
        better += __shfl_xor_sync(0xffffffffu, better, 1);
        better += __shfl_xor_sync(0xffffffffu, better, 2);
        if (quarter == 0 && i < count && better < keep)
            to[better] = e;
    }
}

// A block's bound: the smallest of its group maxima that fewer than `keep` exceed, so that `keep`
// of its values reach it (-inf where fewer than `keep` groups have any).  Where more groups than that
// reach it some tie there: of values equal to the bound only those up to token *last are
// needed then, and those that count lie in `keep` groups at most.
template <int kType>
__device__ __forceinline__ float block_bound(PartSmem &s, const uint4 (&v)[kBeamLoads], float mine, int32_t first, int keep, int32_t *last)
{
    const int tid = threadIdx.x, lane = tid & 31;
    float best = mine;
#pragma unroll
    for (int o = 1; o < kGroupLanes; o <<= 1)
        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
    const bool speaks = tid % kGroupLanes == 0;
    if (speaks)
        s.group[tid / kGroupLanes] = best;
    __syncthreads();
    int over = 0;                       // (a group's threads share the count)
#pragma unroll
    for (int k = 0; k < kGroups / 4 / kGroupLanes; ++k) {
        const float4 o = reinterpret_cast<const float4 *>(s.group)[k * kGroupLanes + tid % kGroupLanes];
        over += (o.x > best) + (o.y > best) + (o.z > best) + (o.w > best);
    }
#pragma unroll
    for (int o = 1; o < kGroupLanes; o <<= 1)
        over += __shfl_xor_sync(0xffffffffu, over, o);
    float bound = over < keep ? best : __int_as_float(0x7f800000);
#pragma unroll
    for (int o = kGroupLanes; o < 32; o <<= 1)
        bound = fminf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
    if (lane == 0)
        s.warp_bound[tid >> 5] = bound;
    __syncthreads();
    bound = s.warp_bound[lane % kWarps];
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1)
        bound = fminf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
    *last = bound == neg_inf() ? -1 : INT_MAX;
    if (bound == neg_inf() || __syncthreads_count(speaks && best >= bound) <= keep)
        return bound;
    const int above = __syncthreads_count(speaks && best > bound);
    int32_t at = INT_MAX;
    if (mine == bound)
        each_value<kType>(v, first, [&](float x, int32_t token) {
            if (x == bound)
                at = min(at, token);
        });
#pragma unroll
    for (int o = 1; o < kGroupLanes; o <<= 1)
        at = min(at, __shfl_xor_sync(0xffffffffu, at, o));
    if (speaks)
        s.first[tid / kGroupLanes] = best == bound ? at : INT_MAX;
    __syncthreads();
    if (tid < kGroups) {
        const int32_t f = s.first[tid];
        int before = 0;
        for (int k = 0; k < kGroups; ++k)
            before += s.first[k] < f;
        // of the tied groups the last one that is still needed
        if (f != INT_MAX && before == keep - above - 1)
            s.last = f;
    }
    __syncthreads();
    *last = s.last;
    return bound;
}

// Values above the bound, and equal ones up to token `last`, to the list, in any order.  Few
// lanes have one: each such lane's values are looked at by the whole warp.  Entries past the
// list's end are counted only.
template <int kType>
__device__ __forceinline__ void to_list(PartSmem &s, BeamEntry *list, int room, const uint4 (&v)[kBeamLoads], float mine, int32_t first,
                                        float bound, int32_t last)
{
    using T = Word<kType>;
    constexpr int kMine = kBeamLoads * T::kW;
    static_assert(kMine <= 32, "a lane each");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t has = __ballot_sync(0xffffffffu, (last < 0 ? mine > bound : mine >= bound) && mine > neg_inf());
    while (has) {
        const int l = __ffs(static_cast<int>(has)) - 1;
        has &= has - 1;
        if (lane == l) {
#pragma unroll
            for (int j = 0; j < kBeamLoads; ++j)
                s.hit[warp][j] = v[j];
        }
        __syncwarp();
        if (lane < kMine) {
            float x[T::kN];
            T::get(reinterpret_cast<const uint32_t *>(s.hit[warp])[lane / T::kN], x);
            const float one = T::kN == 2 && lane % 2 ? x[T::kN - 1] : x[0];
            const int32_t token = first + (lane / T::kW * kBeamThreads + warp * 32 + l) * T::kW + lane % T::kW;
            if (one > bound || (one == bound && token <= last)) {
                const int i = atomicAdd(&s.count, 1);
                if (i < room)
                    list[i] = BeamEntry{one, token};
            }
        }
        __syncwarp();
    }
}

template <int kType> __device__ __forceinline__ float largest(const uint4 (&v)[kBeamLoads])
{
    using T = Word<kType>;
    uint32_t most = T::kNone;
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j)
        most = T::larger(most, T::larger(T::larger(v[j].x, v[j].y), T::larger(v[j].z, v[j].w)));
    float ends[T::kN];
    T::get(most, ends);
    return fmaxf(fmaxf(ends[0], ends[T::kN - 1]), neg_inf());           // (not NaN)
}

// The list once more, where it overflowed: every block with a bound of its own, what is listed cut
// to the best `keep` before it.  Rows that rise along the part and the like come here.
template <int kType>
__device__ __noinline__ int list_again(PartSmem &s, BeamEntry *list, int room, int keep, const unsigned char *row, uint32_t off,
                                       int32_t lo, int32_t hi, int32_t n)
{
    const int tid = threadIdx.x;
    int count = 0;
    float bound = neg_inf();
    for (int32_t first = lo; first < hi; first += kBeamThreads * kBeamLoads * Word<kType>::kW) {
        uint4 v[kBeamLoads];
        load_block<kType>(v, row, off, first, hi, n);
        const float mine = largest<kType>(v);
        if (tid == 0)
            s.count = count;
        int32_t last;
        const float b = block_bound<kType>(s, v, mine, first, keep, &last);     // (its barriers order the count)
        if (b > bound)
            bound = b;
        else
            last = -1;
        to_list<kType>(s, list, room, v, mine, first, bound, last);
        __syncthreads();
        count = s.count;
        rank_list(list, count, keep, list + room);
        __syncthreads();
        count = min(count, keep);
        if (tid < count)
            list[tid] = list[room + tid];
        if (count == keep)
            bound = list[room + keep - 1].x;
        __syncthreads();
    }
    return count;
}

// One part of a row, a block of values (64 bytes a thread) after the other.  Each thread keeps a
// maximum and a sum of exponentials of its own.  What can be among the part's best goes to
// a list: the first block's values that reach its bound, and later ones that exceed it, about `keep`
// a block where the row is in no order; the warps go their own ways from the second block on.
template <int kType> __global__ void __launch_bounds__(kBeamThreads, kRowCtas) select_rows(const BeamSelectArgs a)
{
    using T = Word<kType>;
    constexpr int kBlock = kBeamThreads * kBeamLoads * T::kW;           // values of a block
    __shared__ PartSmem s;
    extern __shared__ __align__(16) unsigned char raw_list[];
    BeamEntry *list = reinterpret_cast<BeamEntry *>(raw_list);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    const uint32_t row = blockIdx.x / static_cast<uint32_t>(a.parts);
    const int32_t part = static_cast<int32_t>(blockIdx.x - row * a.parts);
    const float score = a.scores[row];
    if (!(fabsf(score) < __int_as_float(0x7f800000)) || (a.ended && a.ended[row]))
        return;                         // no candidate, or one that needs no logits
    const uint32_t request = row / static_cast<uint32_t>(a.beams), beam = row - request * a.beams;
    const unsigned char *base = a.logits + request * a.stride_request + beam * a.stride_beam;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) & 15u;
    const int32_t lo = part * a.part, hi = min(lo + a.part, a.vocab);
    if (tid == 0)
        s.count = 0;
    float top = neg_inf(), sum = 0.0f, bound = neg_inf();               // of this thread; of the part
    for (int32_t first = lo; first < hi; first += kBlock) {
        uint4 v[kBeamLoads];
        load_block<kType>(v, base, off, first, hi, a.vocab);
        const float mine = largest<kType>(v);
        int32_t last = -1;
        if (first == lo)
            bound = block_bound<kType>(s, v, mine, first, a.keep, &last);
        to_list<kType>(s, list, a.list, v, mine, first, bound, last);
        // exp(x - top) = 2^((x - top) log2(e)); nothing but -inf sums up to 0
        const float was = top;
        top = fmaxf(top, mine);
        const float from = top == neg_inf() ? 0.0f : top;
        const uint64_t from2 = pack2(-from, -from), log2e = pack2(1.4426950408889634f, 1.4426950408889634f);
        uint64_t sum2 = 0;
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j) {
            const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int k = 0; k < 4; k += 2 / T::kN) {
                float x[T::kN], y[T::kN];
                T::get(w[k], x);
                T::get(w[(k + 1) % 4], y);
                const uint64_t t = mul2(add2(pack2(x[0], T::kN == 2 ? x[T::kN - 1] : y[0]), from2), log2e);
                sum2 = add2(sum2, pack2(pg_exp2(low2(t)), pg_exp2(high2(t))));
            }
        }
        sum = __fmaf_rn(sum, pg_exp2((was - from) * 1.4426950408889634f), low2(sum2) + high2(sum2));
    }
    // the part's maximum and sum
    float all = top;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    if (lane == 0)
        s.warp_top[warp] = all;
    __syncthreads();
    int count = s.count;
    all = s.warp_top[lane % kWarps];
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1)
        all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    sum *= all == neg_inf() ? 1.0f : pg_exp2((top - all) * 1.4426950408889634f);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0)
        s.warp_sum[warp] = sum;
    __syncthreads();
    if (count > a.list)
        count = list_again<kType>(s, list, a.list, a.keep, base, off, lo, hi, a.vocab);
    rank_list(list, count, a.keep, a.entries + static_cast<int64_t>(blockIdx.x) * a.keep);
    if (warp == 0) {
        Pair z{lane < kWarps ? s.warp_sum[lane] : 0.0f, 0.0f};
#pragma unroll
        for (int o = 1; o < kWarps; o <<= 1)
            z = add(z, Pair{__shfl_xor_sync(0xffffffffu, z.hi, o), __shfl_xor_sync(0xffffffffu, z.lo, o)});
        if (lane == 0)
            a.meta[blockIdx.x] = BeamPart{z.hi, z.lo, all, min(count, a.keep)};
    }
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

// log(x) of x > 0 given as a pair, within about 2^-30: x = 2^e f, f in [3/4, 3/2), and with z = (f - 1) / (f + 1)
// log(f) = 2 (z + z^3 / 3 + z^5 / 5 + ..); only the first term needs more than fp32.
__device__ __forceinline__ Pair log_of(const Pair &x)
{
    const uint32_t bits = __float_as_uint(x.hi);
    const int e = static_cast<int>(bits - 0x3f400000u) >> 23;           // (3/4 in fp32)
    const float scale = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    const float f = x.hi * scale, g = x.lo * scale;                     // exact
    const Pair den = two_sum(f, 1.0f);
    const float num = f - 1.0f;                                         // exact
    const float z = __fdividef(num, den.hi);
    // what z misses, the lower number of x with it: d log(f) = g / f
    const float rest = __fmaf_rn(-z, den.hi, num) - z * den.lo;
    const float low = __fdividef(2.0f * rest, den.hi) + __fdividef(g, f);
    const float q = z * z;
    const float tail = z * q * (2.0f / 3 + q * (2.0f / 5 + q * (2.0f / 7 + q * (2.0f / 9 + q * (2.0f / 11)))));
    // e log(2): the first part of log(2) has 12 bits, so its product is exact
    const Pair whole = two_sum(e * 0.693115234375f, 2.0f * z);
    return two_sum(whole.hi, whole.lo + (tail + low + e * 3.194618498e-5f));
}

struct JoinSmem {
    float top[kBeamMost];
    Pair sum[kBeamMost];
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
        Pair sum{0.0f, 0.0f};
        if (kind == 2) {
            float m[kBeamMostParts / 32];
            Pair z[kBeamMostParts / 32];
#pragma unroll
            for (int i = 0; i < kBeamMostParts / 32; ++i) {
                const int p = lane + 32 * i;
                m[i] = neg_inf();
                z[i] = Pair{0.0f, 0.0f};
                if (p < a.parts) {
                    const BeamPart &part = a.meta[row * a.parts + p];
                    m[i] = part.top;
                    z[i] = Pair{part.sum, part.rest};
                }
                top = fmaxf(top, m[i]);
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
            for (int i = 0; i < kBeamMostParts / 32; ++i)
                if (z[i].hi != 0.0f) {  // (an empty part: -inf - -inf)
                    const float w = expf(m[i] - top);
                    sum = add(sum, Pair{z[i].hi * w, __fmaf_rn(z[i].lo, w, __fmaf_rn(z[i].hi, w, -(z[i].hi * w)))});
                }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1)
                sum = add(sum, Pair{__shfl_xor_sync(0xffffffffu, sum.hi, o), __shfl_xor_sync(0xffffffffu, sum.lo, o)});
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
        Pair shift{score, 0.0f};
        if (s.kind[tid] == 2) {
            // NaN or +inf among the logits, or none above -inf: the row's softmax is NaN
            if (!(s.sum[tid].hi > 0.0f))
                s.kind[tid] = 0;
            const Pair l = log_of(s.sum[tid]);
            shift = add(shift, Pair{-l.hi, -l.lo});
        }
        s.shift[tid] = shift;
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
    const int64_t piece = 16 / es, least = kBeamThreads * piece, block = kBeamLoads * least;
    auto up = [](int64_t x, int64_t d) { return (x + d - 1) / d; };
    // about eight parts an SM, of one piece a thread at least, and of whole blocks past one
    int64_t n = up(8 * n_sm, rows < 1 ? 1 : rows);
    n = std::min(std::min(n, up(vocab, least)), int64_t(kBeamMostParts));
    int64_t each = up(up(vocab, n), piece) * piece;
    if (each > block)
        each = up(each, block) * block;
    *part = static_cast<int32_t>(each);
    *parts = static_cast<int32_t>(up(vocab, each));
}

// Entries of a part's list: what a block with a bound of its own may add to what is kept.
static int32_t list_entries(int32_t keep, int dtype)
{
    return std::max(keep, 16) * kGroupLanes * kBeamLoads * (dtype == BSM_F32 ? 4 : 8) + keep;
}

int launch_beam_select(BeamSelectArgs a, int dtype, void *stream)
{
    a.list = list_entries(a.keep, dtype);
    const size_t smem = static_cast<size_t>(a.list + a.keep) * sizeof(BeamEntry);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 grid(static_cast<unsigned>(a.n) * a.beams * a.parts);
    int e = dtype == BSM_F32    ? launch_early(select_rows<BSM_F32>, grid, kBeamThreads, smem, st, a)
            : dtype == BSM_BF16 ? launch_early(select_rows<BSM_BF16>, grid, kBeamThreads, smem, st, a)
                                : launch_early(select_rows<BSM_F16>, grid, kBeamThreads, smem, st, a);
    if (e)
        return e;
    return a.keep <= 32 ? launch_early(select_join<1>, dim3(a.n), kBeamThreads, 0, st, a)
                        : launch_early(select_join<2>, dim3(a.n), kBeamThreads, 0, st, a);
}

int beam_set_smem_limit()
{
    int e = 0;
    auto set = [&](const void *f, int dtype) {
        if (!e)
            e = static_cast<int>(cudaFuncSetAttribute(
                f, cudaFuncAttributeMaxDynamicSharedMemorySize,
                static_cast<int>((list_entries(kBeamMost, dtype) + kBeamMost) * sizeof(BeamEntry))));
    };
    set(reinterpret_cast<const void *>(&select_rows<BSM_F32>), BSM_F32);
    set(reinterpret_cast<const void *>(&select_rows<BSM_BF16>), BSM_BF16);
    set(reinterpret_cast<const void *>(&select_rows<BSM_F16>), BSM_F16);
    return e;
}

}  // namespace bsm
