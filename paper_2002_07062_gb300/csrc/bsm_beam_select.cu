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
constexpr int kMostWarps = 16;
constexpr int kRowThreads = 512, kRowCtas = 3;  // of select_rows; its CTAs on an SM
constexpr int kJoinThreads = 512;                // of select_join and select_together
constexpr int kListRows = 20;                    // see beam_cut
constexpr int kMostTogether = 8;                 // requests (a cluster takes about 0.3 us to start)
constexpr int kCluster = 16;                     // CTAs of select_together that share a request

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

// A number as a whole one of the same order.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);               // (-0 becomes 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float disordered(uint32_t u)
{
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

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
    // whether a value of a is above its counterpart in b (or NaN)
    static __device__ __forceinline__ bool above(uint32_t a, uint32_t b)
    {
        if (kType == BSM_F32)
            return !(__uint_as_float(a) <= __uint_as_float(b));
        if (kType == BSM_BF16)
            return !__hble2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
        return !__hble2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    }
    // whether a value of a is not below its counterpart in b
    static __device__ __forceinline__ bool reaches(uint32_t a, uint32_t b)
    {
        if (kType == BSM_F32)
            return __uint_as_float(a) >= __uint_as_float(b);
        if (kType == BSM_BF16)
            return !__hblt2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
        return !__hblt2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    }
    static __device__ __forceinline__ uint32_t twice(float x)
    {
        if (kType == BSM_F32)
            return __float_as_uint(x);
        if (kType == BSM_BF16) {
            const __nv_bfloat162 v = __float2bfloat162_rn(x);
            return *reinterpret_cast<const uint32_t *>(&v);
        }
        const __half2 v = __float2half2_rn(x);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    // The largest value of the type, twice, that is at most x + 4.
    static __device__ __forceinline__ uint32_t four_above(float x)
    {
        const float y = __fadd_rd(x, 4.0f);
        if (kType == BSM_F32)
            return __float_as_uint(y);
        if (kType == BSM_BF16) {
            const __nv_bfloat162 v = __bfloat162bfloat162(__float2bfloat16_rd(y));
            return *reinterpret_cast<const uint32_t *>(&v);
        }
        const __half2 v = __half2half2(__float2half_rd(y));
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static __device__ __forceinline__ float most(uint32_t w)            // (not NaN)
    {
        float x[kN];
        get(w, x);
        return fmaxf(fmaxf(x[0], x[kN - 1]), neg_inf());
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

// Logits that are not kept in the first-level cache, which has room for what is on its way and little else.  With the
// join: 82 MB of fp32 on changing inputs 27 -> 25 us, 252 MB of bf16 there no change (65), the same ones again, half
// of them in the L2 cache, 64 -> 56; but 82 MB that all lie there 18.7 -> 22, what a product that has just written
// fewer than 100 MB of logits leaves: there plain loads would be better.
__device__ __forceinline__ uint4 stream_load(const unsigned char *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Values [i, i + W) of a row of n, -inf from hi on (the end of a part, or of the row).  A row may
// start `off` bytes past a 16-byte boundary: its pieces are put together from two neighbouring aligned
// ones (the second is the next lane's first and comes from the first-level cache), at the row's ends from
// single values.  Which values a thread gets depends on their index alone, so equal rows give equal
// sums wherever they lie.
template <int kType>
__device__ __forceinline__ uint4 load_piece(const unsigned char *row, uint32_t off, int32_t i, int32_t hi, int32_t n)
{
    using T = Word<kType>;
    constexpr int W = T::kW;
    uint32_t w[4] = {T::kNone, T::kNone, T::kNone, T::kNone};
    if (i >= hi)
        return make_uint4(w[0], w[1], w[2], w[3]);
    const unsigned char *p = row + static_cast<int64_t>(i) * T::kEs;
    if (off == 0 ? i + W <= n : i > 0 && i + 2 * W <= n) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p - off);
        return off == 0 ? v : shifted(v, *reinterpret_cast<const uint4 *>(p - off + 16), off);
    }
#pragma unroll
    for (int k = 0; k < W; ++k) {
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
    alignas(16) float group[kGroups];               // the largest value of each group
    int32_t first[kGroups];             // where a group's value ties with the bound: its lowest token
    float warp_top[kMostWarps], warp_sum[kMostWarps];
    uint32_t bound;
    int32_t count, last, hits;
    int16_t hit[kMostWarps * 32];       // threads whose largest value reaches the bound; entries of a long list
    int16_t four[kMostWarps * 32];      // which four pieces of theirs it is in, -1: several
    uint64_t key[kGroups], key_bound;
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
template <int kType, int kThreads, typename F> __device__ __forceinline__ void each_value(const uint4 (&v)[kBeamLoads], int32_t first, F &&f)
{
    using T = Word<kType>;
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j) {
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        const int32_t token = first + (j * kThreads + static_cast<int>(threadIdx.x)) * T::kW;
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

// An entry as a whole number of its order: larger values first, then lower tokens.
__device__ __forceinline__ uint64_t key_of(const BeamEntry &e)
{
    return static_cast<uint64_t>(ordered(e.x)) << 32 | ~static_cast<uint32_t>(e.token);
}

// The list's best `keep` in order to `to`: four threads count for each entry how many are better.  In
// a long list (equal values, or a part with few of any) the keep-th largest of 128 group maxima first
// says which ones that can be.
template <int kThreads> __device__ __forceinline__ void rank_list(PartSmem &s, const BeamEntry *list, int count, int keep, BeamEntry *to)
{
    constexpr int kLanes = kThreads / kGroups;
    const int tid = threadIdx.x, lane = tid & 31;
    int few = -1;
    if (count > kGroups) {
        uint64_t best = 0;
        for (int i = tid; i < count; i += kThreads)
            best = max(best, key_of(list[i]));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1)
            best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        if (tid % kLanes == 0)
            s.key[tid / kLanes] = best;
        if (tid == 0) {
            s.key_bound = 0;
            s.hits = 0;
        }
        __syncthreads();
        int over = 0;
        for (int k = tid % kLanes; k < kGroups; k += kLanes)
            over += s.key[k] > best;
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1)
            over += __shfl_xor_sync(0xffffffffu, over, o);
        if (over == keep - 1 && best != 0)
            s.key_bound = best;
        __syncthreads();
        const uint64_t bound = s.key_bound;
        for (int i = tid; i < count; i += kThreads)
            if (key_of(list[i]) >= bound) {
                const int at = atomicAdd(&s.hits, 1);
                if (at < kMostWarps * 32)
                    s.hit[at] = static_cast<int16_t>(i);
            }
        __syncthreads();
        few = s.hits <= kMostWarps * 32 ? s.hits : -1;
    }
    const int of = few >= 0 ? few : count;
    for (int i0 = (tid >> 5) * 8; i0 < of; i0 += kThreads / 4) {
        const int i = i0 + lane / 4;
        const BeamEntry e = list[i >= of ? 0 : few >= 0 ? s.hit[i] : i];
        int better = 0;
#pragma unroll 4
        for (int k = lane & 3; k < of; k += 4) {
            const BeamEntry o = list[few >= 0 ? s.hit[k] : k];
            better += (o.x > e.x) | ((o.x == e.x) & (o.token < e.token));
        }
        better += __shfl_xor_sync(0xffffffffu, better, 1);
        better += __shfl_xor_sync(0xffffffffu, better, 2);
        if (lane % 4 == 0 && i < of && better < keep)
            to[better] = e;
    }
}

// The smallest of the group maxima that fewer than `keep` groups exceed, so that `keep` values reach it
// (-inf where fewer than `keep` groups have any).  best: this thread's largest value; becomes
// its group's.  Everything written before by the block can be read after it.
template <int kThreads> __device__ __forceinline__ float group_bound(PartSmem &s, float &best, int keep)
{
    constexpr int kLanes = kThreads / kGroups;
    const int tid = threadIdx.x;
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1)
        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (tid % kLanes == 0)
        s.group[tid / kLanes] = best;
    if (tid == 0)
        s.bound = 0xffffffffu;
    __syncthreads();
    int over = 0;                       // (a group's threads share the count)
#pragma unroll
    for (int k = 0; k < kGroups / 4 / kLanes; ++k) {
        const float4 o = reinterpret_cast<const float4 *>(s.group)[k * kLanes + tid % kLanes];
        over += (o.x > best) + (o.y > best) + (o.z > best) + (o.w > best);
    }
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1)
        over += __shfl_xor_sync(0xffffffffu, over, o);
    if (over < keep && tid % kLanes == 0)
        atomicMin(&s.bound, ordered(best));
    __syncthreads();
    return disordered(s.bound);
}

// A block's bound.  Where more than `keep` groups reach it some tie there: of values equal to the bound
// only those up to token *last are needed then, and those that count lie in `keep` groups at most.
template <int kType, int kThreads>
__device__ __forceinline__ float block_bound(PartSmem &s, const uint4 (&v)[kBeamLoads], float mine, int32_t first, int keep, int32_t *last)
{
    constexpr int kLanes = kThreads / kGroups;
    const int tid = threadIdx.x;
    const bool speaks = tid % kLanes == 0;
    float best = mine;
    const float bound = group_bound<kThreads>(s, best, keep);
    *last = bound == neg_inf() ? -1 : INT_MAX;
    if (bound == neg_inf() || __syncthreads_count(speaks && best >= bound) <= keep)
        return bound;
    const int above = __syncthreads_count(speaks && best > bound);
    int32_t at = INT_MAX;
    if (mine == bound)
        each_value<kType, kThreads>(v, first, [&](float x, int32_t token) {
            if (x == bound)
                at = min(at, token);
        });
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1)
        at = min(at, __shfl_xor_sync(0xffffffffu, at, o));
    if (speaks)
        s.first[tid / kLanes] = best == bound ? at : INT_MAX;
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

// Values above the bound, and equal ones up to token `last`, to the list, in any order; pieces
// without one are skipped.  Entries past the list's end are counted only.
template <int kType, int kThreads>
__device__ __forceinline__ void to_list(PartSmem &s, BeamEntry *list, int room, const uint4 (&v)[kBeamLoads], float mine, int32_t first,
                                        float bound, int32_t last)
{
    using T = Word<kType>;
    if ((last < 0 ? mine <= bound : mine < bound) || mine == neg_inf())
        return;
#pragma unroll
    for (int j = 0; j < kBeamLoads; ++j) {
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        float ends[T::kN];
        T::get(T::larger(T::larger(w[0], w[1]), T::larger(w[2], w[3])), ends);
        if (!(fmaxf(ends[0], ends[T::kN - 1]) >= bound))
            continue;
        const int32_t token = first + (j * kThreads + static_cast<int>(threadIdx.x)) * T::kW;
#pragma unroll
        for (int k = 0; k < T::kW; ++k) {
            float x[T::kN];
            T::get(w[k / T::kN], x);
            const float one = x[k % T::kN];
            if ((one > bound) | ((one == bound) & (token + k <= last))) {
                const int i = atomicAdd(&s.count, 1);
                if (i < room)
                    list[i] = BeamEntry{one, token + k};
            }
        }
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
template <int kType, int kThreads>
__device__ __noinline__ int list_again(PartSmem &s, BeamEntry *list, int room, int keep, const unsigned char *row, uint32_t off,
                                       int32_t lo, int32_t hi, int32_t n)
{
    const int tid = threadIdx.x;
    int count = 0;
    float bound = neg_inf();
    for (int32_t first = lo; first < hi; first += kThreads * kBeamLoads * Word<kType>::kW) {
        uint4 v[kBeamLoads];
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j)
            v[j] = load_piece<kType>(row, off, first + (j * kThreads + tid) * Word<kType>::kW, hi, n);
        const float mine = largest<kType>(v);
        if (tid == 0)
            s.count = count;
        int32_t last;
        const float b = block_bound<kType, kThreads>(s, v, mine, first, keep, &last);     // (its barriers order the count)
        if (b > bound)
            bound = b;
        else
            last = -1;
        to_list<kType, kThreads>(s, list, room, v, mine, first, bound, last);
        __syncthreads();
        count = s.count;
        rank_list<kThreads>(s, list, count, keep, list + room);
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

// Where a row of logits starts.
__device__ __forceinline__ const unsigned char *row_at(const BeamSelectArgs &a, uint32_t row)
{
    const unsigned char *base = a.logits + row * a.stride_beam;
    if (a.stride_request != a.beams * a.stride_beam)
        base += row / static_cast<uint32_t>(a.beams) * (a.stride_request - a.beams * a.stride_beam);
    return base;
}

// Whether a beam's logits matter: it has a score, and is not finished.  (Both are asked for at once.)
__device__ __forceinline__ bool reads_logits(const BeamSelectArgs &a, uint32_t row)
{
    const float score = a.scores[row];
    const uint8_t ended = a.ended ? a.ended[row] : 0;
    return fabsf(score) < __int_as_float(0x7f800000) && ended == 0;
}

// A thread's first pieces of logits [lo, hi) of a row.
template <int kType, int kThreads>
__device__ __forceinline__ void load_first(uint4 (&v)[kBeamLoads], const unsigned char *base, int32_t lo, int32_t hi, int32_t n)
{
    using T = Word<kType>;
    constexpr int kRow = kThreads * T::kW;
    const int tid = threadIdx.x;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) & 15u;
    if (off == 0 && lo + kBeamLoads * kRow <= hi) {
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j)
            v[j] = stream_load(base + static_cast<int64_t>(lo + j * kRow + tid * T::kW) * T::kEs);
    } else {
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j)
            v[j] = load_piece<kType>(base, off, lo + (j * kThreads + tid) * T::kW, hi, n);
    }
}

// One part of a row.  A thread takes a piece of 16 bytes from each 8 KiB (whole rows of the block's
// threads): four are on their way or at hand, and each makes room for the one four further.  A
// thread keeps a maximum and a sum of exponentials of its own and waits for nobody.  At the end the
// keep-th largest of 128 group maxima is a bound that the part's best `keep` values reach and few
// others (about as many again): the threads whose maximum reaches it are few, and the four pieces that it was in
// are read once more (all of theirs, where others of them reach the bound too).
//
// Bound by the bytes while it streams, by about 500 instructions a warp for the list at each part's end: 1024 rows
// of 128000, 249 MB, the join with it: 63 us on changing inputs, 55 on the same ones again, half of them in the L2
// cache (65 and 56 with all pieces of those threads read again: they lie 8 KiB apart and may have left it).  That is with three CTAs of 512 threads (40 registers); of 256 or 128
// threads 64 to 82; eight pieces at hand and two CTAs 71; the values listed on the way under a bound
// carried from block to block 82 to 109; the next CTA's part asked into the L2 cache 80.
// (v: the thread's first pieces.)
template <int kType, int kThreads>
__device__ __forceinline__ void take_part(const BeamSelectArgs &a, PartSmem &s, BeamEntry *list, const unsigned char *base, int32_t lo,
                                          int32_t hi, uint4 (&v)[kBeamLoads], BeamPart *meta, BeamEntry *to)
{
    using T = Word<kType>;
    constexpr int kWarps = kThreads / 32, kRow = kThreads * T::kW;      // values of a row of pieces
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) & 15u;
    auto load = [&](int32_t first) { return load_piece<kType>(base, off, first + tid * T::kW, hi, a.vocab); };
    if (tid == 0)
        s.count = s.hits = 0;
    // exp(x - from) = 2^((x - from) log2(e)), where `from` is a value seen that lies 4 below the largest at
    // most: it seldom moves, and the arguments of the terms that matter stay small, so exact
    float from = neg_inf(), sum = 0.0f;
    uint32_t most = T::kNone, limit = T::kNone;         // the largest of four pieces; from + 4, rounded down
    float top = neg_inf(), second = neg_inf();          // the largest of all; that of the other fours
    int32_t top_at = 0, four = 0;                       // which four pieces it is in
    uint64_t minus = 0, sum2 = 0;       // -from twice (0 while nothing but -inf was seen: it sums up to 0); sums of four pieces
    auto take = [&](const uint4 &x) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        const uint32_t here = T::larger(T::larger(w[0], w[1]), T::larger(w[2], w[3]));
        most = T::larger(most, here);
        if (T::above(here, limit)) {
            const float high = T::most(here);
            if (high > from) {
                const float scale = pg_exp2((from - high) * 1.4426950408889634f);
                sum *= scale;
                sum2 = mul2(sum2, pack2(scale, scale));
                from = high;
                limit = T::four_above(from);
                minus = pack2(-from, -from);
            }
        }
        const uint64_t log2e = pack2(1.4426950408889634f, 1.4426950408889634f);
#pragma unroll
        for (int k = 0; k < 4; k += 2 / T::kN) {
            float y[T::kN], z[T::kN];
            T::get(w[k], y);
            T::get(w[(k + 1) % 4], z);
            const uint64_t t = mul2(add2(pack2(y[0], T::kN == 2 ? y[T::kN - 1] : z[0]), minus), log2e);
            sum2 = add2(sum2, pack2(pg_exp2(low2(t)), pg_exp2(high2(t))));
        }
    };
    auto fold = [&]() {
        sum += low2(sum2) + high2(sum2);
        sum2 = 0;
        const float high = T::most(most);
        second = fmaxf(second, fminf(top, high));
        top_at = high > top ? four : top_at;
        top = fmaxf(top, high);
        most = T::kNone;
        ++four;
    };
    // four rows of pieces are at hand; those four further are on their way while these are worked on
    constexpr int kSpan = kBeamLoads * kRow;
    int further = (hi - lo) / kSpan - 1;                // spans past the first that need no look at the ends
    if (off != 0 && lo + (further + 1) * kSpan + T::kW > a.vocab)
        --further;
    int32_t first = lo;
    const unsigned char *p = base + static_cast<int64_t>(lo + tid * T::kW) * T::kEs - off;
    bool raw = false;                   // the pieces at hand wait to be shifted into place
    if (off == 0) {
        for (int g = 0; g < further; ++g) {
            p += kSpan * T::kEs;
#pragma unroll
            for (int j = 0; j < kBeamLoads; ++j) {
                take(v[j]);
                v[j] = stream_load(p + j * kRow * T::kEs);
            }
            fold();
        }
    } else {
        for (int g = 0; g < further; ++g) {
            p += kSpan * T::kEs;
#pragma unroll
            for (int j = 0; j < kBeamLoads; ++j) {
                take(raw ? shifted(v[j], *reinterpret_cast<const uint4 *>(p + (j - kBeamLoads) * kRow * T::kEs + 16), off) : v[j]);
                v[j] = *reinterpret_cast<const uint4 *>(p + j * kRow * T::kEs);
            }
            raw = true;
            fold();
        }
    }
    first += (further > 0 ? further : 0) * kSpan;
    for (; first < hi; first += kSpan) {
#pragma unroll
        for (int j = 0; j < kBeamLoads; ++j) {
            if (first + j * kRow < hi)
                take(raw ? shifted(v[j], *reinterpret_cast<const uint4 *>(p + j * kRow * T::kEs + 16), off) : v[j]);
            const int32_t then = first + kSpan + j * kRow;
            if (off == 0 && then + kRow <= hi)
                v[j] = *reinterpret_cast<const uint4 *>(p + (kBeamLoads + j) * kRow * T::kEs);
            else if (then < hi)
                v[j] = load(then);
        }
        p += kSpan * T::kEs;
        raw = false;
        fold();
    }
    // the part's maximum and sum: each warp's here, of them all by one warp below
    float all = top;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    sum *= all == neg_inf() ? 1.0f : pg_exp2((from - all) * 1.4426950408889634f);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
        s.warp_top[warp] = all;
        s.warp_sum[warp] = sum;
    }
    float best = top;
    const float bound = group_bound<kThreads>(s, best, a.keep);
    if (top >= bound && top > neg_inf()) {
        const int h = atomicAdd(&s.hits, 1);
        s.hit[h] = static_cast<int16_t>(tid);
        s.four[h] = static_cast<int16_t>(second >= bound ? -1 : top_at);
    }
    __syncthreads();
    const int rows = (hi - lo + kRow - 1) / kRow, found = s.hits;
    const uint32_t bound2 = T::twice(bound);            // (a value of this type)
    auto look = [&](int h, int r) {
        const int32_t i = lo + r * kRow + s.hit[h] * T::kW;
        const uint4 x = load_piece<kType>(base, off, i, hi, a.vocab);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!T::reaches(w[k], bound2))
                continue;
            float z[T::kN];
            T::get(w[k], z);
#pragma unroll
            for (int e = 0; e < T::kN; ++e) {
                if (!(z[e] >= bound) || z[e] == neg_inf())
                    continue;
                const int to_at = atomicAdd(&s.count, 1);
                if (to_at < a.list)
                    list[to_at] = BeamEntry{z[e], i + k * T::kN + e};
            }
        }
    };
    // nearly always in four pieces alone: a piece a lane; else all of them, by a warp
    for (int h = tid / kBeamLoads; h < found; h += kThreads / kBeamLoads)
        if (s.four[h] >= 0)
            look(h, s.four[h] * kBeamLoads + tid % kBeamLoads);
    for (int h = warp; h < found; h += kWarps)
        if (s.four[h] < 0)
            for (int r = lane; r < rows; r += 32)
                look(h, r);
    __syncthreads();
    int count = s.count;
    if (count > a.list) {
        __syncthreads();                // (every thread has read the count)
        count = list_again<kType, kThreads>(s, list, a.list, a.keep, base, off, lo, hi, a.vocab);
    }
    if (warp == kWarps - 1) {           // (the last one to have entries to rank)
        const float warp_top = lane < kWarps ? s.warp_top[lane] : neg_inf();
        all = warp_top;
#pragma unroll
        for (int o = 1; o < kWarps; o <<= 1)
            all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
        all = __shfl_sync(0xffffffffu, all, 0);
        Pair z{lane < kWarps ? s.warp_sum[lane] * (all == neg_inf() ? 1.0f : pg_exp2((warp_top - all) * 1.4426950408889634f)) : 0.0f, 0.0f};
#pragma unroll
        for (int o = 1; o < kWarps; o <<= 1)
            z = add(z, Pair{__shfl_xor_sync(0xffffffffu, z.hi, o), __shfl_xor_sync(0xffffffffu, z.lo, o)});
        if (lane == 0)
            *meta = BeamPart{z.hi, z.lo, all, min(count, a.keep)};
    }
    rank_list<kThreads>(s, list, count, a.keep, to);
}

// A candidate: its value as a whole number of the same order, and its place among the
// request's (beam * vocab + token), the lower one first where values are equal.
struct Cand {
    uint64_t key;                       // 0: none
    int32_t at;
};
__device__ __forceinline__ Cand no_cand() { return Cand{0, INT_MAX}; }
__device__ __forceinline__ Cand cand(const Pair &x, int32_t at)
{
    return Cand{static_cast<uint64_t>(ordered(x.hi)) << 32 | ordered(x.lo), at};
}
// (without branches: it runs in loops over shared memory)
__device__ __forceinline__ bool better(const Cand &a, const Cand &b)
{
    return (a.key > b.key) | ((a.key == b.key) & (a.at < b.at));
}
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

constexpr int kJoinAll = 128;                    // entries that are ordered without a bound

// Entries that a join orders at most: those of fewer groups than are kept (each has the entries of 4 threads), or all.
__host__ __device__ __forceinline__ int most_kept(int keep)
{
    const int n = keep * 4 * ((kBeamMostLists * keep + kJoinThreads - 1) / kJoinThreads);
    return n > kJoinAll ? n : kJoinAll;
}

struct JoinSmem {   // (score and kind are set before the join)
    float score[kBeamMost], top[kBeamMost];
    Pair shift[kBeamMost];              // score - log(sum): what a row adds to x - top
    int32_t kind[kBeamMost];            // 0: no candidate, 1: one (an ended beam), 2: its parts' lists
    int8_t beam[kBeamMostLists];        // of a list
    Cand bound;
    int32_t count;
};

// A request's lists in shared memory.
struct Lists {
    BeamPart *meta;
    BeamEntry *entries;                 // `keep` each
    Cand *heads, *kept;
};

// Entry i of list l, by value: score + (x - top) - log(sum) in two fp32 numbers.
__device__ __forceinline__ Cand entry(const BeamSelectArgs &a, const JoinSmem &s, const Lists &z, int l, int i)
{
    const int b = s.beam[l];
    if (s.kind[b] != 2)
        return s.kind[b] == 1 && l == b * a.parts && i == 0 ? cand(s.shift[b], b * a.vocab + a.end_token) : no_cand();
    if (i >= z.meta[l].count)
        return no_cand();
    const BeamEntry e = z.entries[l * a.keep + i];
    const Pair x = add(two_sum(e.x, -s.top[b]), s.shift[b]);
    return x.hi > neg_inf() ? cand(x, b * a.vocab + e.token) : no_cand();      // (not beyond fp32's range)
}

// How many of n candidates are better than c, which four neighbouring threads share.
__device__ __forceinline__ int count_better(const Cand *all, int n, const Cand &c)
{
    int before = 0;
#pragma unroll 4
    for (int k = threadIdx.x & 3; k < n; k += 4)
        before += better(all[k], c);
    before += __shfl_xor_sync(0xffffffffu, before, 1);
    before += __shfl_xor_sync(0xffffffffu, before, 2);
    return before;
}

// The lists of all parts of all beams of a request, in order: the few entries that reach a bound are
// ordered by counting for each how many are better.  Latency: four barriers and the lists' way to shared
// memory, 5 us (128 requests of 8 lists of 16).  With the lists' first entries alone for the bound 125 lists of 32 left 391
// entries to order and took 20 us.
__device__ __forceinline__ void join(const BeamSelectArgs &a, JoinSmem &s, const Lists &z, int32_t request, int lists)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        s.bound = no_cand();
        s.count = 0;
    }
    for (int b = warp; b < a.beams; b += (kJoinThreads / 32)) {
        const float score = s.score[b];
        int32_t kind = s.kind[b];
        float top = neg_inf();
        Pair shift{score, 0.0f};
        if (kind == 2) {
            const BeamPart *meta = z.meta + b * a.parts;
            for (int p = lane; p < a.parts; p += 32)
                top = fmaxf(top, meta[p].top);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            Pair sum{0.0f, 0.0f};
            for (int p = lane; p < a.parts; p += 32) {
                const BeamPart x = meta[p];
                if (x.sum != 0.0f) {    // (an empty part: -inf - -inf)
                    const float w = expf(x.top - top), m = x.sum * w;
                    sum = add(sum, Pair{m, __fmaf_rn(x.rest, w, __fmaf_rn(x.sum, w, -m))});
                }
            }
            for (int o = 16; o > 0; o >>= 1)
                if (o < a.parts)
                    sum = add(sum, Pair{__shfl_xor_sync(0xffffffffu, sum.hi, o), __shfl_xor_sync(0xffffffffu, sum.lo, o)});
            // NaN or +inf among the logits, or none above -inf: the row's softmax is NaN
            if (!(sum.hi > 0.0f && sum.hi < __int_as_float(0x7f800000)))
                kind = 0;
            const Pair l = log_of(sum);
            shift = add(shift, Pair{-l.hi, -l.lo});
        }
        if (lane == 0) {
            s.top[b] = top;
            s.shift[b] = shift;
            s.kind[b] = kind;
        }
    }
    __syncthreads();
    // the keep-th largest of the maxima of 128 groups of entries (of the lists' first ones, of their second ones,
    // ..) is a bound that `keep` of them reach
    const int entries = lists * a.keep;
    const bool all = entries <= kJoinAll;
    if (!all) {
        Cand best = no_cand();
        for (int e = tid; e < entries; e += kJoinThreads) {
            const int i = e / lists;
            const Cand c = entry(a, s, z, e - i * lists, i);
            best = better(c, best) ? c : best;
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            const Cand c{__shfl_xor_sync(0xffffffffu, best.key, o), __shfl_xor_sync(0xffffffffu, best.at, o)};
            best = better(c, best) ? c : best;
        }
        if (tid % 4 == 0)
            z.heads[tid / 4] = best;
        __syncthreads();
        const int before = count_better(z.heads, kJoinThreads / 4, best);
        if (best.key != 0 && before == a.keep - 1)
            s.bound = best;             // (four threads, the same one)
        __syncthreads();
    }
    const Cand bound = s.bound;         // none where fewer groups have an entry
    for (int e = tid; e < entries; e += kJoinThreads) {
        const int i = e / lists;
        const Cand c = entry(a, s, z, e - i * lists, i);
        if (c.key != 0 && !better(bound, c))
            z.kept[atomicAdd(&s.count, 1)] = c;
    }
    __syncthreads();
    const int count = s.count;
    const int64_t to = static_cast<int64_t>(request) * a.keep;
    for (int i0 = warp * 8; i0 < count; i0 += kJoinThreads / 4) {
        const int i = i0 + lane / 4;
        const Cand c = z.kept[i < count ? i : 0];
        const int before = count_better(z.kept, count, c);
        if (lane % 4 == 0 && i < count && before < a.keep) {
            // (the larger of the two numbers is the value rounded to fp32)
            const int32_t parent = static_cast<int32_t>(static_cast<uint32_t>(c.at) / static_cast<uint32_t>(a.vocab));
            a.out_scores[to + before] = disordered(static_cast<uint32_t>(c.key >> 32));
            a.parents[to + before] = parent;
            a.tokens[to + before] = c.at - parent * a.vocab;
        }
    }
    for (int i = count + tid; i < a.keep; i += kJoinThreads) {
        a.out_scores[to + i] = neg_inf();
        a.parents[to + i] = -1;
        a.tokens[to + i] = -1;
    }
}

// A request's scores, which beams have candidates, and whose each list is.
__device__ __forceinline__ void get_beams(const BeamSelectArgs &a, JoinSmem &s, int32_t request)
{
    const int b = threadIdx.x;
    if (b < a.beams) {
        const int64_t row = static_cast<int64_t>(request) * a.beams + b;
        const float score = a.scores[row];
        const bool ended = a.ended && a.ended[row];
        s.score[b] = score;
        s.kind[b] = !(fabsf(score) < __int_as_float(0x7f800000)) ? 0 : ended ? 1 : 2;
    }
    for (int l = threadIdx.x; l < a.beams * a.parts; l += kJoinThreads)
        s.beam[l] = static_cast<int8_t>(l / a.parts);
}

// Dynamic shared memory of a join.
__device__ __forceinline__ Lists lists_at(const BeamSelectArgs &a, unsigned char *raw, int lists)
{
    Lists z;
    z.heads = reinterpret_cast<Cand *>(raw);
    z.kept = z.heads + kJoinThreads / 4;
    z.meta = reinterpret_cast<BeamPart *>(z.kept + most_kept(a.keep));
    z.entries = reinterpret_cast<BeamEntry *>(z.meta + lists);
    return z;
}

template <int kType> __global__ void __launch_bounds__(kRowThreads, kRowCtas) select_rows(const BeamSelectArgs a)
{
    __shared__ PartSmem s;
    extern __shared__ __align__(16) unsigned char raw[];
    grid_dependency_wait();
    grid_launch_dependents();
    const uint32_t row = a.parts == 1 ? blockIdx.x : blockIdx.x / static_cast<uint32_t>(a.parts);
    const int32_t lo = static_cast<int32_t>(blockIdx.x - row * a.parts) * a.part, hi = min(lo + a.part, a.vocab);
    if (!reads_logits(a, row))
        return;
    const unsigned char *base = row_at(a, row);
    uint4 v[kBeamLoads];
    load_first<kType, kRowThreads>(v, base, lo, hi, a.vocab);
    take_part<kType, kRowThreads>(a, s, reinterpret_cast<BeamEntry *>(raw), base, lo, hi, v, a.meta + blockIdx.x,
                                  a.entries + static_cast<int64_t>(blockIdx.x) * a.keep);
}

__global__ void __launch_bounds__(kJoinThreads) select_join(const BeamSelectArgs a)
{
    __shared__ JoinSmem s;
    extern __shared__ __align__(16) unsigned char raw[];
    const int32_t request = blockIdx.x, lists = a.beams * a.parts;
    const int64_t first = static_cast<int64_t>(request) * lists;
    const Lists z = lists_at(a, raw, lists);
    grid_dependency_wait();
    grid_launch_dependents();
    // (of beams without a list it copies what happens to be there, and nobody reads it)
    for (int i = threadIdx.x; i < lists; i += kJoinThreads)
        reinterpret_cast<uint4 *>(z.meta)[i] = reinterpret_cast<const uint4 *>(a.meta + first)[i];
    for (int i = threadIdx.x; i < lists * a.keep; i += kJoinThreads)
        z.entries[i] = a.entries[first * a.keep + i];
    get_beams(a, s, request);
    __syncthreads();
    join(a, s, z, request, lists);
}

// Both in one launch: a cluster takes a request's parts, their lists go to the first CTA's shared memory,
// and it joins them.  One request of 4 beams over 32000: 7 to 8 us, 9.6 in two launches; a call costs the host 2 us
// less.  A cluster of 16 takes its time to start: 28 requests of one beam over 4000 took 13 us, 7 in two launches.
// Whether a list's beam has logits to read is known before its first load, and asked for while the cluster starts: 7.6 us, 7.65
// where every row was read (8 requests of 8 beams 11.25 and 10.95); with a third CTA on an SM, 40 registers and spills, 8.1.
template <int kType> __global__ void __launch_bounds__(kJoinThreads, 2) select_together(const BeamSelectArgs a)
{
    __shared__ PartSmem s;
    __shared__ JoinSmem j;
    extern __shared__ __align__(16) unsigned char raw[];
    const uint32_t request = blockIdx.x / kCluster, rank = blockIdx.x % kCluster, lists = static_cast<uint32_t>(a.beams) * a.parts;
    // the first CTA's shared memory may be written once it runs
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    const Lists z = lists_at(a, raw + static_cast<size_t>(a.list + a.keep) * sizeof(BeamEntry), lists);
    BeamPart *meta;
    BeamEntry *entries;
    asm("mapa.u64 %0, %1, 0;" : "=l"(meta) : "l"(z.meta));
    asm("mapa.u64 %0, %1, 0;" : "=l"(entries) : "l"(z.entries));
    grid_dependency_wait();
    grid_launch_dependents();
    // (logits of finished and of unused beams are not read, as in select_rows; which a list's are is asked for ahead)
    auto wanted = [&](uint32_t l) { return l < lists && reads_logits(a, request * a.beams + l / static_cast<uint32_t>(a.parts)); };
    bool reads = wanted(rank);
    if (rank == 0)
        get_beams(a, j, static_cast<int32_t>(request));
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    for (uint32_t l = rank; l < lists; l += kCluster) {
        const bool then = wanted(l + kCluster);
        if (reads) {
            const uint32_t b = l / static_cast<uint32_t>(a.parts);
            const int32_t lo = static_cast<int32_t>(l - b * a.parts) * a.part, hi = min(lo + a.part, a.vocab);
            const unsigned char *base = row_at(a, request * a.beams + b);
            uint4 v[kBeamLoads];
            load_first<kType, kJoinThreads>(v, base, lo, hi, a.vocab);
            take_part<kType, kJoinThreads>(a, s, reinterpret_cast<BeamEntry *>(raw), base, lo, hi, v, meta + l,
                                           entries + l * a.keep);
        }
        reads = then;
        __syncthreads();
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    if (rank == 0)
        join(a, j, z, static_cast<int32_t>(request), static_cast<int>(lists));
}

// The launch of a cluster a request.
struct ClusterLaunch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    ClusterLaunch(unsigned requests, size_t smem, cudaStream_t st)
    {
        cfg.gridDim = dim3(requests * kCluster);
        cfg.blockDim = dim3(kJoinThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kCluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
    }
    ClusterLaunch(const ClusterLaunch &) = delete;
};

// Entries of a part's list: what a block with a bound of its own may add to what is kept.
int32_t list_entries(int32_t keep, int dtype, int threads)
{
    return std::max(keep, 16) * (threads / kGroups) * kBeamLoads * (dtype == BSM_F32 ? 4 : 8) + keep;
}
size_t part_smem(int32_t keep, int dtype, int threads) { return static_cast<size_t>(list_entries(keep, dtype, threads) + keep) * sizeof(BeamEntry); }
size_t join_smem(int32_t lists, int32_t keep)
{
    return (kJoinThreads / 4 + most_kept(keep)) * sizeof(Cand) + lists * (sizeof(BeamPart) + keep * sizeof(BeamEntry));
}

}  // namespace

int64_t beam_most_lists(int64_t rows, int n_sm) { return std::max<int64_t>(rows, 8ll * n_sm * kRowCtas); }

// Requests that are few and short go to a cluster each, in one launch; the others' parts to all SMs, and
// their joins to a second launch; so do all where a device (a share of a GPU) places no cluster.  Every row is cut
// alike, so equal rows give equal bits.
BeamCut beam_cut(int32_t n, int32_t beams, int32_t vocab, int es, int n_sm, bool clusters)
{
    const int64_t piece = 16 / es, rows = static_cast<int64_t>(n) * beams;
    auto up = [](int64_t x, int64_t d) { return (x + d - 1) / d; };
    BeamCut c{};
    c.together = clusters && n <= kMostTogether && static_cast<int64_t>(beams) * vocab * es <= kCluster * kTogetherBytes;
    if (c.together) {
        // parts of a piece a thread at least
        int64_t parts = std::min<int64_t>(kCluster / beams, up(vocab, kJoinThreads * piece));
        parts = std::max<int64_t>(parts, 1);
        c.part = static_cast<int32_t>(up(up(vocab, parts), piece) * piece);
        c.parts = static_cast<int32_t>(up(vocab, c.part));
        return c;
    }
    // The parts whose waves take least: a part's list costs as much as kListRows of its rows of pieces.
    const int64_t row = kRowThreads * piece, pieces = up(vocab, row), at_once = static_cast<int64_t>(n_sm) * kRowCtas;
    const int64_t most = std::min(std::min<int64_t>(kBeamMostLists / beams, up(pieces, kBeamLoads)),
                                  std::max<int64_t>(beam_most_lists(rows, n_sm) / rows, 1));
    int64_t best = 0;
    for (int64_t parts = 1; parts <= most; ++parts) {
        const int64_t each = up(pieces, parts), cost = up(rows * up(pieces, each), at_once) * (each + kListRows);
        if (parts == 1 || cost < best) {
            best = cost;
            c.part = static_cast<int32_t>(std::min(each * row, up(vocab, piece) * piece));
            c.parts = static_cast<int32_t>(up(pieces, each));
        }
    }
    return c;
}

int launch_beam_select(BeamSelectArgs a, int dtype, const BeamCut &cut, void *stream)
{
    const int threads = cut.together ? kJoinThreads : kRowThreads;
    a.list = list_entries(a.keep, dtype, threads);
    a.parts = cut.parts;
    a.part = cut.part;
    const size_t part = part_smem(a.keep, dtype, threads), joint = join_smem(a.beams * a.parts, a.keep);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cut.together) {
        const ClusterLaunch l(static_cast<unsigned>(a.n), part + joint, st);
        return static_cast<int>(dtype == BSM_F32    ? cudaLaunchKernelEx(&l.cfg, select_together<BSM_F32>, a)
                                : dtype == BSM_BF16 ? cudaLaunchKernelEx(&l.cfg, select_together<BSM_BF16>, a)
                                                    : cudaLaunchKernelEx(&l.cfg, select_together<BSM_F16>, a));
    }
    const dim3 grid(static_cast<unsigned>(a.n) * a.beams * a.parts);
    const int e = dtype == BSM_F32    ? launch_early(select_rows<BSM_F32>, grid, kRowThreads, part, st, a)
                  : dtype == BSM_BF16 ? launch_early(select_rows<BSM_BF16>, grid, kRowThreads, part, st, a)
                                      : launch_early(select_rows<BSM_F16>, grid, kRowThreads, part, st, a);
    return e ? e : launch_early(select_join, dim3(a.n), kJoinThreads, joint, st, a);
}

int beam_set_smem_limit()
{
    int e = 0;
    auto set = [&](const void *f, size_t smem, bool cluster) {
        if (!e)
            e = static_cast<int>(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        if (!e && cluster)
            e = static_cast<int>(cudaFuncSetAttribute(f, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    };
    const size_t joint = join_smem(kBeamMostLists, kBeamMost);
    auto rows = [&](const void *f, const void *both, int dtype) {
        set(f, part_smem(kBeamMost, dtype, kRowThreads), false);
        set(both, part_smem(kBeamMost, dtype, kJoinThreads) + joint, true);
    };
    rows(reinterpret_cast<const void *>(&select_rows<BSM_F32>), reinterpret_cast<const void *>(&select_together<BSM_F32>), BSM_F32);
    rows(reinterpret_cast<const void *>(&select_rows<BSM_BF16>), reinterpret_cast<const void *>(&select_together<BSM_BF16>), BSM_BF16);
    rows(reinterpret_cast<const void *>(&select_rows<BSM_F16>), reinterpret_cast<const void *>(&select_together<BSM_F16>), BSM_F16);
    set(reinterpret_cast<const void *>(&select_join), joint, false);
    return e;
}

bool beam_clusters_fit()
{
    auto fits = [](void (*f)(BeamSelectArgs), int dtype) {
        ClusterLaunch l(1, part_smem(kBeamMost, dtype, kJoinThreads) + join_smem(kBeamMostLists, kBeamMost), nullptr);
        l.cfg.numAttrs = 1;             // (the cluster alone)
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, f, &l.cfg) != cudaSuccess) {
            cudaGetLastError();
            return false;
        }
        return n > 0;
    };
    return fits(select_together<BSM_F32>, BSM_F32) && fits(select_together<BSM_BF16>, BSM_BF16) &&
           fits(select_together<BSM_F16>, BSM_F16);
}

}  // namespace bsm
