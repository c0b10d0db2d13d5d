// bsm_paged_again.h -- rows of paged attention computed once more, from the
// definition, where the kernels' answer does not hold.
//
//   o = sum p_j v_j / sum p_j over the visible keys whose pages are there, in fp32
//
// A product of a block of rows with a block of keys cannot leave a key out for some of
// the rows: a masked key has weight 0 there, and 0 times an infinity or NaN among its
// values is NaN.  And the tile kernel's copies fill a key whose page is not there with
// zeros, so that it would enter with score 0.  The kernels note that a row of theirs is
// not finite, or that they met such a page, and which tiles they went through; the join
// launch, which follows anyway, looks at those tiles' rows and computes again what a hidden
// key got into: a warp a row, four columns a lane, 32 keys at a time.  Where all is finite
// and there it reads a flag a unit.
// Slow, bound by the latency of its loads: of a chunk of 2048 tokens over 6100 keys (0.17 ms) with a
// NaN among the values of its last token, the 63 tokens before it in their tile take 52 ms; all
// of them where one page of the request is missing 143 ms; a row whose sum or outputs are NaN
// for good ends there (all values NaN: 2.5 ms).  The rest is for the calls that need none of it:
// leaving such keys out in the tile kernel (its query warp looking at the values of keys that
// some rows do not see, its softmax masking keys without a page) cost every call 4 to 15 %.
// Nor is the code made longer than this: its size alone costs, even unexecuted.  With the walk
// along the work line in it (80 KB) that chunk took 163 us, with 39 KB 158.5, with 31 157.4.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged_dev.h"

namespace bsm {

constexpr float kPagedLn2 = 0.6931471805599453f;
constexpr int kAgainKeys = 2, kAgainValues = 4;     // pieces of a key's row, rows of values, loaded ahead

// What a unit's producer went through: the first tile that it starts, how many it has whole
// from there on.
struct PagedSeen {
    int32_t r = -1, head = 0, tile = 0, whole = 0;
    bool gone = false;                  // (of this lane) a key has no page
    __device__ __forceinline__ void note(const PagedPiece &p)
    {
        if (p.starts && r < 0) {
            r = p.r;
            head = p.head;
            tile = p.tile;
        }
        whole += p.starts && p.ends ? 1 : 0;
    }
    __device__ __forceinline__ void store(PagedJoin &j) const       // the whole warp
    {
        if ((threadIdx.x & 31) == 0) {
            j.r = r;
            j.head0 = head;
            j.tile = tile;
            j.whole = whole;
        }
        if (gone)
            atomicOr(&j.flags, kPagedGone);
    }
};

// The kernels add up their outputs to see whether all are finite (a sum that overflows has their
// rows looked at for nothing).
__device__ __forceinline__ bool pg_finite(float x) { return fabsf(x) < INFINITY; }
__device__ __forceinline__ float pg_total(const float4 &v) { return (v.x + v.y) + (v.z + v.w); }

// Whether any of four is an infinity or NaN.
__device__ __forceinline__ bool pg_odd(const float4 &v) { return v.x * 0.0f + v.y * 0.0f + v.z * 0.0f + v.w * 0.0f != 0.0f; }

__device__ __forceinline__ bool pg_all_nan(const float4 &v)
{
    return v.x != v.x && v.y != v.y && v.z != v.z && v.w != v.w;
}

// <(two 16-bit elements), (two more)> in fp32.
template <bool kF16> __device__ __forceinline__ float pg_dot2(uint32_t a, uint32_t b)
{
    if (kF16) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&a));
        const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&b));
        return x.x * y.x + x.y * y.y;
    }
    return __uint_as_float(a << 16) * __uint_as_float(b << 16) +
           __uint_as_float(a & 0xFFFF0000u) * __uint_as_float(b & 0xFFFF0000u);
}

// Four 16-bit elements as fp32.
template <bool kF16> __device__ __forceinline__ float4 pg_wide(const uint2 &w)
{
    if (kF16) {
        const float2 lo = __half22float2(*reinterpret_cast<const __half2 *>(&w.x));
        const float2 hi = __half22float2(*reinterpret_cast<const __half2 *>(&w.y));
        return make_float4(lo.x, lo.y, hi.x, hi.y);
    }
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xFFFF0000u));
}
template <bool kF16> __device__ __forceinline__ float4 pg_load4(const void *base, int64_t at)
{
    return pg_wide<kF16>(*reinterpret_cast<const uint2 *>(static_cast<const unsigned char *>(base) + 2 * at));
}

// A row's keys, and those that took part in its tile's products.
struct PagedAgain {
    int32_t r, pos;                     // request, position of the token
    int32_t k0, k1;                     // keys of the tile's steps
    int32_t len;
    bool gone;                          // some page may not be there
};

// One token (by its place in q) and query head: columns [c0, c1) of its output (and lse where c0 is 0),
// by the whole warp, if it sees a key that is not there, or if its output is not finite and a key that it
// does not see has values that are not.
template <bool kF16>
__device__ __forceinline__ void paged_row_again(const PagedArgs &a, const PagedAgain &w, int64_t token, int32_t head, int32_t c0,
                                                int32_t c1)
{
    const int lane = threadIdx.x & 31, col = lane * 4;
    const bool live = col < a.d, mine = live && col >= c0 && col < c1;
    const int32_t hi = !a.causal ? w.len : w.pos < 0 ? 0 : w.pos + 1;
    const int32_t lo = a.window && w.pos >= a.window ? w.pos - a.window + 1 : 0;
    const int64_t kvh = head / a.group * a.kv_head, q = token * a.q_token + head * a.q_head;
    const int64_t to = token * a.out_token + head * a.out_head + col;
    const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const bool odd = __any_sync(0xffffffffu, mine && pg_odd(pg_load4<kF16>(a.out, mine ? to : 0)));
    if (!odd && !w.gone)
        return;
    // (values that are not finite do not touch lse: the kernels' holds unless a page is missing)
    const bool wants = a.lse && w.gone && c0 == 0;
    bool again = false;
    float top = -INFINITY, sum = 0.0f;
    float4 acc = zero;
    // the first pass looks at the values of hidden keys (0 times them) and for pages, the second computes
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        const int32_t from = pass ? lo : w.k0, end = pass ? hi : w.k1;
#pragma unroll 1
        for (int32_t base = from; base < end; base += 32) {
            if (!pass && !w.gone && base >= lo && base < hi - 32) {
                base += (hi - base) / 32 * 32 - 32;     // (visible keys)
                continue;
            }
            const int32_t key = base + lane, e = key / a.page;
            const bool seen = key >= lo && key < hi;
            int64_t off = -1;           // of this lane's key
            if (key < end) {
                const int32_t page = a.tables[w.r * a.table_stride + e];
                if (page >= 0 && page < a.n_pages)
                    off = page * a.kv_page + (key - e * a.page) * a.kv_token + kvh;
            }
            float p = 0.0f;
            if (pass) {
                float x = 0.0f;         // its score
                const unsigned char *kr = static_cast<const unsigned char *>(a.k) + 2 * (off < 0 ? 0 : off);
                const unsigned char *qr = static_cast<const unsigned char *>(a.q) + 2 * q;
#pragma unroll 1
                for (int32_t c = 0; c < 2 * a.d; c += 16 * kAgainKeys) {
                    uint4 kw[kAgainKeys];           // (loads ahead of their use)
#pragma unroll
                    for (int i = 0; i < kAgainKeys; ++i)
                        kw[i] = c + 16 * i < 2 * a.d ? *reinterpret_cast<const uint4 *>(kr + c + 16 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < kAgainKeys; ++i) {
                        const uint4 qw = *reinterpret_cast<const uint4 *>(qr + (c + 16 * i < 2 * a.d ? c + 16 * i : 0));
                        x += pg_dot2<kF16>(qw.x, kw[i].x) + pg_dot2<kF16>(qw.y, kw[i].y) + pg_dot2<kF16>(qw.z, kw[i].z) +
                             pg_dot2<kF16>(qw.w, kw[i].w);
                    }
                }
                x = off >= 0 ? x * a.scale_log2 : -INFINITY;
                float most = fmaxf(x, top);
#pragma unroll 1
                for (int s = 16; s; s >>= 1)
                    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
                const float f = most == top ? 1.0f : pg_exp2(top - most);
                top = most;
                p = pg_exp2(x - (top == -INFINITY ? 0.0f : top));
                float all = p;
#pragma unroll 1
                for (int s = 16; s; s >>= 1)
                    all += __shfl_xor_sync(0xffffffffu, all, s);
                sum = sum * f + all;
                acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
                // (NaN from here on; not before lse is known)
                if (sum != sum || (!wants && __all_sync(0xffffffffu, !mine || pg_all_nan(acc))))
                    break;
            } else {
                again |= __any_sync(0xffffffffu, seen && off < 0);
                off = seen || !odd ? -1 : off;
            }
            if (!__any_sync(0xffffffffu, off >= 0))
                continue;
#pragma unroll 1
            for (int c = 0; c < 32; c += kAgainValues) {
                uint2 w[kAgainValues];
#pragma unroll
                for (int i = 0; i < kAgainValues; ++i) {
                    const int64_t o = __shfl_sync(0xffffffffu, off, c + i);
                    w[i] = *reinterpret_cast<const uint2 *>(static_cast<const unsigned char *>(a.v) +
                                                            2 * (o >= 0 && live ? o + col : 0));
                }
#pragma unroll
                for (int i = 0; i < kAgainValues; ++i) {
                    const bool in = __shfl_sync(0xffffffffu, off, c + i) >= 0 && live;
                    const float pc = __shfl_sync(0xffffffffu, p, c + i);
                    const float4 v = in ? pg_wide<kF16>(w[i]) : zero;
                    acc = make_float4(acc.x + pc * v.x, acc.y + pc * v.y, acc.z + pc * v.z, acc.w + pc * v.w);
                }
            }
        }
        if (!pass) {
            again |= __any_sync(0xffffffffu, pg_odd(acc));
            acc = zero;
            if (!again)
                return;
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (mine) {
        uint2 o;
        o.x = pg_pack<kF16>(acc.x * inv, acc.y * inv);
        o.y = pg_pack<kF16>(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2 *>(static_cast<unsigned char *>(a.out) + 2 * to) = o;
    }
    if (wants && lane == 0)
        a.lse[token * a.heads_q + head] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kPagedLn2;
}

// Rows of the tiles that unit's entry j tells of: the whole ones if `whole`, of which this warp
// takes rows first, first + stride, ..; and, if `cut`, the one behind them, which this unit starts
// and others end: columns [c0, c1) of the rows mine(token of the tile, head of the tile), after the
// join has stored them.
template <bool kF16, class Mine>
__device__ __forceinline__ void paged_unit_again(const PagedArgs &a, const PagedJoin &j, bool whole, bool cut, bool gone,
                                                 int32_t first, int32_t stride, int32_t c0, int32_t c1, const Mine &mine)
{
    int32_t r = j.r, group = j.head0, tile = j.tile;
#pragma unroll 1
    for (int32_t n = 0; n < j.whole + (cut ? 1 : 0); ++n) {
        PagedSeq s = paged_request(a, r, false);
        while (tile * static_cast<int64_t>(a.tok) >= s.m) {         // the next head group, or request
            tile = 0;
            if (++group == a.heads_kv * a.subs) {
                group = 0;
                if (++r >= a.n)
                    return;
                s = paged_request(a, r, false);
            }
        }
        const int32_t i0 = tile++ * a.tok;
        const bool last = n == j.whole;
        if (!last && !whole)
            continue;
        const int32_t kvh = group / a.subs, sub = group - kvh * a.subs;
        const int32_t tokens = s.m - i0 < a.tok ? s.m - i0 : a.tok;
        const int32_t heads = a.group - sub * a.sub < a.sub ? a.group - sub * a.sub : a.sub;
        const int32_t pos = s.L - s.m + i0, past = pos + tokens < 0 ? 0 : pos + tokens;
        PagedAgain w;
        w.r = r;
        w.len = s.L;
        w.gone = gone;
        // (the longer steps of the two kernels)
        w.k0 = a.window && pos >= a.window ? (pos - a.window + 1) / kPagedTileKeys * kPagedTileKeys : 0;
        w.k1 = a.causal ? (past + kPagedTileKeys - 1) / kPagedTileKeys * kPagedTileKeys : s.L;
        w.k1 = w.k1 < s.L ? w.k1 : s.L;
        int32_t at = first;             // rows until this warp's next
#pragma unroll 1
        for (int32_t t = 0; t < tokens; ++t)
#pragma unroll 1
            for (int32_t h = 0; h < heads; ++h, --at) {
                if (last ? !mine(t, h) : at != 0)
                    continue;
                at += stride;
                w.pos = pos + t;
                paged_row_again<kF16>(a, w, s.t0 + i0 + t, kvh * a.group + sub * a.sub + h, last ? c0 : 0,
                                      last ? c1 : kPagedMaxDim);
            }
    }
}

}  // namespace bsm
