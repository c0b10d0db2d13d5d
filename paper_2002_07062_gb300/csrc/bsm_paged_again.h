// bsm_paged_again.h -- rows of paged attention computed once more, from the
// definition, where the tile kernel's answer does not hold.
//
//   o = sum p_j v_j / sum p_j over the visible keys whose pages are there, in fp32
//
// The tile kernel's copies fill a key whose page is not there with zeros, and its
// products cannot leave a single key out, so such a key would enter with score 0.
// Its producer notes that it met one and which tiles it went through; the join launch,
// which follows anyway, takes their rows that see one again: a warp a row, four
// columns a lane, 32 keys at a time.  Where all pages are there it reads a flag a unit.
// (Masking such keys in the tile kernel's own softmax cost every call 1 to 4 %.  The code is
// kept short because its size costs too: with the walk along the work line in it, 80 KB
// instead of 23, a chunk of 2048 tokens over 6100 keys took 163 us instead of 156.)
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged_dev.h"

namespace bsm {

constexpr float kPagedLn2 = 0.6931471805599453f;

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

// Four 16-bit elements as fp32.
template <bool kF16> __device__ __forceinline__ float4 pg_load4(const void *base, int64_t at)
{
    const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const unsigned char *>(base) + 2 * at);
    if (kF16) {
        const float2 lo = __half22float2(*reinterpret_cast<const __half2 *>(&w.x));
        const float2 hi = __half22float2(*reinterpret_cast<const __half2 *>(&w.y));
        return make_float4(lo.x, lo.y, hi.x, hi.y);
    }
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xFFFF0000u));
}

__device__ __forceinline__ float pg_warp_sum(float x)
{
#pragma unroll 1
    for (int w = 16; w; w >>= 1)
        x += __shfl_xor_sync(0xffffffffu, x, w);
    return x;
}

// A token at position pos of request r and one query head: columns [c0, c1) of its output (and
// lse where c0 is 0), by the whole warp.  Nothing is done where every key that it sees is there.
template <bool kF16>
__device__ __forceinline__ void paged_row_again(const PagedArgs &a, int32_t r, int32_t len, int32_t pos, int64_t token,
                                                int32_t head, int32_t c0, int32_t c1)
{
    const int lane = threadIdx.x & 31, col = lane * 4;
    const bool live = col < a.d;
    const int32_t hi = !a.causal ? len : pos < 0 ? 0 : pos + 1;
    const int32_t lo = a.window && pos >= a.window ? pos - a.window + 1 : 0;
    const int64_t kvh = head / a.group * a.kv_head;
    const float4 q = live ? pg_load4<kF16>(a.q, token * a.q_token + head * a.q_head + col) : make_float4(0, 0, 0, 0);
    bool again = false;
    float top = -INFINITY, sum = 0.0f;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // the first pass looks for a key that is not there, the second computes
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
        for (int32_t base = lo; base < hi; base += 32) {
            const int32_t key = base + lane, e = key / a.page;
            int64_t off = -1;           // of this lane's key
            if (key < hi) {
                const int32_t page = a.tables[r * a.table_stride + e];
                if (page >= 0 && page < a.n_pages)
                    off = page * a.kv_page + (key - e * a.page) * a.kv_token + kvh;
            }
            if (pass == 0) {
                again = __any_sync(0xffffffffu, key < hi && off < 0);
                if (again)
                    break;
                continue;
            }
            float x = -INFINITY;        // its score
#pragma unroll 1
            for (int c = 0; c < 32; ++c) {
                const int64_t o = __shfl_sync(0xffffffffu, off, c);
                if (o < 0)
                    continue;
                const float4 k = live ? pg_load4<kF16>(a.k, o + col) : make_float4(0, 0, 0, 0);
                const float dot = pg_warp_sum(q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w);
                x = lane == c ? dot * a.scale_log2 : x;
            }
            float most = fmaxf(x, top);
#pragma unroll 1
            for (int w = 16; w; w >>= 1)
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, w));
            const float f = most == top ? 1.0f : pg_exp2(top - most);
            top = most;
            const float p = pg_exp2(x - (top == -INFINITY ? 0.0f : top));
            sum = sum * f + pg_warp_sum(p);
            acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
#pragma unroll 1
            for (int c = 0; c < 32; ++c) {
                const int64_t o = __shfl_sync(0xffffffffu, off, c);
                const float pc = __shfl_sync(0xffffffffu, p, c);
                if (o < 0 || !live)
                    continue;
                const float4 v = pg_load4<kF16>(a.v, o + col);
                acc = make_float4(acc.x + pc * v.x, acc.y + pc * v.y, acc.z + pc * v.z, acc.w + pc * v.w);
            }
            if (sum != sum)             // NaN from here on
                break;
        }
        if (!again)
            return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (col >= c0 && col < c1 && live) {
        uint2 w;
        w.x = pg_pack<kF16>(acc.x * inv, acc.y * inv);
        w.y = pg_pack<kF16>(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2 *>(static_cast<unsigned char *>(a.out) + 2 * (token * a.out_token + head * a.out_head + col)) = w;
    }
    if (a.lse && c0 == 0 && lane == 0)
        a.lse[token * a.heads_q + head] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kPagedLn2;
}

// Rows of the tiles that unit's entry j tells of: the whole ones if `whole`, of which this warp
// takes rows first, first + stride, ..; and, if `cut`, the one behind them, which this unit starts
// and others end: columns [c0, c1) of the rows mine(token of the tile, head of the tile), after the
// join has stored them.
template <bool kF16, class Mine>
__device__ __forceinline__ void paged_unit_again(const PagedArgs &a, const PagedJoin &j, bool whole, bool cut, int32_t first,
                                                 int32_t stride, int32_t c0, int32_t c1, const Mine &mine)
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
        int32_t at = first;             // rows until this warp's next
#pragma unroll 1
        for (int32_t t = 0; t < tokens; ++t)
#pragma unroll 1
            for (int32_t h = 0; h < heads; ++h, --at) {
                if (last ? !mine(t, h) : at != 0)
                    continue;
                at += stride;
                paged_row_again<kF16>(a, r, s.L, s.L - s.m + i0 + t, s.t0 + i0 + t, kvh * a.group + sub * a.sub + h,
                                      last ? c0 : 0, last ? c1 : kPagedMaxDim);
            }
    }
}

}  // namespace bsm
