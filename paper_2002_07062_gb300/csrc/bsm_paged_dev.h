// bsm_paged_dev.h -- device code shared by the kernels of paged attention: how
// the batch's work is laid out on a line and cut into equal ranges, and small
// PTX wrappers.
//
// Work is counted in key steps: a tile (a few tokens of one request times the
// query heads that share a key/value head) against `step` consecutive keys.
// All steps of all tiles, request by request, head by head, tile by tile, form
// a line of W steps; unit u of U (a warp or a CTA) takes steps
// [W u / U, W (u + 1) / U).  Every unit gets the same amount whatever the
// lengths are, and a tile is cut at most where two units meet; the parts of a
// cut tile are joined by paged_join in unit order.  The line is never stored:
// the steps before tile i of a request have a closed form (floor sums), so a
// unit finds its place by bisection.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged.h"

namespace bsm {

// sum over i < n of (a i + b) / m, rounded down each (Euclid on the slope).
__device__ __forceinline__ int64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b)
{
    uint64_t ans = 0;
    while (n > 0) {
        if (a >= m) {
            ans += static_cast<uint64_t>(n) * (n - 1) / 2 * (a / m);
            a %= m;
        }
        if (b >= m) {
            ans += static_cast<uint64_t>(n) * (b / m);
            b %= m;
        }
        const uint64_t y = static_cast<uint64_t>(a) * n + b;
        if (y < m)
            break;
        n = static_cast<uint32_t>(y / m);
        b = static_cast<uint32_t>(y % m);
        const uint32_t t = m;
        m = a;
        a = t;
    }
    return static_cast<int64_t>(ans);
}

// One request as the kernels see it: lengths and offsets outside the buffers
// are cut to them (and reported), so that nothing below can leave a buffer.
struct PagedSeq {
    int32_t t0 = 0, m = 0, L = 0;       // first token, tokens, keys
    int32_t tiles = 0;
    int64_t steps = 0;                  // key steps of all tiles of one head group
};

// Keys [lo, hi) that any token of a tile sees.
struct PagedRange {
    int32_t lo, hi;
};

template <int kStep> struct PagedLine {
    const PagedArgs &a;
    __device__ explicit PagedLine(const PagedArgs &args) : a(args) {}

    __device__ __forceinline__ PagedRange range(const PagedSeq &s, int32_t i) const
    {
        PagedRange r{0, s.L};
        if (a.causal) {
            const int32_t end = (i + 1) * a.tok < s.m ? (i + 1) * a.tok : s.m;
            r.hi = s.L - s.m + end;
            r.hi = r.hi < 0 ? 0 : r.hi;
            if (a.window) {
                const int64_t lo = static_cast<int64_t>(s.L) - s.m + i * a.tok - a.window + 1;
                r.lo = lo < 0 ? 0 : static_cast<int32_t>(lo);
                r.lo = r.lo < r.hi ? r.lo : r.hi;
            }
        }
        return r;
    }

    // key steps of a tile; one that sees no key still takes one (it has to be written)
    __device__ __forceinline__ int32_t steps_of(const PagedRange &r) const
    {
        const int32_t n = static_cast<int32_t>((static_cast<uint32_t>(r.hi) + kStep - 1) / kStep) - r.lo / kStep;
        return n > 1 ? n : 1;
    }

    // steps of tiles 0 .. i-1 of one head group
    __device__ int64_t before(const PagedSeq &s, int32_t i) const
    {
        if (i <= 0)
            return 0;
        if (!a.causal)
            return static_cast<int64_t>(i) * steps_of(PagedRange{0, s.L});
        int64_t tail = 0;
        if (i == s.tiles) {             // the last tile may be short
            --i;
            tail = steps_of(range(s, i));
        }
        const int64_t base = static_cast<int64_t>(s.L) - s.m;
        // tiles whose last token lies before the first key see none
        int32_t none = 0;
        if (base < 0)
            none = static_cast<int32_t>(-base / a.tok);
        if (i <= none)
            return i + tail;
        int64_t n = none + floor_sum(i - none, kStep, a.tok, static_cast<uint32_t>(base + static_cast<int64_t>(none + 1) * a.tok + kStep - 1));
        if (a.window) {
            // whole steps that lie left of a tile's window
            const int64_t past = static_cast<int64_t>(a.window) - 1 - base;
            int64_t j = past < 0 ? 0 : past / a.tok + 1;
            j = j < none ? none : j;
            if (j < i)
                n -= floor_sum(static_cast<uint32_t>(i - j), kStep, a.tok, static_cast<uint32_t>(base + j * a.tok - a.window + 1));
        }
        return n + tail;
    }

    __device__ PagedSeq seq(int32_t r, bool report) const
    {
        PagedSeq s;
        const int32_t raw0 = a.starts[r], raw1 = a.starts[r + 1], rawL = a.lengths[r];
        const int64_t cap = static_cast<int64_t>(a.width) * a.page;
        const int32_t most = cap < INT32_MAX ? static_cast<int32_t>(cap) : INT32_MAX;
        const int32_t t0 = raw0 < 0 ? 0 : raw0 > a.n_tokens ? a.n_tokens : raw0;
        const int32_t t1 = raw1 < t0 ? t0 : raw1 > a.n_tokens ? a.n_tokens : raw1;
        const int32_t L = rawL < 0 ? 0 : rawL > most ? most : rawL;
        if (report && (t0 != raw0 || t1 != raw1 || L != rawL))
            atomicOr(a.status, BSM_DEV_BOUNDS);
        s.t0 = t0;
        s.m = t1 - t0;
        s.L = L;
        const int64_t rows = static_cast<int64_t>(s.m) * a.group;
        if (s.m == 0 || rows <= a.rows_min || rows > a.rows_max) {
            s.m = 0;
            return s;
        }
        s.tiles = (s.m + a.tok - 1) / a.tok;
        s.steps = before(s, s.tiles);
        return s;
    }

    __device__ __forceinline__ int64_t all_steps(const PagedSeq &s) const
    {
        return s.steps * (static_cast<int64_t>(a.heads_kv) * a.subs);
    }
};

// Steps before the requests of every thread of the block: thread i holds those
// of requests [i * per, (i + 1) * per).
template <int kThreads> struct PagedPrefix {
    int64_t pre[kThreads + 1];
    int64_t warp[kThreads / 32];
};

// Fills p (all threads of the block; ends with __syncthreads).
template <int kStep, int kThreads>
__device__ void paged_prefix(const PagedLine<kStep> &line, PagedPrefix<kThreads> &p, bool report)
{
    const PagedArgs &a = line.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t per = (a.n + kThreads - 1) / kThreads;
    int64_t sum = 0;
    if (tid < kThreads) {
        for (int32_t i = 0; i < per; ++i) {
            const int64_t r = static_cast<int64_t>(tid) * per + i;
            if (r < a.n)
                sum += line.all_steps(line.seq(static_cast<int32_t>(r), report));
        }
        int64_t inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
            inc += lane >= o ? v : 0;
        }
        if (lane == 31)
            p.warp[warp] = inc;
        p.pre[tid] = inc - sum;         // within the warp
    }
    __syncthreads();
    if (tid < kThreads) {
        int64_t base = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            base += w < warp ? p.warp[w] : 0;
            all += p.warp[w];
        }
        p.pre[tid] += base;
        if (tid == 0)
            p.pre[kThreads] = all;
    }
    __syncthreads();
}

// How the line is cut: `units` ranges of at least min_steps steps.
struct PagedCut {
    int64_t W;
    int32_t units;
    __device__ PagedCut(const PagedArgs &a, int64_t steps) : W(steps)
    {
        const int64_t u = steps / a.min_steps;
        units = u >= a.units ? a.units : u < 1 ? 1 : static_cast<int32_t>(u);
    }
    __device__ __forceinline__ int64_t begin(int32_t u) const { return W * u / units; }
    // the unit that takes step x
    __device__ __forceinline__ int32_t owner(int64_t x) const
    {
        return static_cast<int32_t>(((x + 1) * units - 1) / W);
    }
};

// A walk along the line: the piece of a tile that comes next.
struct PagedPiece {
    int32_t r;                          // request
    int32_t head;                       // head group: kv head * subs + sub
    int32_t tile;
    PagedRange keys;                    // keys the tile sees
    int32_t first, steps;               // first step (of kStep keys, from key 0), steps of this piece
    bool starts, ends;                  // the piece holds the tile's first, last step
    int64_t tile_end;                   // end of the tile on the line
};

// The closed form finds the range's first tile; from there the walk counts on.
template <int kStep> struct PagedWalk {
    const PagedLine<kStep> &line;
    int64_t x, end;                     // next step, end of the unit's range
    int32_t r = 0, head = 0, tile = 0, at = 0;
    PagedSeq s;

    template <int kThreads>
    __device__ PagedWalk(const PagedLine<kStep> &l, const PagedPrefix<kThreads> &p, int64_t begin, int64_t end_)
        : line(l), x(begin), end(end_)
    {
        if (x >= end)
            return;
        int lo = 0, hi = kThreads;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.pre[mid] <= x)
                lo = mid;
            else
                hi = mid;
        }
        int64_t o = x - p.pre[lo];
        r = lo * ((l.a.n + kThreads - 1) / kThreads);
        s = l.seq(r, false);
        while (o >= line.all_steps(s) && r + 1 < l.a.n) {       // (the line's end is past x: some request holds it)
            o -= line.all_steps(s);
            s = line.seq(++r, false);
        }
        head = static_cast<int32_t>(o / s.steps);
        o -= head * s.steps;
        int32_t t0 = 0, t1 = s.tiles;
        while (t1 - t0 > 1) {
            const int32_t mid = (t0 + t1) >> 1;
            if (line.before(s, mid) <= o)
                t0 = mid;
            else
                t1 = mid;
        }
        tile = t0;
        at = static_cast<int32_t>(o - line.before(s, t0));
    }

    __device__ bool next(PagedPiece &pc)
    {
        if (x >= end)
            return false;
        if (tile == s.tiles) {
            tile = 0;
            if (++head == line.a.heads_kv * line.a.subs) {
                head = 0;
                do {
                    if (++r >= line.a.n)
                        return false;
                    s = line.seq(r, false);
                } while (s.m == 0);
            }
        }
        pc.r = r;
        pc.head = head;
        pc.tile = tile;
        pc.keys = line.range(s, tile);
        const int32_t n = line.steps_of(pc.keys);
        const int64_t left = end - x;
        pc.tile_end = x + (n - at);
        pc.steps = left < n - at ? static_cast<int32_t>(left) : n - at;
        pc.first = pc.keys.lo / kStep + at;
        pc.starts = at == 0;
        pc.ends = at + pc.steps == n;
        x += pc.steps;
        at = 0;
        ++tile;
        return true;
    }
};

__device__ __forceinline__ uint32_t pg_saddr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ float pg_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Probabilities are held as 2^(s - m + shift): f16 would lose those below
// 2^-14 of the largest, so its exponents start at the top of its range.
template <bool kF16> __device__ __forceinline__ constexpr float pg_shift(float lag) { return kF16 ? 14.0f - lag : 0.0f; }

template <bool kF16> __device__ __forceinline__ uint32_t pg_pack(float lo, float hi)
{
    uint32_t r;
    if (kF16)
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace bsm
