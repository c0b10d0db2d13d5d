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
// cut tile are joined in unit order by a second launch (paged_join,
// paged_tile_join).  The line is never stored:
// the steps before tile i of a request have a closed form (floor sums), so a
// unit finds its place by bisection.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged.h"

namespace bsm {

// Quotients of counts that nearly always fit 32 bits (a 64-bit division costs
// several hundred cycles in the one warp that needs it).
__device__ __forceinline__ int64_t pg_div(int64_t a, int64_t b)
{
    if (((a | b) >> 32) == 0)
        return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// sum over i < n of (a i + b) / kStep, rounded down each: the sum of a i + b less that of
// the remainders, which repeat every P = kStep / gcd(a, kStep) terms and in a period
// are (b mod g), (b mod g) + g, ...; those of the last part of a period are added up one by
// one (fewer than P).  a n + b < 2^32.  Needs no division: three prompts under a window
// of 1024 take 152.5 us with Euclid's steps on the slope, 148 so.
template <int kStep> __device__ __forceinline__ int64_t floor_sum(uint32_t n, uint32_t a, uint32_t b)
{
    static_assert((kStep & (kStep - 1)) == 0, "steps are powers of two");
    const uint32_t low = a & (0u - a), g = low < kStep ? low : kStep, lg = 31 - __clz(g);
    const uint32_t P = static_cast<uint32_t>(kStep) >> lg;
    const uint32_t rest = n & (P - 1);
    uint32_t part = 0, x = b;
    for (uint32_t i = 0; i < rest; ++i, x += a)
        part += x & (kStep - 1);
    const uint64_t periods = (n - rest) * static_cast<uint64_t>(g) / kStep;
    const uint64_t mods = periods * (P * (b & (g - 1)) + kStep * (P - 1) / 2) + part;
    const uint64_t all = static_cast<uint64_t>(n) * (n - 1) / 2 * a + static_cast<uint64_t>(n) * b;
    return static_cast<int64_t>((all - mods) / kStep);
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

// Its tokens and keys.
__device__ __forceinline__ PagedSeq paged_request(const PagedArgs &a, int32_t r, bool report)
{
    PagedSeq s;
    const int32_t raw0 = a.starts[r], raw1 = a.starts[r + 1], rawL = a.lengths[r];
    const int64_t cap = static_cast<int64_t>(a.width) * a.page;
    const int32_t most = cap < kPagedMostKeys ? static_cast<int32_t>(cap) : kPagedMostKeys;
    const int32_t t0 = raw0 < 0 ? 0 : raw0 > a.n_tokens ? a.n_tokens : raw0;
    const int32_t t1 = raw1 < t0 ? t0 : raw1 > a.n_tokens ? a.n_tokens : raw1;
    const int32_t L = rawL < 0 ? 0 : rawL > most ? most : rawL;
    if (report && (t0 != raw0 || t1 != raw1 || L != rawL))
        atomicOr(a.status, BSM_DEV_BOUNDS);
    s.t0 = t0;
    s.m = t1 - t0;
    s.L = L;
    return s;
}

template <int kStep> struct PagedLine {
    const PagedArgs &a;
    __device__ explicit PagedLine(const PagedArgs &args) : a(args) {}

    __device__ __forceinline__ PagedRange range(const PagedSeq &s, int32_t i) const
    {
        PagedRange r{0, s.L};
        if (a.causal) {
            const int32_t first = s.L - s.m + i * a.tok, left = s.m - i * a.tok;
            r.hi = first + (left < a.tok ? left : a.tok);
            r.hi = r.hi < 0 ? 0 : r.hi;
            if (a.window && first >= a.window)
                r.lo = first - a.window + 1;
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
        int32_t tail = 0;
        if (i == s.tiles) {             // the last tile may be short
            --i;
            tail = steps_of(range(s, i));
        }
        const int32_t base = s.L - s.m;
        const uint32_t tok = static_cast<uint32_t>(a.tok);
        // tiles whose last token lies before the first key see none
        const uint32_t none = base < 0 ? (0u - static_cast<uint32_t>(base)) / tok : 0u;
        if (static_cast<uint32_t>(i) <= none)
            return static_cast<int64_t>(i) + tail;
        int64_t n = tail + static_cast<int64_t>(none) +
                    floor_sum<kStep>(i - none, tok, static_cast<uint32_t>(base) + (none + 1) * tok + kStep - 1);
        if (a.window) {
            // whole steps that lie left of a tile's window: of tiles j and on
            uint32_t j = none;
            if (base < a.window) {
                const uint32_t past = (static_cast<uint32_t>(a.window) - 1u - static_cast<uint32_t>(base)) / tok + 1;
                j = j < past ? past : j;
            }
            if (j < static_cast<uint32_t>(i))
                n -= floor_sum<kStep>(i - j, tok, static_cast<uint32_t>(base) + j * tok - static_cast<uint32_t>(a.window) + 1u);
        }
        return n;
    }

    // known >= 0: the request's steps, all head groups
    __device__ PagedSeq seq(int32_t r, bool report, int64_t known = -1) const
    {
        PagedSeq s = paged_request(a, r, report);
        if (s.m == 0)
            return s;
        s.tiles = (s.m + a.tok - 1) / a.tok;
        s.steps = known >= 0 ? pg_div(known, static_cast<int64_t>(a.heads_kv) * a.subs) : before(s, s.tiles);
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

// How the line is cut: `units` ranges of at least min_steps steps (the line may be
// shorter: one range); unit u begins at W u / units.
struct PagedCut {
    int64_t W, q;
    int32_t units, rem;
    __device__ PagedCut(const PagedArgs &a, int64_t steps) : W(steps)
    {
        const int64_t most = pg_div(steps, a.min_steps);
        units = most >= a.units ? a.units : most < 1 ? 1 : static_cast<int32_t>(most);
        q = pg_div(W, units);
        rem = static_cast<int32_t>(W - q * units);
    }
    __device__ __forceinline__ int64_t begin(int32_t u) const
    {
        return q * u + static_cast<uint32_t>(rem) * static_cast<uint32_t>(u) / static_cast<uint32_t>(units);
    }
    // the unit that takes step x: a guess in fp32, put right
    __device__ __forceinline__ int32_t owner(int64_t x) const
    {
        int32_t u = static_cast<int32_t>(static_cast<float>(x) * static_cast<float>(units) / static_cast<float>(W));
        u = u < 0 ? 0 : u >= units ? units - 1 : u;
        while (u + 1 < units && begin(u + 1) <= x)
            ++u;
        while (u > 0 && begin(u) > x)
            --u;
        return u;
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
        // the whole warp searches: 32 candidates at once
        const int lane = threadIdx.x & 31;
        constexpr int kEach = kThreads / 32;
        int lo = (__popc(__ballot_sync(0xffffffffu, p.pre[lane * kEach] <= x)) - 1) * kEach;
        lo += __popc(__ballot_sync(0xffffffffu, lane < kEach && p.pre[lo + lane] <= x)) - 1;
        int64_t o = x - p.pre[lo];
        r = lo * ((l.a.n + kThreads - 1) / kThreads) - 1;
        int64_t all = 0;
        do {                                    // (the line's end is past x: some request holds it)
            o -= all;
            // (a thread's sum over one request is that request's steps)
            const int64_t known = l.a.n <= kThreads ? p.pre[r + 2] - p.pre[r + 1] : -1;
            s = line.seq(++r, false, known);
            all = line.all_steps(s);
        } while (o >= all && r + 1 < l.a.n);
        head = static_cast<int32_t>(pg_div(o, s.steps));
        o -= head * s.steps;
        int32_t left = s.tiles;
        int64_t first = 0;
        while (left > 1) {
            const int32_t each = (left + 31) / 32, mine = lane * each;
            const int64_t f = mine < left ? line.before(s, tile + mine) : 0;
            const int k = 31 - __clz(__ballot_sync(0xffffffffu, mine < left && f <= o));
            first = __shfl_sync(0xffffffffu, f, k);
            tile += k * each;
            left = each < left - k * each ? each : left - k * each;
            if (each <= 8) {                    // the rest one by one
                for (int32_t n; left > 1 && first + (n = line.steps_of(line.range(s, tile))) <= o; --left) {
                    first += n;
                    ++tile;
                }
                break;
            }
        }
        at = static_cast<int32_t>(o - first);
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

// Launches a kernel that may start while the one before it in the stream ends
// (it waits for that one's writes itself).
template <typename... Ks, typename... As>
inline int launch_early(void (*kernel)(Ks...), dim3 grid, int threads, size_t smem, cudaStream_t st, const As &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return static_cast<int>(cudaLaunchKernelEx(&cfg, kernel, args...));
}

__device__ __forceinline__ uint32_t pg_saddr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ float pg_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Probabilities are held as 2^(s - m + shift), s at most `lag` above the reference m: f16 would
// lose those below 2^-14 of the largest, so its exponents start at the top of its range (its
// values are below 2^16, far from where fp32 sums end); bf16 has values up to the end of
// that range, so its probabilities stay at 1 or less.
template <bool kF16> __device__ __forceinline__ constexpr float pg_shift(float lag) { return (kF16 ? 14.0f : 0.0f) - lag; }

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
