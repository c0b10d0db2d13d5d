// bsm_paged_rows.cu -- attention of a few new tokens over a paged cache:
// tiles of at most 16 rows (tokens times the query heads that share a
// key/value head), the keys split over every warp of the device.
//
//   s = scale q k^T,  p = exp(s - m),  o = sum p v / sum p   (m a running maximum)
//
// Bound: the cache's bytes.  A row of 16 query heads costs one key 4 D
// operations a byte pair, far below what mma.sync gives, so the kernel is
// built for loads: every warp is on its own, with its own range of the work,
// its own three stages of 16 keys (8 KiB of K and V at D = 128) filled by
// 16-byte asynchronous copies, its own running maximum and sum; no barrier of
// the block after the work is laid out.  24 stages an SM keep 128 to 192 KiB
// in flight.  GB300: 128 requests of up to 8192 keys, 32/8 heads of 128, 2.25 GB:
// 350 to 364 us, 0.91 to 0.95 of the copy rate; one request of 2000 keys 14.7 us.
#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged_again.h"
#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kRowThreads = kPagedWarps * 32;
constexpr int kRowStages = 3;
constexpr int kStageBytes = 8192;                       // of one warp: K and V of a step

// Tiles of 32 rows (two 16-row blocks a warp) spilled and ran at 0.45 of the copy
// rate; such batches go to the tile kernel.
// keys of a step: 16 rows of 256 bytes, or 32 of 128
template <int DP> struct RowShape {
    static constexpr int kKeys = DP == 128 ? 16 : 32;
    static constexpr int kRowBytes = DP * 2;
    static constexpr int kChunks = DP / 8;              // 16-byte pieces of a row
};

struct RowSmem {
    PagedPrefix<kRowThreads> prefix;
};
constexpr int kRowHeader = 4096;
static_assert(sizeof(RowSmem) <= kRowHeader, "row header");
constexpr int kRowSmem = kRowHeader + kPagedWarps * kRowStages * kStageBytes;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

// d += a b: 16 x 16 times 16 x 8, fp32 sums
template <bool kF16> __device__ __forceinline__ void mma16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    if (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                     "{%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, "
                     "%9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The sum over the parts of a row: with M the largest of their references m_i,
// o = sum 2^(m_i - M) o_i, l = sum 2^(m_i - M) l_i.  A lane has four columns.
struct RowSum {
    float top = -INFINITY, sum = 0.0f;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __device__ __forceinline__ void add(const float2 &ml, const float4 &v)
    {
        const float f = pg_exp2(ml.x - (top == -INFINITY ? 0.0f : top));
        sum += f * ml.y;
        acc.x += f * v.x;
        acc.y += f * v.y;
        acc.z += f * v.z;
        acc.w += f * v.w;
    }
    template <bool kF16>
    __device__ __forceinline__ void store(const PagedArgs &a, int64_t token, int32_t head, int lane, float &odd) const
    {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (lane * 4 < a.d) {
            uint2 w;
            w.x = pg_pack<kF16>(acc.x * inv, acc.y * inv);
            w.y = pg_pack<kF16>(acc.z * inv, acc.w * inv);
            odd += pg_total(acc);
            *reinterpret_cast<uint2 *>(static_cast<unsigned char *>(a.out) +
                                       2 * (token * a.out_token + head * a.out_head + lane * 4)) = w;
        }
        if (a.lse && lane == 0)
            a.lse[token * a.heads_q + head] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kPagedLn2;
    }
};

// Where the rows of a tile come from and go to.
struct RowTile {
    int32_t token, head, tokens, heads; // first token, first query head, tokens, heads
    int32_t pos;                        // position of the first token
};

__device__ __forceinline__ RowTile row_tile(const PagedArgs &a, const PagedSeq &s, const PagedPiece &p)
{
    RowTile t;
    const int32_t kvh = p.head / a.subs, sub = p.head - kvh * a.subs;
    t.token = s.t0 + p.tile * a.tok;
    t.tokens = s.m - p.tile * a.tok < a.tok ? s.m - p.tile * a.tok : a.tok;
    t.head = kvh * a.group + sub * a.sub;
    t.heads = a.group - sub * a.sub < a.sub ? a.group - sub * a.sub : a.sub;
    t.pos = s.L - s.m + p.tile * a.tok;
    return t;
}

// DP: the head size padded to 64 or 128.
template <int DP, bool kF16>
__global__ void __launch_bounds__(kRowThreads, 1) paged_rows(const PagedArgs a)
{
    using Shape = RowShape<DP>;
    constexpr int kKeys = Shape::kKeys, kChunks = Shape::kChunks, kRB = Shape::kRowBytes;
    constexpr int kSubs = kKeys / 16;
    constexpr int kHalf = kKeys * kRB;                  // V behind K in a stage
    static_assert(2 * kHalf == kStageBytes, "stage");
    extern __shared__ __align__(128) unsigned char raw[];
    RowSmem &sm = *reinterpret_cast<RowSmem *>(raw);
    const int lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    // neighbouring units on different SMs: a small batch spreads over the device
    const int32_t unit = warp * gridDim.x + blockIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    if (lane == 0) {
        a.join[unit].count = 0;
        a.join[unit].flags = 0;
    }
    const PagedLine<kKeys> line(a);
    paged_prefix<kKeys, kRowThreads>(line, sm.prefix, blockIdx.x == 0);
    const int64_t W = sm.prefix.pre[kRowThreads];
    const PagedCut cut(a, W);
    if (W == 0 || unit >= cut.units)
        return;
    const int64_t begin = cut.begin(unit), end = cut.begin(unit + 1);
    const int32_t total = static_cast<int32_t>(end - begin);
    PagedWalk<kKeys> fetch(line, sm.prefix, begin, end), walk = fetch;

    const uint32_t stages = pg_saddr(raw) + kRowHeader + warp * (kRowStages * kStageBytes);
    const unsigned char *kbase = static_cast<const unsigned char *>(a.k), *vbase = static_cast<const unsigned char *>(a.v);

    // ---- loads: one step of kKeys keys at a time, in the order of the walk
    PagedPiece fp{};
    int32_t fleft = 0, fstep = 0;       // steps left of the piece being fetched, its next step
    int64_t fhead = 0;
    // byte offset of this lane's key of the next step (-1: none), read one step ahead
    auto key_offset = [&]() -> int64_t {
        const int32_t key = fstep * kKeys + (lane & (kKeys - 1));
        if (key < fp.keys.lo || key >= fp.keys.hi)
            return -1;
        const int32_t e = key / a.page;
        const int32_t page = a.tables[fp.r * a.table_stride + e];
        if (page < 0 || page >= a.n_pages) {
            atomicOr(a.status, BSM_DEV_BOUNDS);
            return -1;
        }
        return 2 * (page * a.kv_page + (key - e * a.page) * a.kv_token + fhead);
    };
    auto advance = [&]() {
        if (fleft == 0) {
            if (!fetch.next(fp))
                return;
            fleft = fp.steps;
            fstep = fp.first;
            fhead = (fp.head / a.subs) * a.kv_head;
        }
    };
    int64_t off = -1;
    int32_t issued = 0;
    uint32_t there[kRowStages];         // of the stages in order: the keys of the tile that have a page
    advance();
    off = key_offset();
    auto issue = [&]() {
#pragma unroll
        for (int i = 0; i + 1 < kRowStages; ++i)
            there[i] = there[i + 1];
        there[kRowStages - 1] = __ballot_sync(0xffffffffu, off >= 0);
        if (issued < total) {
            const uint32_t st = stages + (issued % kRowStages) * kStageBytes;
            constexpr int kRowsAtOnce = 32 / kChunks;
            const int c = lane % kChunks;
#pragma unroll
            for (int i = 0; i < kKeys / kRowsAtOnce; ++i) {
                const int row = i * kRowsAtOnce + lane / kChunks;
                const int64_t o = __shfl_sync(0xffffffffu, off, row);
                const bool in = o >= 0 && c * 8 < a.d;
                const int64_t at = in ? o + c * 16 : 0;
                const uint32_t dst = st + row * kRB + ((c ^ (row & 7)) << 4);
                cp_async16(dst, kbase + at, in ? 16u : 0u);
                cp_async16(dst + kHalf, vbase + at, in ? 16u : 0u);
            }
            ++issued;
            --fleft;
            ++fstep;
            if (issued < total) {
                advance();
                off = key_offset();
            }
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < kRowStages; ++i)
        issue();

    // ---- one piece after another
    PagedPiece p{};
    PagedSeen passed;
    float odd = 0.0f;                   // sum of the outputs: not finite if one of them is not
    int32_t done = 0;
    while (walk.next(p)) {
        passed.note(p);
        const RowTile t = row_tile(a, walk.s, p);
        const int32_t rows = t.tokens * a.sub;
        // this lane's rows: lane / 4 and lane / 4 + 8
        int32_t lo[2], hi[2];
        uint32_t q[DP / 16][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = i * 8 + lane / 4;
            const int32_t tt = row / a.sub, h = row - tt * a.sub;
            const bool live = row < rows && h < t.heads;
            const int32_t pos = t.pos + tt;
            hi[i] = !live ? 0 : a.causal ? (pos + 1 < p.keys.hi ? pos + 1 : p.keys.hi) : p.keys.hi;
            lo[i] = a.window && pos >= a.window ? pos - a.window + 1 : 0;
            const uint32_t *src = reinterpret_cast<const uint32_t *>(
                static_cast<const unsigned char *>(a.q) + 2 * ((t.token + tt) * a.q_token + (t.head + h) * a.q_head));
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                const int d0 = k * 16 + (lane & 3) * 2;
                q[k][i] = live && d0 < a.d ? src[d0 / 2] : 0u;
                q[k][i + 2] = live && d0 + 8 < a.d ? src[d0 / 2 + 4] : 0u;
            }
        }
        float o[DP / 8][4];
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
            o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
        for (int32_t st = 0; st < p.steps; ++st) {
            cp_wait<kRowStages - 1>();
            __syncwarp();
            const uint32_t kst = stages + (done % kRowStages) * kStageBytes;
#pragma unroll
            for (int sb = 0; sb < kSubs; ++sb) {
                const int32_t key0 = (p.first + st) * kKeys + sb * 16;
                float s[2][4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[0][j] = s[1][j] = 0.0f;
                // keys 0-7 / 8-15 and halves of 8 columns: matrices of lanes 0-7, 8-15, 16-23, 24-31
                const int krow = sb * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    uint32_t b[4];
                    ldsm4(kst + krow * kRB + (((2 * k + ((lane >> 3) & 1)) ^ (krow & 7)) << 4), b);
                    mma16<kF16>(s[0], q[k], b[0], b[1]);
                    mma16<kF16>(s[1], q[k], b[2], b[3]);
                }
                const uint32_t have = there[0] >> (sb * 16 + (lane & 3) * 2);
                uint32_t pa[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x[4];
                    float top = m[i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int32_t key = key0 + (j >> 1) * 8 + (lane & 3) * 2 + (j & 1);
                        const float v = s[j >> 1][i * 2 + (j & 1)] * a.scale_log2;
                        const bool in = key >= lo[i] && key < hi[i] && (have >> ((j >> 1) * 8 + (j & 1)) & 1u);
                        x[j] = in ? v : -INFINITY;
                        top = fmaxf(top, x[j]);
                    }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // a row that has seen no key yet: exponents against 0, all of them -inf
                    const float ref = top == -INFINITY ? 0.0f : top - pg_shift<kF16>(0.0f);
                    if (__any_sync(0xffffffffu, top != m[i])) {
                        const float f = top == m[i] ? 1.0f : pg_exp2(m[i] - top);
                        l[i] *= f;
#pragma unroll
                        for (int n = 0; n < DP / 8; ++n) {
                            o[n][2 * i] *= f;
                            o[n][2 * i + 1] *= f;
                        }
                    }
                    m[i] = top;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = pg_exp2(x[j] - ref);
                        l[i] += x[j];
                    }
                    pa[i] = pg_pack<kF16>(x[0], x[1]);
                    pa[i + 2] = pg_pack<kF16>(x[2], x[3]);
                }
                const int vrow = sb * 16 + (lane & 15);
#pragma unroll
                for (int n = 0; n < DP / 16; ++n) {
                    uint32_t b[4];
                    ldsm4t(kst + kHalf + vrow * kRB + (((2 * n + (lane >> 4)) ^ (vrow & 7)) << 4), b);
                    mma16<kF16>(o[2 * n], pa, b[0], b[1]);
                    mma16<kF16>(o[2 * n + 1], pa, b[2], b[3]);
                }
            }
            __syncwarp();
            ++done;
            issue();
        }
        // ---- the tile's output, or this unit's part of it
        const bool whole = p.starts && p.ends;
        const int64_t slot = static_cast<int64_t>(2 * unit + (p.starts ? 1 : 0)) * kPagedRowTile;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float sum = l[i];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            const float ref = m[i] - pg_shift<kF16>(0.0f);
            const int row = i * 8 + lane / 4;
            const int32_t tt = row / a.sub, h = row - tt * a.sub;
            if (row >= rows || h >= t.heads)
                continue;
            if (whole) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                uint32_t *dst = reinterpret_cast<uint32_t *>(static_cast<unsigned char *>(a.out) +
                                                             2 * ((t.token + tt) * a.out_token + (t.head + h) * a.out_head));
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
                    if (n * 8 < a.d) {
                        const float x = o[n][2 * i] * inv, y = o[n][2 * i + 1] * inv;
                        odd += x + y;
                        dst[n * 4 + (lane & 3)] = pg_pack<kF16>(x, y);
                    }
                if (a.lse && (lane & 3) == 0)
                    a.lse[static_cast<int64_t>(t.token + tt) * a.heads_q + t.head + h] =
                        sum == 0.0f ? -INFINITY : (ref + log2f(sum)) * kPagedLn2;
            } else {
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
                    *reinterpret_cast<float2 *>(a.part_o + (slot + row) * kPagedMaxDim + n * 8 + (lane & 3) * 2) =
                        make_float2(o[n][2 * i], o[n][2 * i + 1]);
                if ((lane & 3) == 0)
                    *reinterpret_cast<float2 *>(a.part_ml + (slot + row) * 2) = make_float2(ref, sum);
            }
        }
        if (p.starts && !p.ends && lane == 0) {
            PagedJoin &j = a.join[unit];
            j.token = t.token;
            j.head = t.head;
            j.tokens = t.tokens;
            j.heads = t.heads;
            j.count = cut.owner(p.tile_end - 1) - unit + 1;
        }
    }
    cp_wait<0>();
    passed.store(a.join[unit]);
    if (!pg_finite(odd))
        atomicOr(&a.join[unit].flags, kPagedOdd);
}

// Joins the parts of every cut tile, in unit order.  CTA (x, y) has units 8 x ..
// 8 x + 7 (one a warp) and the rows y, y + grid: a warp joins its unit's few parts
// alone, many parts are split over the CTA's warps.  128 requests: 353 us in
// all; joining the parts of a CTA's warps in shared memory first 367 (a row after
// another there, in code run once), by the CTA that arrives last 372.  One request
// of 100 thousand keys and one key/value head is one tile in 1216 parts: 40 us
// in all, 357 with one CTA for all its rows.  8 requests of 300 keys and less take
// 15.4 us so, 13.0 with a CTA a unit.
constexpr int kJoinWarps = 8;
constexpr int kJoinAlone = 16;          // parts a warp joins alone

// (Five CTAs an SM, the registers of the join itself: with what the rows to be computed again
// would take, three fit, and one token over 2000 keys takes 17.1 us instead of 14.6.)
template <bool kF16> __global__ void __launch_bounds__(kJoinWarps * 32, 5) paged_join(const PagedArgs a)
{
    __shared__ PagedJoin join[kJoinWarps];
    __shared__ float4 part[kJoinWarps][32];
    __shared__ float2 part_ml[kJoinWarps];
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int first = blockIdx.x * kJoinWarps, mine = first + warp;
    if (lane == 0)
        join[warp] = a.join[mine];
    __syncthreads();
    // parts [from, to) of a row of the tile that unit `unit` starts
    auto sum = [&](int unit, int row, int from, int to) {
        auto at = [&](int i) { return static_cast<int64_t>(i == 0 ? 2 * unit + 1 : 2 * (unit + i)) * kPagedRowTile + row; };
        RowSum r;
        for (int i = from + lane; i < to; i += 32)
            r.top = fmaxf(r.top, a.part_ml[at(i) * 2]);
#pragma unroll
        for (int o = 16; o; o >>= 1)
            r.top = fmaxf(r.top, __shfl_xor_sync(0xffffffffu, r.top, o));
#pragma unroll 8
        for (int i = from; i < to; ++i)
            r.add(*reinterpret_cast<const float2 *>(a.part_ml + at(i) * 2),
                  *reinterpret_cast<const float4 *>(a.part_o + at(i) * kPagedMaxDim + lane * 4));
        return r;
    };
    float odd = 0.0f, odd_many = 0.0f;  // of this warp's rows; of those of tiles in many parts
    for (int row = blockIdx.y; row < kPagedRowTile; row += gridDim.y) {
        const int tt = row / a.sub, h = row - tt * a.sub;
        const PagedJoin &j = join[warp];
        if (j.count > 0 && j.count <= kJoinAlone && tt < j.tokens && h < j.heads)
            sum(mine, row, 0, j.count).template store<kF16>(a, j.token + tt, j.head + h, lane, odd);
        for (int w = 0; w < kJoinWarps; ++w) {
            const PagedJoin &c = join[w];
            if (c.count <= kJoinAlone || tt >= c.tokens || h >= c.heads)
                continue;
            RowSum r = sum(first + w, row, c.count * warp / kJoinWarps, c.count * (warp + 1) / kJoinWarps);
            part[warp][lane] = r.acc;
            if (lane == 0)
                part_ml[warp] = make_float2(r.top, r.sum);
            __syncthreads();
            if (warp == 0) {
                r = RowSum{};
                for (int i = 0; i < kJoinWarps; ++i)
                    r.top = fmaxf(r.top, part_ml[i].x);
                for (int i = 0; i < kJoinWarps; ++i)
                    r.add(part_ml[i], part[i][lane]);
                r.store<kF16>(a, c.token + tt, c.head + h, lane, odd_many);
            }
            __syncthreads();
        }
    }
    // rows once more, of this warp's unit (its cut tile after all have stored)
    const PagedJoin &j = join[warp];
    if (__syncthreads_or(!pg_finite(odd + odd_many) || j.flags)) {
        const bool many = __syncthreads_or(!pg_finite(odd_many)) && j.count > kJoinAlone;
        const bool cut = many || __any_sync(0xffffffffu, !pg_finite(odd));
        const int32_t y = blockIdx.y, ny = gridDim.y;
        if (cut || j.flags)
            paged_unit_again<kF16>(a, j, j.flags != 0, cut, false, y, ny, 0, kPagedMaxDim,
                                   [&](int32_t t, int32_t h) { return (t * a.sub + h) % ny == y; });
    }
}

template <int DP, bool kF16> int launch_rows(const PagedArgs &a, int grid, cudaStream_t st)
{
    if (int e = launch_early(paged_rows<DP, kF16>, dim3(grid), kRowThreads, kRowSmem, st, a))
        return e;
    static_assert(kJoinWarps == kPagedWarps, "a unit a warp");
    const int rows = a.tok * a.sub;
    return launch_early(paged_join<kF16>, dim3(grid, rows < kPagedRowTile ? rows : kPagedRowTile), kJoinWarps * 32, 0, st, a);
}

}  // namespace

int launch_paged_rows(const PagedArgs &a, bool f16, int grid, void *stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.d <= 64)
        return f16 ? launch_rows<64, true>(a, grid, st) : launch_rows<64, false>(a, grid, st);
    return f16 ? launch_rows<128, true>(a, grid, st) : launch_rows<128, false>(a, grid, st);
}

int paged_tables_set_smem();
int paged_tiles_set_smem();

int paged_set_smem_limit()
{
    int e = paged_tables_set_smem();
    if (!e)
        e = paged_tiles_set_smem();
    auto set = [&](const void *f) {
        if (!e)
            e = static_cast<int>(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowSmem));
    };
    set(reinterpret_cast<const void *>(&paged_rows<64, false>));
    set(reinterpret_cast<const void *>(&paged_rows<64, true>));
    set(reinterpret_cast<const void *>(&paged_rows<128, false>));
    set(reinterpret_cast<const void *>(&paged_rows<128, true>));
    return e;
}

}  // namespace bsm
