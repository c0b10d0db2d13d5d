// bsm_paged_reorder.cu -- the paged cache follows the beams that were kept: table
// rows and lengths by parents, private copies of partly filled pages that two
// beams would go on writing to, and the pages that no beam holds any more.

#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "bsm_beam.h"
#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

// One tile of columns of a request's rows.  A thread holds a column: whole pages are
// shared, so its new entries are its old ones by parents, and what it drops it sees without
// another thread (a page lies in one column).  It reads a column before it writes it, so the
// tables may change in place.  Latency: 7 us for 64 requests of 5 rows, 8 for 16 of 16 rows of 1500 (13 with
// the old entries in shared memory alone: 16 x 16 dependent comparisons).
// kBeams: at most so many beams, a thread's old entries in registers; 0: any number, in shared memory.
template <int kBeams> __global__ void __launch_bounds__(kReorderTile) reorder_tables(const PagedReorderArgs a)
{
    extern __shared__ int32_t old_rows[];               // beams x kReorderTile
    __shared__ int32_t s_parent[kBeamMost], s_length[kBeamMost], s_had[kBeamMost], s_need[kBeamMost], s_tail[kBeamMost];
    __shared__ int32_t s_fresh[kBeamMost];              // the column of a row that waits for a page, or -1
    __shared__ uint32_t s_mask[2];
    __shared__ int32_t s_warp[kReorderTile / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t r = static_cast<int32_t>(blockIdx.x / static_cast<uint32_t>(a.tiles));
    const int32_t z = static_cast<int32_t>(blockIdx.x - static_cast<uint32_t>(r) * a.tiles);
    const int32_t first = z * kReorderTile, col = first + tid, B = a.beams;
    const int64_t row0 = static_cast<int64_t>(r) * B;
    grid_dependency_wait();
    grid_launch_dependents();
    int32_t *old = old_rows + tid;
    // (every entry, used or not: which are is known when the lengths have come)
    int32_t mine_old[kBeams ? kBeams : 1];
    if (kBeams) {
#pragma unroll
        for (int b = 0; b < kBeams; ++b)
            mine_old[b] = b < B && col < a.width ? a.tables[(row0 + b) * a.table_stride + col] : -1;
#pragma unroll
        for (int b = 0; b < kBeams; ++b)
            if (b < B)
                old[b * kReorderTile] = mine_old[b];
    } else {
#pragma unroll 8
        for (int b = 0; b < B; ++b)
            old[b * kReorderTile] = col < a.width ? a.tables[(row0 + b) * a.table_stride + col] : -1;
    }
    if (tid < B) {
        const int32_t p = a.parents[r * a.parent_stride + tid], raw = a.lengths[row0 + tid];
        const int64_t most = static_cast<int64_t>(a.width) * a.page;
        const int32_t length = raw < 0 ? 0 : raw > most ? static_cast<int32_t>(most) : raw;
        if (z == 0 && (p >= B || length != raw))
            atomicOr(a.status, BSM_DEV_BOUNDS);
        s_parent[tid] = p < B ? p : -1;
        s_length[tid] = length;
        s_had[tid] = length / a.page + (length % a.page ? 1 : 0);
    }
    __syncthreads();
    int32_t mine = -1, full = -1, tail = -1;            // of new row tid
    if (tid < B) {
        mine = s_parent[tid];
        const int32_t length = mine >= 0 ? s_length[mine] : 0;
        s_need[tid] = mine >= 0 ? s_had[mine] : 0;
        full = length / a.page;
        if (z == 0)
            a.row_length[row0 + tid] = length;
        if (length % a.page && full >= first && full < first + kReorderTile) {
            tail = old_rows[mine * kReorderTile + full - first];
            // (-1: a page that was missing before; what lies outside the cache is passed on as it is)
            if (tail < -1 || tail >= a.n_pages) {
                atomicOr(a.status, BSM_DEV_BOUNDS);
                tail = -1;
            }
        }
        s_tail[tid] = tail;
    }
    __syncthreads();
    // a partly filled page stays with the first row that takes it
    bool copy = false;
    if (tail >= 0)
        for (int j = 0; j < tid; ++j)
            copy |= s_tail[j] == tail;
    if (warp < 2) {
        const uint32_t m = __ballot_sync(0xffffffffu, copy);
        if (lane == 0)
            s_mask[warp] = m;
        s_fresh[tid] = copy ? full : -1;
        if (copy)
            a.row_source[row0 + tid] = tail;
    }
    __syncthreads();
    uint64_t held = 0, gone = 0;                        // old rows whose page here is in a new row; dropped ones
    auto follow = [&](int i) {
        const int32_t p = s_parent[i];
        if (col < s_need[i] && col != s_fresh[i]) {
            held |= uint64_t(1) << p;
            a.new_tables[(row0 + i) * a.new_table_stride + col] = old[p * kReorderTile];
        }
    };
    // (comparisons without branches: everything follows closely)
    if (kBeams) {
#pragma unroll
        for (int i = 0; i < kBeams; ++i)
            if (i < B)
                follow(i);
        uint32_t had = 0;
#pragma unroll
        for (int b = 0; b < kBeams; ++b)
            had |= b < B && col < s_had[b] ? 1u << b : 0u;
        const uint32_t kept = static_cast<uint32_t>(held);
#pragma unroll
        for (int b = 0; b < kBeams; ++b) {
            uint32_t same = 0;          // rows with this one's page
#pragma unroll
            for (int k = 0; k < kBeams; ++k)
                same |= mine_old[k] == mine_old[b] ? 1u << k : 0u;
            const bool last_seen = (same & kept) == 0 && (same & had & ((1u << b) - 1u)) == 0;
            gone |= (had >> b & 1) && mine_old[b] >= 0 && last_seen ? uint64_t(1) << b : 0;
        }
    } else {
        for (int i = 0; i < B; ++i)
            follow(i);
        for (int b = 0; b < B; ++b) {
            const int32_t e = col < s_had[b] ? old[b * kReorderTile] : -1;
            if (e < 0 || (held >> b & 1))
                continue;
            bool other = false;
#pragma unroll 8
            for (int k = 0; k < B; ++k)
                other |= (old[k * kReorderTile] == e) & (k < b ? col < s_had[k] : (held >> k & 1) != 0);
            if (!other)
                gone |= uint64_t(1) << b;
        }
    }
    // in order of columns, then beams
    int32_t before = __popcll(gone);
    const int32_t n = before;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t v = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o)
            before += v;
    }
    if (lane == 31)
        s_warp[warp] = before;
    __syncthreads();
    int32_t all = 0;
    before -= n;
#pragma unroll
    for (int w = 0; w < kReorderTile / 32; ++w) {
        if (w < warp)
            before += s_warp[w];
        all += s_warp[w];
    }
    int32_t *list = a.lists + static_cast<int64_t>(blockIdx.x) * kReorderTile * B;
    while (gone) {
        list[before++] = old[(__ffsll(static_cast<long long>(gone)) - 1) * kReorderTile];
        gone &= gone - 1;
    }
    if (tid == 0) {
        a.copies[blockIdx.x] = static_cast<uint64_t>(s_mask[1]) << 32 | s_mask[0];
        a.counts[blockIdx.x] = all;
    }
}

constexpr int kFinishThreads = 256, kFinishCtas = 4;    // its CTAs on an SM
constexpr int kFinishAhead = 4;                         // pieces of a thread in flight
constexpr int kSlices = 8;                              // warps that copy a list of dropped pages
constexpr uint32_t kUnitPieces = 256;                   // 16-byte pieces that a warp copies at a time, about

// Sum over the block's threads before this one; *all gets the block's.
__device__ __forceinline__ int32_t before_me(int32_t x, int32_t *warps, int32_t *all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t sum = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o)
            sum += v;
    }
    if (lane == 31)
        warps[warp] = sum;
    __syncthreads();
    int32_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kFinishThreads / 32; ++w) {
        if (w < warp)
            base += warps[w];
        total += warps[w];
    }
    *all = total;
    return base + sum - x;
}

// The pages that requests dropped, in order: each CTA of these counts all (request, tile) lists, 1024 at
// once, and copies some, several warps a list.  The first one knows all counts and writes info.
__device__ void list_dropped(const PagedReorderArgs &a, int cta, int ctas)
{
    constexpr int kAtOnce = 4 * kFinishThreads;
    __shared__ int32_t s_first[kAtOnce + 1];
    __shared__ int32_t s_warp[2][kFinishThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t lists = static_cast<int64_t>(a.n) * a.tiles;
    int64_t dropped = 0, taken = 0;                     // of the lists before
    for (int64_t l0 = 0; l0 < lists; l0 += kAtOnce) {
        int32_t c[4], sum = 0, copies = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t l = l0 + tid * 4 + i;
            c[i] = l < lists ? a.counts[l] : 0;
            sum += c[i];
            copies += l < lists && cta == 0 ? __popcll(a.copies[l]) : 0;
        }
        int32_t all, all_copies = 0;
        int32_t at = before_me(sum, s_warp[0], &all);
        if (cta == 0)
            before_me(copies, s_warp[1], &all_copies);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s_first[tid * 4 + i] = at;
            at += c[i];
        }
        if (tid == 0)
            s_first[kAtOnce] = all;
        __syncthreads();
        const int here = static_cast<int>(lists - l0 < kAtOnce ? lists - l0 : kAtOnce);
        for (int x = cta * (kFinishThreads / 32) + (tid >> 5); x < here * kSlices; x += ctas * (kFinishThreads / 32)) {
            const int l = x / kSlices, slice = x % kSlices, count = s_first[l + 1] - s_first[l];
            const int64_t to = dropped + s_first[l], room = a.n_dropped - to;
            // (more than 2^31 may be past the caller's room, so its sign is asked for in 64 bits)
            const int32_t end = count * (slice + 1) / kSlices, n = room < end ? static_cast<int32_t>(room > 0 ? room : 0) : end;
            const int32_t *list = a.lists + (l0 + l) * kReorderTile * a.beams;
#pragma unroll 4
            for (int i = count * slice / kSlices + lane; i < n; i += 32)
                a.dropped[to + i] = list[i];
        }
        dropped += all;
        taken += all_copies;
        __syncthreads();
    }
    if (cta == 0 && tid == 0) {
        a.info[0] = taken < a.n_free ? taken : a.n_free;
        a.info[1] = taken < a.n_free ? 0 : taken - a.n_free;
        a.info[2] = dropped;
        a.info[3] = (taken > a.n_free ? BSM_PAGED_PAGES : 0u) | (dropped > a.n_dropped ? BSM_PAGED_DROPPED : 0u);
    }
}

// Pages for the rows that copy, in order of requests and rows, and the copies, a warp at a time about
// 4 KiB (some tokens of one row in one layer's keys or values).  Every CTA counts all requests' copies
// itself (256 at once) instead of waiting for another's sums.  The launch's last CTAs list the
// dropped pages.  Bound by the copies: 362 MB 55 us, 0.97 of a copy's rate (a CTA a copy 61; 8 or 16 loads a lane
// in fewer CTAs 57 to 59).
__global__ void __launch_bounds__(kFinishThreads, kFinishCtas) reorder_pages(const PagedReorderArgs a)
{
    __shared__ unsigned long long s_rows[kFinishThreads];   // rows of a request that copy
    __shared__ int32_t s_copies[kFinishThreads];
    __shared__ int32_t s_from[kFinishThreads], s_to[kFinishThreads], s_part[kFinishThreads], s_units[kFinishThreads];
    __shared__ int32_t s_warp[2][kFinishThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31;
    const int ctas = gridDim.x - a.listers;
    const int warps = ctas * (kFinishThreads / 32), me = blockIdx.x * (kFinishThreads / 32) + (tid >> 5);
    const int32_t B = a.beams;
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t rows = static_cast<int64_t>(a.n) * B;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kFinishThreads + tid; i < rows;
         i += static_cast<int64_t>(gridDim.x) * kFinishThreads)
        a.new_lengths[i] = a.row_length[i];
    if (static_cast<int>(blockIdx.x) >= ctas) {
        list_dropped(a, blockIdx.x - ctas, a.listers);
        return;
    }
    const uint32_t per = static_cast<uint32_t>(a.heads) * a.chunks, both = static_cast<uint32_t>(a.layers) * 2;
    const bool whole = a.head == a.chunks * 16ll && a.token == per * 16ll;      // a page's tokens are one run of bytes
    const int32_t tokens = per >= kUnitPieces ? 1 : static_cast<int32_t>(kUnitPieces / per);       // of a unit
    int64_t taken = 0;                                  // of the requests before
    for (int32_t r0 = 0; r0 < a.n; r0 += kFinishThreads) {
        const int32_t here = a.n - r0 < kFinishThreads ? a.n - r0 : kFinishThreads;
        s_rows[tid] = 0;
        __syncthreads();
        // (a request's tiles have different rows)
        for (int64_t l = tid; l < static_cast<int64_t>(here) * a.tiles; l += kFinishThreads)
            if (const unsigned long long m = a.copies[static_cast<int64_t>(r0) * a.tiles + l])
                atomicOr(&s_rows[pg_div(l, a.tiles)], m);
        __syncthreads();
        int32_t all_copies;
        s_copies[tid] = before_me(__popcll(s_rows[tid]), s_warp[0], &all_copies);
        __syncthreads();
        for (int32_t e0 = 0; e0 < all_copies; e0 += kFinishThreads) {
            // copy e0 + tid: its row, where from and where to
            int32_t units = 0;
            if (e0 + tid < all_copies) {
                const int32_t e = e0 + tid;
                int lo = 0, hi = kFinishThreads;        // its request
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_copies[mid] <= e)
                        lo = mid;
                    else
                        hi = mid;
                }
                uint64_t m = s_rows[lo];
                for (int k = e - s_copies[lo]; k > 0; --k)
                    m &= m - 1;
                const int64_t row = static_cast<int64_t>(r0 + lo) * B + (__ffsll(static_cast<long long>(m)) - 1);
                const int64_t k = taken + e;
                const int32_t length = a.row_length[row], full = length / a.page, part = length - full * a.page;
                const int32_t page = k < a.n_free ? a.free_pages[k] : -1;
                const bool there = page >= 0 && page < a.n_pages;
                if (blockIdx.x == 0) {
                    a.new_tables[row * a.new_table_stride + full] = page;
                    if (k < a.n_free && !there)
                        atomicOr(a.status, BSM_DEV_BOUNDS);
                }
                if (there)
                    units = (part + tokens - 1) / tokens;
                s_from[tid] = a.row_source[row];
                s_to[tid] = page;
                s_part[tid] = part;
            }
            int32_t all_units;
            s_units[tid] = before_me(units, s_warp[1], &all_units);
            __syncthreads();
            const int64_t items = static_cast<int64_t>(all_units) * both;
            for (int64_t it = me; it < items; it += warps) {
                const int32_t unit = static_cast<int32_t>(pg_div(it, both));
                const uint32_t which = static_cast<uint32_t>(it - static_cast<int64_t>(unit) * both);
                int lo = 0, hi = kFinishThreads;        // the copy it belongs to
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_units[mid] <= unit)
                        lo = mid;
                    else
                        hi = mid;
                }
                const int32_t t0 = (unit - s_units[lo]) * tokens, t1 = min(t0 + tokens, s_part[lo]);
                unsigned char *base = a.cache[which & 1] + static_cast<int64_t>(which >> 1) * a.layer + t0 * a.token;
                const unsigned char *from = base + s_from[lo] * a.page_bytes;
                unsigned char *to = base + s_to[lo] * a.page_bytes;
                const uint32_t pieces = static_cast<uint32_t>(t1 - t0) * per;
                if (whole) {
                    from += lane * 16;
                    to += lane * 16;
                    uint32_t x = lane;
                    for (; x + 32 * (kFinishAhead - 1) < pieces; x += 32 * kFinishAhead) {
                        uint4 v[kFinishAhead];
#pragma unroll
                        for (int u = 0; u < kFinishAhead; ++u)
                            v[u] = *reinterpret_cast<const uint4 *>(from + u * 512);
#pragma unroll
                        for (int u = 0; u < kFinishAhead; ++u)
                            *reinterpret_cast<uint4 *>(to + u * 512) = v[u];
                        from += kFinishAhead * 512;
                        to += kFinishAhead * 512;
                    }
                    for (; x < pieces; x += 32) {
                        *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
                        from += 512;
                        to += 512;
                    }
                    continue;
                }
                for (uint32_t x = lane; x < pieces; x += 32 * kFinishAhead) {
                    uint4 v[kFinishAhead];
                    int64_t off[kFinishAhead];
#pragma unroll
                    for (int u = 0; u < kFinishAhead; ++u) {
                        const uint32_t y = x + u * 32;
                        if (y >= pieces)
                            continue;
                        const uint32_t t = y / per, rest = y - t * per, h = rest / static_cast<uint32_t>(a.chunks);
                        off[u] = t * a.token + h * a.head + (rest - h * a.chunks) * 16;
                        v[u] = *reinterpret_cast<const uint4 *>(from + off[u]);
                    }
#pragma unroll
                    for (int u = 0; u < kFinishAhead; ++u)
                        if (x + u * 32 < pieces)
                            *reinterpret_cast<uint4 *>(to + off[u]) = v[u];
                }
            }
            __syncthreads();
        }
        taken += all_copies;
    }
}

}  // namespace

int launch_paged_reorder(PagedReorderArgs a, int n_sm, void *stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.n > 0) {
        const dim3 grid(static_cast<unsigned>(a.n) * a.tiles);
        const size_t smem = static_cast<size_t>(a.beams) * kReorderTile * 4;
        const int e = a.beams <= 4    ? launch_early(reorder_tables<4>, grid, kReorderTile, smem, st, a)
                      : a.beams <= 8  ? launch_early(reorder_tables<8>, grid, kReorderTile, smem, st, a)
                      : a.beams <= 16 ? launch_early(reorder_tables<16>, grid, kReorderTile, smem, st, a)
                                      : launch_early(reorder_tables<0>, grid, kReorderTile, smem, st, a);
        if (e)
            return e;
    }
    // a warp for each unit that may be copied and each list of dropped pages, as far as they are on the
    // device at once
    const int64_t most = static_cast<int64_t>(n_sm) * kFinishCtas, warps = kFinishThreads / 32;
    const int64_t pieces = static_cast<int64_t>(a.page) * a.heads * a.chunks, units = (pieces + kUnitPieces - 1) / kUnitPieces;
    const int64_t copies = static_cast<int64_t>(a.n) * a.beams * a.layers * 2, lists = static_cast<int64_t>(a.n) * a.tiles;
    const int64_t listers = std::max<int64_t>(1, std::min((lists * kSlices + warps - 1) / warps, most / 8));
    const int64_t copiers = std::max<int64_t>(1, copies > most * warps ? most : std::min(copies * units / warps, most));
    a.listers = static_cast<int32_t>(listers);
    return launch_early(reorder_pages, dim3(static_cast<unsigned>(listers + std::min(copiers, most - listers))),
                        kFinishThreads, 0, st, a);
}

}  // namespace bsm
