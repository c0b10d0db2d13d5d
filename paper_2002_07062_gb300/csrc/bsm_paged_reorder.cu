// bsm_paged_reorder.cu -- the paged cache follows the beams that were kept: table
// rows and lengths by parents, private copies of partly filled pages that two
// beams would go on writing to, and the pages that no beam holds any more.

#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_beam.h"
#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

// One tile of columns of a request's rows.  A thread holds a column: whole pages are
// shared, so its new entries are its old ones by parents, and what it drops it sees without
// another thread (a page lies in one column).  It reads a column before it writes it, so the
// tables may change in place.
__global__ void __launch_bounds__(kReorderTile) reorder_tables(const PagedReorderArgs a)
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
#pragma unroll 8
    for (int b = 0; b < B; ++b)
        old[b * kReorderTile] = col < a.width ? a.tables[(row0 + b) * a.table_stride + col] : -1;
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
            if (tail >= a.n_pages) {
                atomicOr(a.status, BSM_DEV_BOUNDS);     // passed on as it is
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
    for (int i = 0; i < B; ++i) {
        const int32_t p = s_parent[i];
        if (col < s_need[i] && col != s_fresh[i]) {
            held |= uint64_t(1) << p;
            a.new_tables[(row0 + i) * a.new_table_stride + col] = old[p * kReorderTile];
        }
    }
    for (int b = 0; b < B; ++b) {
        const int32_t e = col < s_had[b] ? old[b * kReorderTile] : -1;
        if (e < 0 || (held >> b & 1))
            continue;
        bool other = false;             // (without branches: the loads follow one another closely)
#pragma unroll 4
        for (int k = 0; k < B; ++k)
            other |= (old[k * kReorderTile] == e) & (k < b ? col < s_had[k] : (held >> k & 1) != 0);
        if (!other)
            gone |= uint64_t(1) << b;
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

constexpr int kFinishThreads = 256;
constexpr int kFinishAhead = 4;                         // pieces of a thread in flight
constexpr uint32_t kUnitPieces = 512;                   // 16-byte pieces that a warp copies at a time, about

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

// Pages for the rows that copy, in order of requests and rows, and the copies, a warp at a time about
// 8 KiB (some tokens of one row in one layer's keys or values).  Every CTA counts all requests' copies
// itself (256 at once) instead of waiting for another's sums.
__global__ void __launch_bounds__(kFinishThreads) reorder_pages(const PagedReorderArgs a)
{
    __shared__ uint64_t s_rows[kFinishThreads];         // rows of a request that copy
    __shared__ int32_t s_copies[kFinishThreads], s_dropped[kFinishThreads];
    __shared__ int32_t s_from[kFinishThreads], s_to[kFinishThreads], s_part[kFinishThreads], s_units[kFinishThreads];
    __shared__ int32_t s_warp[3][kFinishThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31;
    const int warps = gridDim.x * (kFinishThreads / 32), me = blockIdx.x * (kFinishThreads / 32) + (tid >> 5);
    const int32_t B = a.beams;
    const uint32_t per = static_cast<uint32_t>(a.heads) * a.chunks, both = static_cast<uint32_t>(a.layers) * 2;
    const bool whole = a.head == a.chunks * 16ll && a.token == per * 16ll;      // a page's tokens are one run of bytes
    const int32_t tokens = per >= kUnitPieces ? 1 : static_cast<int32_t>(kUnitPieces / per);       // of a unit
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t rows = static_cast<int64_t>(a.n) * B;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kFinishThreads + tid; i < rows;
         i += static_cast<int64_t>(gridDim.x) * kFinishThreads)
        a.new_lengths[i] = a.row_length[i];
    int64_t taken = 0, dropped = 0;                     // of the requests before
    for (int32_t r0 = 0; r0 < a.n; r0 += kFinishThreads) {
        uint64_t mask = 0;
        int32_t count = 0;
        if (r0 + tid < a.n) {
            const int64_t at = static_cast<int64_t>(r0 + tid) * a.tiles;
            for (int z = 0; z < a.tiles; ++z) {
                mask |= a.copies[at + z];
                count += a.counts[at + z];
            }
        }
        int32_t all_copies, all_dropped;
        const int32_t pc = before_me(__popcll(mask), s_warp[0], &all_copies);
        s_dropped[tid] = before_me(count, s_warp[1], &all_dropped);
        s_rows[tid] = mask;
        s_copies[tid] = pc;
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
                if (blockIdx.x == 0) {
                    a.new_tables[row * a.new_table_stride + full] = page;
                    if (page >= a.n_pages)
                        atomicOr(a.status, BSM_DEV_BOUNDS);
                }
                if (page >= 0 && page < a.n_pages)
                    units = (part + tokens - 1) / tokens;
                s_from[tid] = a.row_source[row];
                s_to[tid] = page;
                s_part[tid] = part;
            }
            int32_t all_units;
            s_units[tid] = before_me(units, s_warp[2], &all_units);
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
                for (uint32_t x = lane; x < pieces; x += 32 * kFinishAhead) {
                    uint4 v[kFinishAhead];
                    int64_t off[kFinishAhead];
#pragma unroll
                    for (int u = 0; u < kFinishAhead; ++u) {
                        const uint32_t y = x + u * 32;
                        if (y >= pieces)
                            continue;
                        if (whole) {
                            off[u] = y * 16ll;
                        } else {
                            const uint32_t t = y / per, rest = y - t * per, h = rest / static_cast<uint32_t>(a.chunks);
                            off[u] = t * a.token + h * a.head + (rest - h * a.chunks) * 16;
                        }
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
        // the dropped pages, a warp a tile of a request
        const int32_t here = min(kFinishThreads, a.n - r0);
        for (int64_t l = me; l < static_cast<int64_t>(here) * a.tiles; l += warps) {
            const int32_t q = static_cast<int32_t>(pg_div(l, a.tiles)), z = static_cast<int32_t>(l - static_cast<int64_t>(q) * a.tiles);
            const int64_t first = static_cast<int64_t>(r0 + q) * a.tiles;
            int32_t before = 0;                         // of the request's tiles before
            for (int k = lane; k < z; k += 32)
                before += a.counts[first + k];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1)
                before += __shfl_xor_sync(0xffffffffu, before, o);
            const int64_t at = dropped + s_dropped[q] + before;
            const int32_t c = a.counts[first + z];
            const int32_t *list = a.lists + (first + z) * kReorderTile * B;
            const int32_t room = static_cast<int32_t>(at >= a.n_dropped ? 0 : min(static_cast<int64_t>(c), a.n_dropped - at));
#pragma unroll 4
            for (int i = lane; i < room; i += 32)
                a.dropped[at + i] = list[i];
        }
        taken += all_copies;
        dropped += all_dropped;
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.info[0] = taken < a.n_free ? taken : a.n_free;
        a.info[1] = taken < a.n_free ? 0 : taken - a.n_free;
        a.info[2] = dropped;
        a.info[3] = (taken > a.n_free ? BSM_PAGED_PAGES : 0u) | (dropped > a.n_dropped ? BSM_PAGED_DROPPED : 0u);
    }
}

}  // namespace

int launch_paged_reorder(const PagedReorderArgs &a, int n_sm, void *stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.n == 0)                                       // (info alone)
        return launch_early(reorder_pages, dim3(1), kFinishThreads, 0, st, a);
    if (int e = launch_early(reorder_tables, dim3(static_cast<unsigned>(a.n) * a.tiles), kReorderTile,
                             static_cast<size_t>(a.beams) * kReorderTile * 4, st, a))
        return e;
    const int64_t want = static_cast<int64_t>(a.n) * a.beams * a.layers * 2, most = static_cast<int64_t>(n_sm) * 6;
    return launch_early(reorder_pages, dim3(static_cast<unsigned>(want < most ? want : most)), kFinishThreads, 0, st, a);
}

}  // namespace bsm
