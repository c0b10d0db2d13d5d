// bsm_paged_tables.cu -- what a server's step needs before attention over a
// paged cache: block tables and slot maps from the requests' lengths
// (paged_tables), and the new keys and values copied to their slots
// (paged_write).

#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "bsm_paged.h"

namespace bsm {
namespace {

constexpr int kTabThreads = 512;
constexpr int kTabPer = 4;                              // requests of a thread
constexpr int kTabTile = kTabThreads * kTabPer;         // requests scanned at once

struct TabSmem {
    int64_t tok[kTabTile + 1];      // tokens before each request of the tile
    int64_t pg[kTabTile + 1];       // new pages before it
    int64_t warp_tok[kTabThreads / 32], warp_pg[kTabThreads / 32];
    int32_t cached[kTabTile], have[kTabTile];
};

// Largest i with pre[i] <= x, pre[0] <= x < pre[n] ascending.
__device__ __forceinline__ int find_last(const int64_t *pre, int n, int64_t x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pre[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Prefix sums of the requests' tokens and of the pages they take, then every
// token's owner, position and slot, and the new table entries.  Each CTA scans
// all requests (two loads of 4 bytes each, 2048 requests at a time) instead of
// waiting for another's sums, and writes its own range of tokens and entries;
// a token finds its owner by bisection in the shared prefix.  One launch, no
// scratch, no order between CTAs: a page of a new token comes from the free
// list, not from the table entry another CTA writes.
__global__ void __launch_bounds__(kTabThreads) paged_tables(const PagedTablesArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    TabSmem &s = *reinterpret_cast<TabSmem *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // this CTA's tokens
    const int64_t t_lo = static_cast<int64_t>(a.n_slots) * blockIdx.x / gridDim.x;
    const int64_t t_hi = static_cast<int64_t>(a.n_slots) * (blockIdx.x + 1) / gridDim.x;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kTabThreads;
    const int64_t limit = static_cast<int64_t>(a.width) * a.page;
    int64_t tok_base = 0, pg_base = 0;
    uint32_t flags = 0;

    for (int r0 = 0; r0 < a.n; r0 += kTabTile) {
        int64_t tok[kTabPer], pg[kTabPer];
        int64_t tsum = 0, psum = 0;
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int j = tid * kTabPer + i, r = r0 + j;
            int64_t c = 0, f = 0;
            if (r < a.n) {
                c = a.cached[r];
                f = a.fresh[r];
                if (c < 0 || f < 0) {
                    flags |= BSM_PAGED_NEGATIVE;
                    c = c < 0 ? 0 : c;
                    f = f < 0 ? 0 : f;
                }
                if (c + f > limit)
                    flags |= BSM_PAGED_WIDTH;
            }
            const int64_t have_all = (c + a.page - 1) / a.page, need_all = (c + f + a.page - 1) / a.page;
            const int64_t have = have_all < a.width ? have_all : a.width;
            const int64_t need = need_all < a.width ? need_all : a.width;
            tok[i] = tsum;
            pg[i] = psum;
            tsum += f;
            psum += need - have;
            s.cached[j] = static_cast<int32_t>(c);
            s.have[j] = static_cast<int32_t>(have);
        }
        int64_t ti = tsum, pi = psum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t tv = __shfl_up_sync(0xffffffffu, ti, o), pv = __shfl_up_sync(0xffffffffu, pi, o);
            if (lane >= o) {
                ti += tv;
                pi += pv;
            }
        }
        if (lane == 31) {
            s.warp_tok[warp] = ti;
            s.warp_pg[warp] = pi;
        }
        __syncthreads();
        int64_t tw = 0, pw = 0, tall = 0, pall = 0;
#pragma unroll
        for (int w = 0; w < kTabThreads / 32; ++w) {
            const int64_t tv = s.warp_tok[w], pv = s.warp_pg[w];
            if (w < warp) {
                tw += tv;
                pw += pv;
            }
            tall += tv;
            pall += pv;
        }
        const int64_t tb = tok_base + tw + ti - tsum, pb = pg_base + pw + pi - psum;
        const bool mine = (r0 / kTabTile) % gridDim.x == blockIdx.x;
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int j = tid * kTabPer + i, r = r0 + j;
            s.tok[j] = tb + tok[i];
            s.pg[j] = pb + pg[i];
            if (mine && r < a.n) {
                const int64_t end = s.cached[j] + (i + 1 < kTabPer ? tok[i + 1] : tsum) - tok[i];
                a.starts[r] = static_cast<int32_t>(tb + tok[i] < INT_MAX ? tb + tok[i] : INT_MAX);
                a.lengths[r] = static_cast<int32_t>(end < INT_MAX ? end : INT_MAX);
            }
        }
        if (tid == 0) {
            s.tok[kTabTile] = tok_base + tall;
            s.pg[kTabTile] = pg_base + pall;
        }
        __syncthreads();
        // tokens of these requests that are this CTA's
        const int64_t lo = tok_base > t_lo ? tok_base : t_lo;
        const int64_t hi = tok_base + tall < t_hi ? tok_base + tall : t_hi;
        for (int64_t t = lo + tid; t < hi; t += kTabThreads) {
            const int j = find_last(s.tok, kTabTile, t);
            const int64_t pos = s.cached[j] + (t - s.tok[j]);
            const int64_t e = pos / a.page;
            int32_t page = -1;
            if (e < a.width) {
                if (e < s.have[j]) {
                    page = a.tables[(r0 + j) * a.table_stride + e];
                } else {
                    const int64_t k = s.pg[j] + (e - s.have[j]);
                    page = k < a.n_free ? a.free_pages[k] : -1;
                }
            }
            a.slots[t] = page >= 0 ? static_cast<int64_t>(page) * a.page + (pos - e * a.page) : -1;
            a.positions[t] = static_cast<int32_t>(pos < INT_MAX ? pos : INT_MAX);
            a.owners[t] = r0 + j;
        }
        // new entries, dealt over all threads of the launch by their place in the free list
        const int64_t me = static_cast<int64_t>(blockIdx.x) * kTabThreads + tid;
        int64_t k = pg_base - pg_base % stride + me;
        k += k < pg_base ? stride : 0;
        for (; k < pg_base + pall; k += stride) {
            const int j = find_last(s.pg, kTabTile, k);
            a.tables[(r0 + j) * a.table_stride + s.have[j] + (k - s.pg[j])] = k < a.n_free ? a.free_pages[k] : -1;
        }
        tok_base += tall;
        pg_base += pall;
        __syncthreads();
    }
    for (int64_t t = (tok_base > t_lo ? tok_base : t_lo) + tid; t < t_hi; t += kTabThreads) {
        a.slots[t] = -1;
        a.positions[t] = -1;
        a.owners[t] = -1;
    }
    if (blockIdx.x == 0) {
        // every CTA has met every request: this one's flags are the batch's
        const int any_neg = __syncthreads_or(flags & BSM_PAGED_NEGATIVE);
        const int any_wide = __syncthreads_or(flags & BSM_PAGED_WIDTH);
        if (tid == 0) {
            a.starts[a.n] = static_cast<int32_t>(tok_base < INT_MAX ? tok_base : INT_MAX);
            uint32_t f = (any_neg ? BSM_PAGED_NEGATIVE : 0u) | (any_wide ? BSM_PAGED_WIDTH : 0u);
            if (pg_base > a.n_free)
                f |= BSM_PAGED_PAGES;
            if (tok_base > a.n_slots)
                f |= BSM_PAGED_TOKENS;
            a.info[0] = tok_base;
            a.info[1] = pg_base < a.n_free ? pg_base : a.n_free;
            a.info[2] = pg_base < a.n_free ? 0 : pg_base - a.n_free;
            a.info[3] = f;
        }
    }
}

// The copy: 16 bytes a thread and step, kWriteAhead of them in flight.
constexpr int kWriteThreads = 256;
constexpr int kWriteAhead = 4;

__global__ void __launch_bounds__(kWriteThreads) paged_write(const PagedWriteArgs a)
{
    const int64_t per_token = static_cast<int64_t>(a.heads) * a.chunks;
    const int64_t total = 2 * a.n_tokens * per_token;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWriteThreads;
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * kWriteThreads + threadIdx.x; i0 < total;
         i0 += step * kWriteAhead) {
        uint4 val[kWriteAhead];
        unsigned char *dst[kWriteAhead];
#pragma unroll
        for (int u = 0; u < kWriteAhead; ++u) {
            const int64_t i = i0 + u * step;
            dst[u] = nullptr;
            if (i >= total)
                continue;
            const int kv = i >= total / 2;
            const int64_t x = kv ? i - total / 2 : i;
            const int64_t t = x / per_token;
            const int32_t y = static_cast<int32_t>(x - t * per_token);
            const int32_t h = y / a.chunks, c = y - h * a.chunks;
            const int64_t slot = a.slots[t];
            if (slot < 0)
                continue;
            if (slot >= a.n_slots_cache) {
                atomicOr(a.status, BSM_DEV_BOUNDS);
                continue;
            }
            const int64_t page = slot / a.page;
            val[u] = *reinterpret_cast<const uint4 *>(a.src[kv] + t * a.src_token[kv] + h * a.src_head[kv] + c * 16);
            dst[u] = a.dst[kv] + page * a.dst_page + (slot - page * a.page) * a.dst_token + h * a.dst_head + c * 16;
        }
#pragma unroll
        for (int u = 0; u < kWriteAhead; ++u)
            if (dst[u])
                *reinterpret_cast<uint4 *>(dst[u]) = val[u];
    }
}

}  // namespace

int launch_paged_tables(const PagedTablesArgs &a, int n_sm, void *stream)
{
    const int64_t want = (static_cast<int64_t>(a.n_slots) + kTabThreads - 1) / kTabThreads;
    const int grid = static_cast<int>(want < 1 ? 1 : want > n_sm ? n_sm : want);
    paged_tables<<<grid, kTabThreads, sizeof(TabSmem), static_cast<cudaStream_t>(stream)>>>(a);
    return static_cast<int>(cudaGetLastError());
}

int launch_paged_write(const PagedWriteArgs &a, int n_sm, void *stream)
{
    const int64_t total = 2 * a.n_tokens * a.heads * a.chunks;
    const int64_t want = (total + kWriteThreads - 1) / kWriteThreads;
    const int64_t most = static_cast<int64_t>(n_sm) * 8;
    paged_write<<<static_cast<int>(want < most ? want : most), kWriteThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return static_cast<int>(cudaGetLastError());
}

int paged_tables_set_smem()
{
    return static_cast<int>(cudaFuncSetAttribute(paged_tables, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(sizeof(TabSmem))));
}

}  // namespace bsm
