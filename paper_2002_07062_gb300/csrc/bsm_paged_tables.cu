// bsm_paged_tables.cu -- what a server's step needs before attention over a
// paged cache: block tables and slot maps from the requests' lengths
// (paged_tables), and the new keys and values copied to their slots
// (paged_write).

#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kTabThreads = 512;
constexpr int kTabPer = 4;                              // requests of a thread
constexpr int kTabTile = kTabThreads * kTabPer;         // requests scanned at once

struct TabSmem {
    int32_t tok[kTabTile + 1];      // tokens of the tile before each request
    int32_t pg[kTabTile + 1];       // new pages of the tile before it
    int64_t warp_tok[kTabThreads / 32];
    int32_t warp_pg[kTabThreads / 32];
    int32_t cached[kTabTile], have[kTabTile];
};

// Largest i with pre[i] <= x, pre[0] <= x < pre[n] ascending.
__device__ __forceinline__ int find_last(const int32_t *pre, int n, int32_t x)
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

__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, uint32_t page) { return tokens / page + (tokens % page ? 1u : 0u); }

// Prefix sums of the requests' tokens and of the pages they take, then every
// token's owner, position and slot, and the new table entries.  Each CTA scans
// all requests (two loads of 4 bytes each, 2048 requests at a time) instead of
// waiting for another's sums, and writes its own range of tokens and entries;
// a token finds its owner by bisection in the shared prefix.  One launch, no
// scratch, no order between CTAs: a page of a new token comes from the free
// list, not from the table entry another CTA writes.  Bound by latency: loads,
// scan, search and stores follow one another (64 requests 4.5 us, 4096 requests
// with 224 thousand tokens 9.5 us on a GB300; with 64-bit quotients 6.5 and 12.2).  Everything per token and request
// is 32-bit (a tile's new pages fit, tables being less than 2^20 wide; its
// tokens are cut at 2^31, past any slot); only running totals are 64-bit.
__global__ void __launch_bounds__(kTabThreads) paged_tables(const PagedTablesArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    TabSmem &s = *reinterpret_cast<TabSmem *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // this CTA's tokens
    const int64_t t_lo = static_cast<int64_t>(a.n_slots) * blockIdx.x / gridDim.x;
    const int64_t t_hi = static_cast<int64_t>(a.n_slots) * (blockIdx.x + 1) / gridDim.x;
    const uint32_t stride = gridDim.x * kTabThreads;
    const int64_t limit = static_cast<int64_t>(a.width) * a.page;
    const uint32_t page_size = static_cast<uint32_t>(a.page), width = static_cast<uint32_t>(a.width);
    int64_t tok_base = 0, pg_base = 0;
    uint32_t flags = 0;
    grid_dependency_wait();
    grid_launch_dependents();

    for (int r0 = 0; r0 < a.n; r0 += kTabTile) {
        int64_t tok[kTabPer], tsum = 0;
        int32_t pg[kTabPer], psum = 0;
        int32_t cs[kTabPer], fs[kTabPer];
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int r = r0 + tid * kTabPer + i;
            cs[i] = r < a.n ? a.cached[r] : 0;
            fs[i] = r < a.n ? a.fresh[r] : 0;
        }
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int j = tid * kTabPer + i;
            if (cs[i] < 0 || fs[i] < 0)
                flags |= BSM_PAGED_NEGATIVE;
            const uint32_t c = cs[i] < 0 ? 0u : static_cast<uint32_t>(cs[i]);
            const uint32_t f = fs[i] < 0 ? 0u : static_cast<uint32_t>(fs[i]);
            if (static_cast<int64_t>(c) + f > limit)
                flags |= BSM_PAGED_WIDTH;
            const uint32_t have = min(pages_of(c, page_size), width), need = min(pages_of(c + f, page_size), width);
            tok[i] = tsum;
            pg[i] = psum;
            tsum += f;
            psum += static_cast<int32_t>(need - have);
            s.cached[j] = static_cast<int32_t>(c);
            s.have[j] = static_cast<int32_t>(have);
        }
        int64_t ti = tsum;
        int32_t pi = psum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t tv = __shfl_up_sync(0xffffffffu, ti, o);
            const int32_t pv = __shfl_up_sync(0xffffffffu, pi, o);
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
        int64_t tw = 0, tall = 0;
        int32_t pw = 0, pall = 0;
#pragma unroll
        for (int w = 0; w < kTabThreads / 32; ++w) {
            const int64_t tv = s.warp_tok[w];
            const int32_t pv = s.warp_pg[w];
            if (w < warp) {
                tw += tv;
                pw += pv;
            }
            tall += tv;
            pall += pv;
        }
        const int64_t tb = tw + ti - tsum;              // of the tile, before this thread
        const int32_t pb = pw + pi - psum;
        const bool mine = static_cast<uint32_t>(r0 / kTabTile) % gridDim.x == blockIdx.x;
#pragma unroll
        for (int i = 0; i < kTabPer; ++i) {
            const int j = tid * kTabPer + i, r = r0 + j;
            const int64_t at = tb + tok[i];
            s.tok[j] = static_cast<int32_t>(at < INT_MAX ? at : INT_MAX);
            s.pg[j] = pb + pg[i];
            if (mine && r < a.n) {
                const int64_t start = tok_base + at;
                const uint32_t len = static_cast<uint32_t>(s.cached[j]) + (fs[i] < 0 ? 0u : static_cast<uint32_t>(fs[i]));
                a.starts[r] = static_cast<int32_t>(start < INT_MAX ? start : INT_MAX);
                a.lengths[r] = static_cast<int32_t>(len < INT_MAX ? len : INT_MAX);
            }
        }
        if (tid == 0) {
            s.tok[kTabTile] = static_cast<int32_t>(tall < INT_MAX ? tall : INT_MAX);
            s.pg[kTabTile] = pall;
        }
        __syncthreads();
        // tokens of these requests that are this CTA's
        const int64_t lo = tok_base > t_lo ? tok_base : t_lo;
        const int64_t hi = tok_base + tall < t_hi ? tok_base + tall : t_hi;
        for (int64_t t = lo + tid; t < hi; t += kTabThreads) {
            const int32_t rel = static_cast<int32_t>(t - tok_base);
            const int j = find_last(s.tok, kTabTile, rel);
            const uint32_t pos = static_cast<uint32_t>(s.cached[j]) + static_cast<uint32_t>(rel - s.tok[j]);
            const uint32_t e = pos / page_size;
            int32_t page = -1;
            if (e < width) {
                if (e < static_cast<uint32_t>(s.have[j])) {
                    page = a.tables[(r0 + j) * a.table_stride + e];
                } else {
                    const int64_t k = pg_base + s.pg[j] + (e - static_cast<uint32_t>(s.have[j]));
                    page = k < a.n_free ? a.free_pages[k] : -1;
                }
            }
            a.slots[t] = page >= 0 ? static_cast<int64_t>(page) * page_size + (pos - e * page_size) : -1;
            a.positions[t] = static_cast<int32_t>(pos < INT_MAX ? pos : INT_MAX);
            a.owners[t] = r0 + j;
        }
        // new entries, dealt over all threads of the launch
        for (uint32_t k = blockIdx.x * kTabThreads + tid; k < static_cast<uint32_t>(pall); k += stride) {
            const int j = find_last(s.pg, kTabTile, static_cast<int32_t>(k));
            const int64_t from = pg_base + k;
            a.tables[(r0 + j) * a.table_stride + s.have[j] + (static_cast<int32_t>(k) - s.pg[j])] =
                from < a.n_free ? a.free_pages[from] : -1;
        }
        tok_base += tall;
        pg_base += pall;
        if (r0 + kTabTile < a.n)
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

// The copy, bound by its bytes.  A thread keeps its place in the row of a
// token (16 bytes of one head) and goes from token to token, eight loads in
// flight; the divisions that find a slot's page are one a token.  (Plain loads: the kernel before
// this one may still write the keys while this one starts.)  237 MB: 38.3 us,
// 0.91 of the copy rate (57 with the place divided out for every piece).
constexpr int kWriteThreads = 256;
constexpr int kWriteAhead = 4;

__global__ void __launch_bounds__(kWriteThreads) paged_write(const PagedWriteArgs a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const uint32_t per = static_cast<uint32_t>(a.heads) * static_cast<uint32_t>(a.chunks);
    const uint32_t at_once = per < kWriteThreads ? kWriteThreads / per : 1u;     // tokens of a block and pass
    const uint32_t sub = at_once > 1 ? threadIdx.x / per : 0u;
    if (sub >= at_once)
        return;
    const int64_t step = static_cast<int64_t>(gridDim.x) * at_once;
    for (uint32_t y = threadIdx.x - sub * per; y < per; y += kWriteThreads) {
        const uint32_t head = y / static_cast<uint32_t>(a.chunks), piece = y - head * static_cast<uint32_t>(a.chunks);
        const unsigned char *src[2];
        unsigned char *dst[2];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            src[kv] = a.src[kv] + head * a.src_head[kv] + piece * 16;
            dst[kv] = a.dst[kv] + head * a.dst_head + piece * 16;
        }
        for (int64_t t0 = blockIdx.x * static_cast<int64_t>(at_once) + sub; t0 < a.n_tokens; t0 += step * kWriteAhead) {
            int64_t to[kWriteAhead];
            uint4 val[kWriteAhead][2];
#pragma unroll
            for (int u = 0; u < kWriteAhead; ++u) {
                const int64_t t = t0 + u * step;
                to[u] = t < a.n_tokens ? a.slots[t] : -1;
            }
#pragma unroll
            for (int u = 0; u < kWriteAhead; ++u) {
                if (to[u] < 0)
                    continue;
                if (to[u] >= a.n_slots_cache) {
                    atomicOr(a.status, BSM_DEV_BOUNDS);
                    to[u] = -1;
                    continue;
                }
                const int64_t t = t0 + u * step;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv)
                    val[u][kv] = *reinterpret_cast<const uint4 *>(src[kv] + t * a.src_token[kv]);
                const int64_t page = to[u] >> 32 ? to[u] / a.page
                                                 : static_cast<int64_t>(static_cast<uint32_t>(to[u]) / static_cast<uint32_t>(a.page));
                to[u] = page * a.dst_page + (to[u] - page * a.page) * a.dst_token;
            }
#pragma unroll
            for (int u = 0; u < kWriteAhead; ++u)
                if (to[u] >= 0)
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv)
                        *reinterpret_cast<uint4 *>(dst[kv] + to[u]) = val[u][kv];
        }
    }
}

}  // namespace

int launch_paged_tables(const PagedTablesArgs &a, int n_sm, void *stream)
{
    const int64_t want = (static_cast<int64_t>(a.n_slots) + kTabThreads - 1) / kTabThreads;
    const int grid = static_cast<int>(want < 1 ? 1 : want > n_sm ? n_sm : want);
    return launch_early(paged_tables, dim3(grid), kTabThreads, sizeof(TabSmem), static_cast<cudaStream_t>(stream), a);
}

int launch_paged_write(const PagedWriteArgs &a, int n_sm, void *stream)
{
    const int64_t per = static_cast<int64_t>(a.heads) * a.chunks, at_once = per < kWriteThreads ? kWriteThreads / per : 1;
    const int64_t want = (a.n_tokens + at_once - 1) / at_once;
    const int64_t most = static_cast<int64_t>(n_sm) * 8;
    return launch_early(paged_write, dim3(static_cast<unsigned>(want < most ? want : most)), kWriteThreads, 0,
                        static_cast<cudaStream_t>(stream), a);
}

int paged_tables_set_smem()
{
    return static_cast<int>(cudaFuncSetAttribute(paged_tables, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(sizeof(TabSmem))));
}

}  // namespace bsm
