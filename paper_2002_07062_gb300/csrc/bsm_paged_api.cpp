// bsm_paged_api.cpp -- C ABI of the paged-cache operators: argument checks,
// how a call's work is tiled and split, the workspace's layout.

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <mutex>

#include "bsm_internal.h"
#include "bsm_paged.h"
#include "bsm_trace.h"

namespace bsm {

int device_status_word(int device, uint32_t **out);

namespace {

struct PagedDev {
    bool ready = false;
    int n_sm = 0;
    uint32_t *status = nullptr;
};

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

std::mutex g_paged_mu;
PagedDev g_pdev[64];
EncodeTiled g_paged_encode = nullptr;

int paged_device(int device, PagedDev **out)
{
    if (device < 0 && cudaGetDevice(&device) != cudaSuccess)
        return BSM_ERR_NO_DEVICE;
    if (device < 0 || device >= 64)
        return BSM_ERR_NO_DEVICE;
    std::lock_guard<std::mutex> lk(g_paged_mu);
    PagedDev &d = g_pdev[device];
    if (!d.ready) {
        if (cudaDeviceGetAttribute(&d.n_sm, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
            return BSM_ERR_NO_DEVICE;
        if (int rc = device_status_word(device, &d.status))
            return rc;
        if (!g_paged_encode) {
            void *fn = nullptr;
            cudaDriverEntryPointQueryResult q{};
            if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
                    cudaSuccess ||
                !fn)
                return BSM_ERR_NO_DEVICE;
            g_paged_encode = reinterpret_cast<EncodeTiled>(fn);
        }
        // (the kernels' attributes belong to the current device)
        int prev = -1;
        if (cudaGetDevice(&prev) != cudaSuccess || (prev != device && cudaSetDevice(device) != cudaSuccess))
            return BSM_ERR_NO_DEVICE;
        const int e = paged_set_smem_limit();
        if (prev != device)
            cudaSetDevice(prev);
        if (e)
            return record_cuda_error(e, "cudaFuncSetAttribute(paged)");
        d.ready = true;
    }
    *out = &d;
    return BSM_OK;
}

bool misaligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// [address, end) of a strided array (non-negative strides).
struct Span {
    uintptr_t lo = 0, hi = 0;
    bool meets(const Span &o) const { return lo < o.hi && o.lo < hi; }
};

Span span(const void *p, int64_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes}; }

// A dimension of a strided array, in elements.  The stride of a dimension of one
// entry is never used and may be anything.
struct Dim {
    int64_t n, stride;
};

// Bytes from the first element to the end of the last row (`row` contiguous
// elements) of an array with these dimensions, in any order; -1 when its rows
// overlap or the strides overflow.
template <size_t N> int64_t extent(Dim (&&d)[N], int64_t row, int es)
{
    constexpr int64_t kMost = int64_t(1) << 60;
    std::sort(d, d + N, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    int64_t cur = row;
    for (const Dim &x : d) {
        if (x.n <= 1)
            continue;
        if (x.stride < cur || x.stride > kMost / x.n)
            return -1;
        cur += (x.n - 1) * x.stride;
    }
    return cur < kMost ? cur * es : -1;
}

// Whether two arrays of these dimensions (the first k, by stride; rows apart as extent() asks)
// whose first elements lie `delta` elements apart have a place in common: of the largest stride
// only the two multiples around delta can bring the rest of it within reach.
bool share_a_place(const Dim *d, int k, int64_t row, int64_t delta)
{
    if (k == 0)
        return delta < row && -delta < row;
    const Dim &x = d[k - 1];
    if (x.n <= 1)
        return share_a_place(d, k - 1, row, delta);
    const int64_t at = delta / x.stride - (delta % x.stride < 0);
    for (int64_t i = at; i <= at + 1; ++i)
        if (i < x.n && -i < x.n && share_a_place(d, k - 1, row, delta - i * x.stride))
            return true;
    return false;
}

template <size_t N> bool unaligned(Dim (&&d)[N], int es)
{
    for (const Dim &x : d)
        if (x.n > 1 && x.stride * es % 16)
            return true;
    return false;
}

int elem_size(int dtype) { return dtype == BSM_F32 ? 4 : 2; }

// Workspace: partial outputs, maxima and sums of cut tiles, and who joins them.
struct PagedLayout {
    int64_t rows_o, rows_ml, rows_join, tiles_o, tiles_ml, tiles_join, bytes;
};

PagedLayout paged_layout(int n_sm)
{
    PagedLayout l{};
    auto up = [](int64_t x) { return (x + 255) & ~int64_t(255); };
    const int64_t units = static_cast<int64_t>(n_sm) * kPagedWarps, parts = units * 2 * kPagedRowTile;
    l.rows_o = 0;
    l.rows_ml = l.rows_o + up(parts * kPagedMaxDim * 4);
    l.rows_join = l.rows_ml + up(parts * 8);
    l.tiles_o = l.rows_join + up(units * static_cast<int64_t>(sizeof(PagedJoin)));
    l.tiles_ml = l.tiles_o + up(static_cast<int64_t>(n_sm) * 2 * kPagedTileRows * kPagedMaxDim * 4);
    l.tiles_join = l.tiles_ml + up(static_cast<int64_t>(n_sm) * 2 * kPagedTileRows * 8);
    l.bytes = l.tiles_join + up(static_cast<int64_t>(n_sm) * static_cast<int64_t>(sizeof(PagedJoin)));
    return l;
}

// A tensor map of 16-bit elements with rows of 64 columns and the 128-byte
// swizzle: dims[0] elements contiguous, strides of the others in elements.
// False where the encoder refuses (a stride past its range).
bool paged_map(CUtensorMap *m, bool f16, const void *base, int rank, const int64_t *dims, const int64_t *strides,
               const int *box)
{
    cuuint64_t d[5], s[4];
    cuuint32_t b[5], e[5] = {1u, 1u, 1u, 1u, 1u};
    for (int i = 0; i < rank; ++i) {
        d[i] = static_cast<cuuint64_t>(dims[i]);
        b[i] = static_cast<cuuint32_t>(box[i]);
        // (the stride of a dimension of one entry is never used: any valid one will do)
        if (i > 0)
            s[i - 1] = static_cast<cuuint64_t>(dims[i] > 1 ? strides[i] * 2 : 16);
    }
    return g_paged_encode(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                          static_cast<cuuint32_t>(rank), const_cast<void *>(base), d, s, b, e,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Heads of one key/value head's group that share a tile of at most `rows` rows.
void split_group(PagedArgs &a, int rows)
{
    a.subs = (a.group + rows - 1) / rows;
    a.sub = (a.group + a.subs - 1) / a.subs;
}

bool paged_heads_ok(int32_t hq, int32_t hkv, int32_t d)
{
    return hkv >= 1 && hq >= hkv && hq % hkv == 0 && d >= 8 && d <= kPagedMaxDim && d % 8 == 0;
}

int paged_tables(const bsm_paged_tables_desc *d, bsm_stream_t stream)
{
    if (!d || d->n_requests < 0 || d->n_free < 0 || d->page_size < 1 || d->table_width < 1 || d->n_slots < 0 ||
        d->table_stride < d->table_width)
        return BSM_ERR_INVALID_ARG;
    if (d->table_width >= (1 << 20) || d->n_requests > kPagedMostCount)
        return BSM_ERR_UNSUPPORTED;
    if (!d->starts || !d->info || (d->n_requests > 0 && (!d->cached || !d->fresh || !d->tables || !d->lengths)) ||
        (d->n_free > 0 && !d->free_pages) || (d->n_slots > 0 && (!d->slots || !d->positions || !d->owners)))
        return BSM_ERR_INVALID_ARG;
    if (misaligned(d->slots, 8) || misaligned(d->info, 8) || misaligned(d->cached, 4) || misaligned(d->fresh, 4) ||
        misaligned(d->free_pages, 4) || misaligned(d->tables, 4) || misaligned(d->starts, 4) ||
        misaligned(d->lengths, 4) || misaligned(d->positions, 4) || misaligned(d->owners, 4))
        return BSM_ERR_MISALIGNED;
    const int64_t n = d->n_requests;
    const Span in[3] = {span(d->cached, 4 * n), span(d->fresh, 4 * n), span(d->free_pages, 4ll * d->n_free)};
    const Span out[7] = {span(d->tables, n ? 4 * ((n - 1) * d->table_stride + d->table_width) : 0),
                         span(d->starts, 4 * (n + 1)), span(d->lengths, 4 * n), span(d->slots, 8ll * d->n_slots),
                         span(d->positions, 4ll * d->n_slots), span(d->owners, 4ll * d->n_slots), span(d->info, 32)};
    for (int i = 0; i < 7; ++i) {
        for (int j = i + 1; j < 7; ++j)
            if (out[i].meets(out[j]))
                return BSM_ERR_INVALID_ARG;
        for (const Span &s : in)
            if (out[i].meets(s))
                return BSM_ERR_INVALID_ARG;
    }
    PagedDev *dev = nullptr;
    if (int rc = paged_device(-1, &dev))
        return rc;
    TraceRange tr("bsm_paged_tables");
    PagedTablesArgs a{};
    a.cached = d->cached;
    a.fresh = d->fresh;
    a.free_pages = d->free_pages;
    a.tables = d->tables;
    a.starts = d->starts;
    a.lengths = d->lengths;
    a.slots = d->slots;
    a.positions = d->positions;
    a.owners = d->owners;
    a.info = d->info;
    a.table_stride = d->table_stride;
    a.n = d->n_requests;
    a.n_free = d->n_free;
    a.page = d->page_size;
    a.width = d->table_width;
    a.n_slots = d->n_slots;
    if (int e = launch_paged_tables(a, dev->n_sm, stream))
        return record_cuda_error(e, "paged tables launch");
    return BSM_OK;
}

int paged_write(const bsm_paged_write_desc *d, bsm_stream_t stream)
{
    if (!d || d->n_tokens < 0 || d->n_heads < 1 || d->head_dim < 1 || d->page_size < 1 || d->n_pages < 0 ||
        (d->dtype != BSM_F32 && d->dtype != BSM_BF16 && d->dtype != BSM_F16))
        return BSM_ERR_INVALID_ARG;
    if (d->n_tokens == 0)
        return BSM_OK;
    if (!d->k || !d->v || !d->k_cache || !d->v_cache || !d->slots || d->n_pages == 0)
        return BSM_ERR_INVALID_ARG;
    if (static_cast<int64_t>(d->n_heads) * d->head_dim >= (int64_t(1) << 31))
        return BSM_ERR_UNSUPPORTED;
    const int es = elem_size(d->dtype);
    const int64_t row = static_cast<int64_t>(d->head_dim) * es;
    const int64_t ks = extent({Dim{d->n_tokens, d->k_stride_token}, Dim{d->n_heads, d->k_stride_head}}, d->head_dim, es);
    const int64_t vs = extent({Dim{d->n_tokens, d->v_stride_token}, Dim{d->n_heads, d->v_stride_head}}, d->head_dim, es);
    const int64_t all = extent({Dim{d->n_pages, d->kv_stride_page}, Dim{d->page_size, d->kv_stride_token},
                                Dim{d->n_heads, d->kv_stride_head}},
                               d->head_dim, es);
    if (ks < 0 || vs < 0 || all < 0)
        return BSM_ERR_INVALID_ARG;
    if (row % 16 || misaligned(d->k, 16) || misaligned(d->v, 16) || misaligned(d->k_cache, 16) ||
        misaligned(d->v_cache, 16) || misaligned(d->slots, 8) ||
        unaligned({Dim{d->n_tokens, d->k_stride_token}, Dim{d->n_heads, d->k_stride_head},
                   Dim{d->n_tokens, d->v_stride_token}, Dim{d->n_heads, d->v_stride_head}, Dim{d->n_pages, d->kv_stride_page},
                   Dim{d->page_size, d->kv_stride_token}, Dim{d->n_heads, d->kv_stride_head}},
                  es))
        return BSM_ERR_MISALIGNED;
    const Span kc = span(d->k_cache, all), vc = span(d->v_cache, all), k = span(d->k, ks), v = span(d->v, vs),
               sl = span(d->slots, 8ll * d->n_tokens);
    // (keys and values may be interleaved in one allocation: only equal places clash)
    Dim dims[3] = {Dim{d->n_pages, d->kv_stride_page}, Dim{d->page_size, d->kv_stride_token}, Dim{d->n_heads, d->kv_stride_head}};
    std::sort(dims, dims + 3, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    if ((kc.meets(vc) && share_a_place(dims, 3, d->head_dim, (static_cast<int64_t>(vc.lo) - static_cast<int64_t>(kc.lo)) / es)) ||
        kc.meets(k) || kc.meets(v) || kc.meets(sl) || vc.meets(k) || vc.meets(v) ||
        vc.meets(sl))
        return BSM_ERR_INVALID_ARG;
    PagedDev *dev = nullptr;
    if (int rc = paged_device(-1, &dev))
        return rc;
    TraceRange tr("bsm_paged_write");
    PagedWriteArgs a{};
    a.src[0] = static_cast<const unsigned char *>(d->k);
    a.src[1] = static_cast<const unsigned char *>(d->v);
    a.dst[0] = static_cast<unsigned char *>(d->k_cache);
    a.dst[1] = static_cast<unsigned char *>(d->v_cache);
    a.slots = d->slots;
    a.src_token[0] = d->k_stride_token * es;
    a.src_token[1] = d->v_stride_token * es;
    a.src_head[0] = d->k_stride_head * es;
    a.src_head[1] = d->v_stride_head * es;
    a.dst_page = d->kv_stride_page * es;
    a.dst_token = d->kv_stride_token * es;
    a.dst_head = d->kv_stride_head * es;
    a.n_slots_cache = static_cast<int64_t>(d->n_pages) * d->page_size;
    a.n_tokens = d->n_tokens;
    a.page = d->page_size;
    a.heads = d->n_heads;
    a.chunks = static_cast<int32_t>(row / 16);
    a.status = dev->status;
    if (int e = launch_paged_write(a, dev->n_sm, stream))
        return record_cuda_error(e, "paged write launch");
    return BSM_OK;
}

int paged_attention(const bsm_paged_desc *d, bsm_stream_t stream)
{
    if (!d || d->n_requests < 0 || d->n_tokens < 0 || d->page_size < 1 || d->n_pages < 0 || d->table_width < 1 ||
        d->table_stride < d->table_width || d->max_new < 0 || d->window < 0 || (d->flags & ~BSM_FLAG_CAUSAL) ||
        (d->dtype != BSM_F32 && d->dtype != BSM_BF16 && d->dtype != BSM_F16))
        return BSM_ERR_INVALID_ARG;
    const float scale_log2 = d->scale * 1.4426950408889634f;
    if (!(d->scale > 0.0f) || std::isinf(scale_log2) || (d->window > 0 && !(d->flags & BSM_FLAG_CAUSAL)))
        return BSM_ERR_INVALID_ARG;
    if (d->heads_kv < 1 || d->heads_q < d->heads_kv || d->heads_q % d->heads_kv || d->head_dim < 1)
        return BSM_ERR_INVALID_ARG;
    if (d->dtype == BSM_F32 || !paged_heads_ok(d->heads_q, d->heads_kv, d->head_dim) ||
        d->n_requests > kPagedMostCount || d->n_tokens > kPagedMostCount)
        return BSM_ERR_UNSUPPORTED;
    if (d->n_requests == 0 || d->n_tokens == 0)
        return BSM_OK;
    if (!d->q || !d->k_cache || !d->v_cache || !d->out || !d->starts || !d->lengths || !d->tables || !d->workspace ||
        d->n_pages == 0)
        return BSM_ERR_INVALID_ARG;
    const int64_t qs = extent({Dim{d->n_tokens, d->q_stride_token}, Dim{d->heads_q, d->q_stride_head}}, d->head_dim, 2);
    const int64_t os = extent({Dim{d->n_tokens, d->out_stride_token}, Dim{d->heads_q, d->out_stride_head}}, d->head_dim, 2);
    const int64_t all = extent({Dim{d->n_pages, d->kv_stride_page}, Dim{d->page_size, d->kv_stride_token},
                                Dim{d->heads_kv, d->kv_stride_head}},
                               d->head_dim, 2);
    if (qs < 0 || os < 0 || all < 0)
        return BSM_ERR_INVALID_ARG;
    if (misaligned(d->q, 16) || misaligned(d->k_cache, 16) || misaligned(d->v_cache, 16) || misaligned(d->out, 16) ||
        misaligned(d->lse, 4) || misaligned(d->starts, 4) || misaligned(d->lengths, 4) || misaligned(d->tables, 4) ||
        misaligned(d->workspace, 256) ||
        unaligned({Dim{d->n_tokens, d->q_stride_token}, Dim{d->heads_q, d->q_stride_head},
                   Dim{d->n_tokens, d->out_stride_token}, Dim{d->heads_q, d->out_stride_head},
                   Dim{d->n_pages, d->kv_stride_page}, Dim{d->page_size, d->kv_stride_token},
                   Dim{d->heads_kv, d->kv_stride_head}},
                  2))
        return BSM_ERR_MISALIGNED;
    const int64_t n = d->n_requests;
    const Span o = span(d->out, os), w = span(d->workspace, d->workspace_bytes),
               ls = span(d->lse, d->lse ? 4ll * d->n_tokens * d->heads_q : 0);
    const Span in[6] = {span(d->q, qs), span(d->k_cache, all), span(d->v_cache, all), span(d->starts, 4 * (n + 1)),
                        span(d->lengths, 4 * n), span(d->tables, 4 * ((n - 1) * d->table_stride + d->table_width))};
    for (const Span &s : in)
        if (o.meets(s) || w.meets(s) || ls.meets(s))
            return BSM_ERR_INVALID_ARG;
    if (o.meets(w) || o.meets(ls) || w.meets(ls))
        return BSM_ERR_INVALID_ARG;
    PagedDev *dev = nullptr;
    if (int rc = paged_device(-1, &dev))
        return rc;
    const PagedLayout lay = paged_layout(dev->n_sm);
    if (d->workspace_bytes < lay.bytes)
        return BSM_ERR_INVALID_ARG;
    TraceRange tr("bsm_paged_attention");
    const bool f16 = d->dtype == BSM_F16;
    PagedArgs a{};
    a.q = d->q;
    a.k = d->k_cache;
    a.v = d->v_cache;
    a.out = d->out;
    a.lse = d->lse;
    a.q_token = d->q_stride_token;
    a.q_head = d->q_stride_head;
    a.out_token = d->out_stride_token;
    a.out_head = d->out_stride_head;
    a.kv_page = d->kv_stride_page;
    a.kv_token = d->kv_stride_token;
    a.kv_head = d->kv_stride_head;
    a.starts = d->starts;
    a.lengths = d->lengths;
    a.tables = d->tables;
    a.table_stride = d->table_stride;
    a.n = d->n_requests;
    a.n_tokens = d->n_tokens;
    a.heads_q = d->heads_q;
    a.heads_kv = d->heads_kv;
    a.d = d->head_dim;
    a.page = d->page_size;
    a.n_pages = d->n_pages;
    a.width = d->table_width;
    a.causal = (d->flags & BSM_FLAG_CAUSAL) ? 1 : 0;
    // (a window as long as any request can be hides nothing)
    a.window = d->window < static_cast<int64_t>(d->table_width) * d->page_size ? d->window : 0;
    a.scale_log2 = scale_log2;
    a.group = d->heads_q / d->heads_kv;
    a.status = dev->status;
    unsigned char *ws = static_cast<unsigned char *>(d->workspace);
    // A batch with requests of more than 16 rows (new tokens times the heads that
    // share a key/value head) goes to the tile kernel, its single tokens too: it
    // keeps up with the cache's bytes there, and one launch deals all the work.
    // Pages of whole groups of eight rows come by TMA (box >= 8), others row by row.
    int box = 1;
    while (box < kPagedTileKeys && d->page_size % (2 * box) == 0)
        box *= 2;
    PagedArgs b = a;
    split_group(b, kPagedTileRows / 2);
    b.tok = 2 * (kPagedTileRows / 2 / b.sub);
    CUtensorMap maps[3] = {};
    int per_page = 0;
    bool tiles = static_cast<int64_t>(d->max_new) * a.group > kPagedRowTile;
    if (tiles) {
        const int64_t qd[3] = {d->head_dim, d->heads_q, d->n_tokens}, qst[3] = {1, d->q_stride_head, d->q_stride_token};
        const int qb[3] = {64, b.sub, b.tok / 2};
        // Whole rows of 128 columns a copy, the 64-column halves of eight rows side by
        // side: a map of groups of eight rows, where pages lie whole groups apart.
        const int64_t token = d->kv_stride_token, each = d->page_size / 8;
        if (box >= 8 && d->head_dim == 128 && token > 0) {
            const int64_t apart = d->n_pages == 1 ? each : d->kv_stride_page / (8 * token);
            const int64_t groups = (d->n_pages - 1) * apart + each;
            if (apart >= each && (d->n_pages == 1 || d->kv_stride_page == apart * 8 * token) &&
                groups + apart <= INT32_MAX) {
                const int64_t gd[5] = {64, 8, 2, groups, d->heads_kv};
                const int64_t gst[5] = {1, token, 64, 8 * token, d->kv_stride_head};
                const int gb[5] = {64, 8, 2, box / 8, 1};
                if (paged_map(&maps[1], f16, d->k_cache, 5, gd, gst, gb) &&
                    paged_map(&maps[2], f16, d->v_cache, 5, gd, gst, gb))
                    per_page = static_cast<int>(apart);
            }
        }
        const int64_t kd[4] = {d->head_dim, d->page_size, d->heads_kv, d->n_pages};
        const int64_t kst[4] = {1, d->kv_stride_token, d->kv_stride_head, d->kv_stride_page};
        const int kb[4] = {64, box, 1, 1};
        tiles = paged_map(&maps[0], f16, d->q, 3, qd, qst, qb);
        if (box >= 8 && !per_page &&
            !(paged_map(&maps[1], f16, d->k_cache, 4, kd, kst, kb) && paged_map(&maps[2], f16, d->v_cache, 4, kd, kst, kb)))
            box = 0;
    }
    if (tiles) {
        b.units = dev->n_sm;
        b.min_steps = 1;
        b.part_o = reinterpret_cast<float *>(ws + lay.tiles_o);
        b.part_ml = reinterpret_cast<float *>(ws + lay.tiles_ml);
        b.join = reinterpret_cast<PagedJoin *>(ws + lay.tiles_join);
        if (int e = launch_paged_tiles(maps, b, f16, box, per_page, stream))
            return record_cuda_error(e, "paged attention tile launch");
        return BSM_OK;
    }
    split_group(a, kPagedRowTile);
    a.tok = std::max(1, kPagedRowTile / a.sub);
    a.units = dev->n_sm * kPagedWarps;
    a.min_steps = a.d <= 64 ? 2 : 4;
    a.part_o = reinterpret_cast<float *>(ws + lay.rows_o);
    a.part_ml = reinterpret_cast<float *>(ws + lay.rows_ml);
    a.join = reinterpret_cast<PagedJoin *>(ws + lay.rows_join);
    if (int e = launch_paged_rows(a, f16, dev->n_sm, stream))
        return record_cuda_error(e, "paged attention launch");
    return BSM_OK;
}

}  // namespace
}  // namespace bsm

extern "C" {

int bsm_paged_tables(const bsm_paged_tables_desc *d, bsm_stream_t stream) { return bsm::paged_tables(d, stream); }

int bsm_paged_write(const bsm_paged_write_desc *d, bsm_stream_t stream) { return bsm::paged_write(d, stream); }

int bsm_paged_attention(const bsm_paged_desc *d, bsm_stream_t stream) { return bsm::paged_attention(d, stream); }

int64_t bsm_paged_workspace_bytes(int device, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t max_new)
{
    if (max_new < 0 || !bsm::paged_heads_ok(heads_q, heads_kv, head_dim))
        return -1;
    bsm::PagedDev *dev = nullptr;
    if (bsm::paged_device(device, &dev))
        return -1;
    return bsm::paged_layout(dev->n_sm).bytes;
}

}  // extern "C"
