// bsm_beam_api.cpp -- C ABI of the beam operators: argument checks and the
// workspaces' layouts.

#include <cuda_runtime.h>

#include <algorithm>
#include <climits>

#include "bsm_beam.h"
#include "bsm_internal.h"
#include "bsm_paged.h"
#include "bsm_paged_host.h"
#include "bsm_trace.h"

namespace bsm {
namespace {

int64_t up256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct SelectLayout {
    BeamCut cut;
    int64_t meta, bytes;
};

int64_t entries_bytes(int64_t lists, int32_t keep) { return up256(lists * keep * static_cast<int64_t>(sizeof(BeamEntry))); }
int64_t meta_bytes(int64_t lists) { return up256(lists * static_cast<int64_t>(sizeof(BeamPart))); }

SelectLayout select_layout(int32_t n, int32_t beams, int32_t vocab, int32_t keep, int es, const PagedDev &dev)
{
    SelectLayout l{};
    l.cut = beam_cut(n, beams, vocab, es, dev.n_sm, dev.clusters);
    const int64_t lists = static_cast<int64_t>(n) * beams * l.cut.parts;        // (a cluster's are in shared memory)
    l.meta = entries_bytes(lists, keep);
    l.bytes = l.meta + meta_bytes(lists);
    return l;
}

bool select_sizes(int32_t n, int32_t beams, int32_t vocab, int32_t keep)
{
    return n >= 0 && beams >= 1 && vocab >= 1 && keep >= 1;
}

bool select_limits(int32_t n, int32_t beams, int32_t vocab, int32_t keep)
{
    return beams <= kBeamMost && keep <= kBeamMost && vocab <= kBeamMostVocab &&
           static_cast<int64_t>(n) * beams <= kBeamMostRows;
}

int beam_select(const bsm_beam_select_desc *d, bsm_stream_t stream)
{
    if (!d || !select_sizes(d->n_requests, d->beams, d->vocab, d->keep) || d->stride_request < 0 || d->stride_beam < 0 ||
        (d->dtype != BSM_F32 && d->dtype != BSM_BF16 && d->dtype != BSM_F16) ||
        (d->ended && (d->end_token < 0 || d->end_token >= d->vocab)))
        return BSM_ERR_INVALID_ARG;
    if (!select_limits(d->n_requests, d->beams, d->vocab, d->keep))
        return BSM_ERR_UNSUPPORTED;
    if (d->n_requests == 0)
        return BSM_OK;
    if (!d->logits || !d->scores || !d->out_scores || !d->parents || !d->tokens || !d->workspace)
        return BSM_ERR_INVALID_ARG;
    constexpr int64_t kMost = int64_t(1) << 60;
    const int64_t n = d->n_requests, rows = n * d->beams;
    const int es = elem_size(d->dtype);
    if (d->stride_request > kMost / n || d->stride_beam > kMost / d->beams)
        return BSM_ERR_INVALID_ARG;
    const int64_t all = (n - 1) * d->stride_request + (d->beams - 1) * d->stride_beam + d->vocab;
    if (misaligned(d->logits, es) || misaligned(d->scores, 4) || misaligned(d->out_scores, 4) || misaligned(d->parents, 4) ||
        misaligned(d->tokens, 4) || misaligned(d->workspace, 256))
        return BSM_ERR_MISALIGNED;
    const Span in[3] = {span(d->logits, all * es), span(d->scores, 4 * rows), span(d->ended, d->ended ? rows : 0)};
    const Span out[4] = {span(d->out_scores, 4 * n * d->keep), span(d->parents, 4 * n * d->keep),
                         span(d->tokens, 4 * n * d->keep), span(d->workspace, std::max<int64_t>(d->workspace_bytes, 0))};
    for (int i = 0; i < 4; ++i) {
        for (int j = i + 1; j < 4; ++j)
            if (out[i].meets(out[j]))
                return BSM_ERR_INVALID_ARG;
        for (const Span &s : in)
            if (out[i].meets(s))
                return BSM_ERR_INVALID_ARG;
    }
    PagedDev *dev = nullptr;
    if (int rc = paged_device(-1, &dev))
        return rc;
    const SelectLayout l = select_layout(d->n_requests, d->beams, d->vocab, d->keep, es, *dev);
    if (d->workspace_bytes < l.bytes)
        return BSM_ERR_INVALID_ARG;
    TraceRange tr("bsm_beam_select");
    BeamSelectArgs a{};
    a.logits = static_cast<const unsigned char *>(d->logits);
    a.scores = d->scores;
    a.ended = d->ended;
    a.out_scores = d->out_scores;
    a.parents = d->parents;
    a.tokens = d->tokens;
    unsigned char *ws = static_cast<unsigned char *>(d->workspace);
    a.entries = reinterpret_cast<BeamEntry *>(ws);
    a.meta = reinterpret_cast<BeamPart *>(ws + l.meta);
    a.stride_request = d->stride_request * es;
    a.stride_beam = d->stride_beam * es;
    a.n = d->n_requests;
    a.beams = d->beams;
    a.vocab = d->vocab;
    a.keep = d->keep;
    a.end_token = d->end_token;
    if (int e = launch_beam_select(a, d->dtype, l.cut, stream))
        return record_cuda_error(e, "beam select launch");
    return BSM_OK;
}

struct ReorderLayout {
    int64_t tiles, source, copies, counts, lists, bytes;
};

ReorderLayout reorder_layout(int64_t n, int32_t beams, int32_t width)
{
    ReorderLayout l{};
    l.tiles = (width + kReorderTile - 1) / kReorderTile;
    l.source = up256(4 * n * beams);
    l.copies = l.source + up256(4 * n * beams);
    l.counts = l.copies + up256(8 * n * l.tiles);
    l.lists = l.counts + up256(4 * n * l.tiles);
    l.bytes = l.lists + up256(4 * n * l.tiles * kReorderTile * beams);
    return l;
}

bool reorder_sizes(int32_t n, int32_t beams, int32_t width) { return n >= 0 && beams >= 1 && width >= 1; }

bool reorder_limits(int32_t n, int32_t beams, int32_t width)
{
    return beams <= kBeamMost && width < (1 << 20) && static_cast<int64_t>(n) * beams <= kPagedMostCount &&
           n * ((static_cast<int64_t>(width) + kReorderTile - 1) / kReorderTile) <= kReorderMost;
}

int paged_reorder(const bsm_paged_reorder_desc *d, bsm_stream_t stream)
{
    if (!d || !reorder_sizes(d->n_requests, d->beams, d->table_width) || d->n_free < 0 || d->n_dropped < 0 ||
        d->page_size < 1 || d->n_layers < 1 || d->n_pages < 0 || d->n_heads < 1 || d->head_dim < 1 ||
        d->parent_stride < 0 || d->table_stride < d->table_width || d->new_table_stride < d->table_width ||
        (d->dtype != BSM_F32 && d->dtype != BSM_BF16 && d->dtype != BSM_F16))
        return BSM_ERR_INVALID_ARG;
    const int es = elem_size(d->dtype);
    const int64_t row = static_cast<int64_t>(d->head_dim) * es;
    if (!reorder_limits(d->n_requests, d->beams, d->table_width) ||
        row / 16 * d->n_heads > kReorderMost / d->page_size || d->n_layers > (1 << 20))
        return BSM_ERR_UNSUPPORTED;
    if (!d->info || (d->n_requests > 0 && (!d->parents || !d->lengths || !d->tables || !d->new_lengths || !d->new_tables ||
                                           !d->k_cache || !d->v_cache || !d->workspace || d->n_pages == 0)) ||
        (d->n_free > 0 && !d->free_pages) || (d->n_dropped > 0 && !d->dropped))
        return BSM_ERR_INVALID_ARG;
    constexpr int64_t kMost = int64_t(1) << 60;
    const int64_t n = d->n_requests, rows = n * d->beams;
    if (n > 0 && (d->parent_stride > kMost / n || d->table_stride > kMost / rows || d->new_table_stride > kMost / rows))
        return BSM_ERR_INVALID_ARG;
    Dim dims[4] = {Dim{d->n_layers, d->kv_stride_layer}, Dim{d->n_pages, d->kv_stride_page},
                   Dim{d->page_size, d->kv_stride_token}, Dim{d->n_heads, d->kv_stride_head}};
    const int64_t all = n ? extent({dims[0], dims[1], dims[2], dims[3]}, d->head_dim, es) : 0;
    if (all < 0)
        return BSM_ERR_INVALID_ARG;
    if (misaligned(d->parents, 4) || misaligned(d->lengths, 4) || misaligned(d->tables, 4) || misaligned(d->free_pages, 4) ||
        misaligned(d->new_lengths, 4) || misaligned(d->new_tables, 4) || misaligned(d->dropped, 4) || misaligned(d->info, 8))
        return BSM_ERR_MISALIGNED;
    if (n && (row % 16 || misaligned(d->k_cache, 16) || misaligned(d->v_cache, 16) || misaligned(d->workspace, 256) ||
              unaligned({dims[0], dims[1], dims[2], dims[3]}, es)))
        return BSM_ERR_MISALIGNED;
    const int64_t tables = n ? 4 * ((rows - 1) * d->table_stride + d->table_width) : 0;
    const int64_t new_tables = n ? 4 * ((rows - 1) * d->new_table_stride + d->table_width) : 0;
    const Span in[4] = {span(d->parents, n ? 4 * ((n - 1) * d->parent_stride + d->beams) : 0), span(d->free_pages, 4ll * d->n_free),
                        span(d->lengths, 4 * rows), span(d->tables, tables)};
    const Span out[7] = {span(d->new_lengths, 4 * rows), span(d->new_tables, new_tables), span(d->dropped, 4ll * d->n_dropped),
                         span(d->info, 32), span(d->workspace, n ? std::max<int64_t>(d->workspace_bytes, 0) : 0),
                         span(d->k_cache, all), span(d->v_cache, all)};
    // lengths and tables may change in place
    const bool same_lengths = d->new_lengths == d->lengths;
    const bool same_tables = d->new_tables == d->tables && (rows <= 1 || d->new_table_stride == d->table_stride);
    for (int i = 0; i < 7; ++i) {
        for (int j = i + 1; j < 7; ++j)
            if (out[i].meets(out[j]) && !(i == 5 && j == 6))
                return BSM_ERR_INVALID_ARG;
        for (int j = 0; j < 4; ++j)
            if (out[i].meets(in[j]) && !(i == 0 && j == 2 && same_lengths) && !(i == 1 && j == 3 && same_tables))
                return BSM_ERR_INVALID_ARG;
    }
    std::sort(dims, dims + 4, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    if (n && out[5].meets(out[6]) &&
        share_a_place(dims, 4, d->head_dim, (static_cast<int64_t>(out[6].lo) - static_cast<int64_t>(out[5].lo)) / es))
        return BSM_ERR_INVALID_ARG;
    PagedDev *dev = nullptr;
    if (int rc = paged_device(-1, &dev))
        return rc;
    const ReorderLayout l = reorder_layout(n, d->beams, d->table_width);
    if (n && d->workspace_bytes < l.bytes)
        return BSM_ERR_INVALID_ARG;
    TraceRange tr("bsm_paged_reorder");
    PagedReorderArgs a{};
    a.parents = d->parents;
    a.lengths = d->lengths;
    a.tables = d->tables;
    a.free_pages = d->free_pages;
    a.new_lengths = d->new_lengths;
    a.new_tables = d->new_tables;
    a.dropped = d->dropped;
    a.info = d->info;
    a.cache[0] = static_cast<unsigned char *>(d->k_cache);
    a.cache[1] = static_cast<unsigned char *>(d->v_cache);
    a.layer = d->kv_stride_layer * es;
    a.page_bytes = d->kv_stride_page * es;
    a.token = d->kv_stride_token * es;
    a.head = d->kv_stride_head * es;
    a.parent_stride = d->parent_stride;
    a.table_stride = d->table_stride;
    a.new_table_stride = d->new_table_stride;
    unsigned char *ws = static_cast<unsigned char *>(d->workspace);
    a.row_length = reinterpret_cast<int32_t *>(ws);
    a.row_source = reinterpret_cast<int32_t *>(ws + l.source);
    a.copies = reinterpret_cast<uint64_t *>(ws + l.copies);
    a.counts = reinterpret_cast<int32_t *>(ws + l.counts);
    a.lists = reinterpret_cast<int32_t *>(ws + l.lists);
    a.n = d->n_requests;
    a.beams = d->beams;
    a.width = d->table_width;
    a.tiles = static_cast<int32_t>(l.tiles);
    a.n_free = d->n_free;
    a.n_dropped = d->n_dropped;
    a.page = d->page_size;
    a.n_pages = d->n_pages;
    a.heads = d->n_heads;
    a.chunks = static_cast<int32_t>(row / 16);
    a.layers = d->n_layers;
    a.status = dev->status;
    if (int e = launch_paged_reorder(a, dev->n_sm, stream))
        return record_cuda_error(e, "paged reorder launch");
    return BSM_OK;
}

}  // namespace
}  // namespace bsm

extern "C" {

int bsm_paged_reorder(const bsm_paged_reorder_desc *d, bsm_stream_t stream) { return bsm::paged_reorder(d, stream); }

int64_t bsm_paged_reorder_workspace_bytes(int32_t n_requests, int32_t beams, int32_t table_width)
{
    if (!bsm::reorder_sizes(n_requests, beams, table_width) || !bsm::reorder_limits(n_requests, beams, table_width))
        return -1;
    return bsm::reorder_layout(n_requests, beams, table_width).bytes;
}

int bsm_beam_select(const bsm_beam_select_desc *d, bsm_stream_t stream) { return bsm::beam_select(d, stream); }

int64_t bsm_beam_select_workspace_bytes(int device, int32_t n_requests, int32_t beams, int32_t vocab, int32_t keep)
{
    if (!bsm::select_sizes(n_requests, beams, vocab, keep) || !bsm::select_limits(n_requests, beams, vocab, keep))
        return -1;
    bsm::PagedDev *dev = nullptr;
    if (bsm::paged_device(device, &dev))
        return -1;
    // (enough for fewer requests too, which may be cut into more parts)
    const int64_t lists = bsm::beam_most_lists(static_cast<int64_t>(n_requests) * beams, dev->n_sm);
    return bsm::entries_bytes(lists, keep) + bsm::meta_bytes(lists);
}

}  // extern "C"
