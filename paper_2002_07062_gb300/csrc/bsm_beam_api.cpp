// bsm_beam_api.cpp -- C ABI of the beam operators: argument checks and the
// workspaces' layouts.

#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "bsm_beam.h"
#include "bsm_internal.h"
#include "bsm_paged.h"
#include "bsm_paged_host.h"
#include "bsm_trace.h"

namespace bsm {
namespace {

int64_t up256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct SelectLayout {
    int32_t parts, part;
    int64_t meta, bytes;
};

SelectLayout select_layout(int64_t rows, int32_t vocab, int32_t keep, int es, int n_sm)
{
    SelectLayout l{};
    beam_parts(rows, vocab, es, n_sm, &l.parts, &l.part);
    const int64_t lists = rows * l.parts;
    l.meta = up256(lists * keep * static_cast<int64_t>(sizeof(BeamEntry)));
    l.bytes = l.meta + up256(lists * static_cast<int64_t>(sizeof(BeamPart)));
    return l;
}

bool select_sizes(int32_t n, int32_t beams, int32_t vocab, int32_t keep)
{
    return n >= 0 && beams >= 1 && vocab >= 1 && keep >= 1;
}

bool select_limits(int32_t n, int32_t beams, int32_t vocab, int32_t keep)
{
    return beams <= kBeamMost && keep <= kBeamMost && vocab <= kBeamMostVocab &&
           static_cast<int64_t>(n) * beams * kBeamMostParts <= INT32_MAX;
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
    const SelectLayout l = select_layout(rows, d->vocab, d->keep, es, dev->n_sm);
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
    a.parts = l.parts;
    a.part = l.part;
    if (int e = launch_beam_select(a, d->dtype, stream))
        return record_cuda_error(e, "beam select launch");
    return BSM_OK;
}

}  // namespace
}  // namespace bsm

extern "C" {

int bsm_beam_select(const bsm_beam_select_desc *d, bsm_stream_t stream) { return bsm::beam_select(d, stream); }

int64_t bsm_beam_select_workspace_bytes(int device, int32_t n_requests, int32_t beams, int32_t vocab, int32_t keep)
{
    if (!bsm::select_sizes(n_requests, beams, vocab, keep) || !bsm::select_limits(n_requests, beams, vocab, keep))
        return -1;
    bsm::PagedDev *dev = nullptr;
    if (bsm::paged_device(device, &dev))
        return -1;
    const int64_t rows = static_cast<int64_t>(n_requests) * beams;
    return std::max(bsm::select_layout(rows, vocab, keep, 2, dev->n_sm).bytes,
                    bsm::select_layout(rows, vocab, keep, 4, dev->n_sm).bytes);
}

}  // extern "C"
