// bsm_beam.h -- types shared by the beam operators' kernels and their host side.
// Not part of the public ABI.
#pragma once

#include <climits>
#include <cstdint>

#include "../../include/bsm.h"

namespace bsm {

constexpr int kBeamMost = 64;                   // beams of a request, and continuations kept
constexpr int32_t kBeamMostVocab = 1 << 20;
constexpr int64_t kBeamMostRows = (1 << 24) - 1;
constexpr int kBeamLoads = 4;                   // pieces of 16 bytes that a thread holds
constexpr int kBeamMostLists = 128;             // parts of all rows of a request
constexpr int64_t kTogetherBytes = 128 << 10;   // of logits that a CTA of a cluster reads at most

// The best logits of a part of a row, and what its softmax needs.
struct BeamPart {
    float sum, rest;                            // of exp(x - top): two numbers that add up to it
    float top;                                  // one of the part's largest values
    int32_t count;                              // entries in its list
};
struct BeamEntry {
    float x;
    int32_t token;
};

struct BeamSelectArgs {
    const unsigned char *logits;
    const float *scores;
    const uint8_t *ended;                       // may be null
    float *out_scores;
    int32_t *parents, *tokens;
    BeamEntry *entries;                         // a list of `keep` for each part of each row
    BeamPart *meta;
    int64_t stride_request, stride_beam;        // bytes
    int32_t n, beams, vocab, keep, end_token;
    int32_t parts, part;                        // parts of a row, logits of each (whole pieces of 16 bytes)
    int32_t list;                               // entries of a part's list (set by the launch)
};

constexpr int kReorderTile = 128;               // columns of the tables that a CTA takes
constexpr int64_t kReorderMost = INT32_MAX;     // requests x tiles, and pieces of 16 bytes of a page

struct PagedReorderArgs {
    const int32_t *parents, *lengths, *tables, *free_pages;
    int32_t *new_lengths, *new_tables, *dropped;
    int64_t *info;
    unsigned char *cache[2];
    int64_t layer, page_bytes, token, head;     // strides of the caches, bytes
    int64_t parent_stride, table_stride, new_table_stride;
    // workspace: per row its new length and the page that it copies from; per request and
    // tile the rows that copy (a bit each) and the pages that it dropped
    int32_t *row_length, *row_source;
    uint64_t *copies;
    int32_t *counts, *lists;
    int32_t n, beams, width, tiles, n_free, n_dropped, page, n_pages, heads, chunks, layers;
    int32_t listers;                            // CTAs of the second launch for the dropped pages (set by it)
    uint32_t *status;
};

int launch_paged_reorder(PagedReorderArgs a, int n_sm, void *stream);

// How the rows are cut: parts of `part` logits.
struct BeamCut {
    int32_t parts, part;
    bool together;                              // a cluster takes a request, in one launch
};
// Lists that any cut of at most `rows` rows makes, whatever the vocabulary.
int64_t beam_most_lists(int64_t rows, int n_sm);
BeamCut beam_cut(int32_t n, int32_t beams, int32_t vocab, int es, int n_sm, bool clusters);

int launch_beam_select(BeamSelectArgs a, int dtype, const BeamCut &cut, void *stream);
int beam_set_smem_limit();
// Whether the current device places a cluster of the one-launch form at its largest (after beam_set_smem_limit).
bool beam_clusters_fit();

}  // namespace bsm
