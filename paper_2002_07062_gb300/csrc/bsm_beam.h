// bsm_beam.h -- types shared by the beam operators' kernels and their host side.
// Not part of the public ABI.
#pragma once

#include <cstdint>

#include "../../include/bsm.h"

namespace bsm {

constexpr int kBeamMost = 64;                   // beams of a request, and continuations kept
constexpr int32_t kBeamMostVocab = 1 << 20;
constexpr int kBeamThreads = 512;               // of a part of a row
constexpr int kBeamLoads = 4;                   // pieces of 16 bytes that a thread holds
constexpr int kBeamMostParts = 128;             // of a row: kBeamMostVocab fp32 logits

// The best logits of a part of a row, and what its softmax needs.
struct BeamPart {
    double sum;                                 // of exp(x - top)
    float top;
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
    int32_t parts, part;                        // parts of a row, logits of each
};

// How rows of `vocab` logits are cut: *parts of *part logits (whole pieces of 16 bytes).
void beam_parts(int64_t rows, int32_t vocab, int es, int n_sm, int32_t *parts, int32_t *part);

int launch_beam_select(const BeamSelectArgs &a, int dtype, void *stream);
int beam_set_smem_limit();

}  // namespace bsm
