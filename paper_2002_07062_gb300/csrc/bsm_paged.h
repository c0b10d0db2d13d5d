// bsm_paged.h -- types shared by the paged-cache operators' kernels and their
// host side.  Not part of the public ABI.
#pragma once

#include <cstdint>

#include "../../include/bsm.h"

namespace bsm {

struct PagedTablesArgs {
    const int32_t *cached, *fresh, *free_pages;
    int32_t *tables, *starts, *lengths;
    int64_t *slots;
    int32_t *positions, *owners;
    int64_t *info;
    int64_t table_stride;
    int32_t n, n_free, page, width, n_slots;
};

struct PagedWriteArgs {
    const unsigned char *src[2];        // new keys, new values
    unsigned char *dst[2];              // their caches
    const int64_t *slots;
    int64_t src_token[2], src_head[2];  // strides, bytes
    int64_t dst_page, dst_token, dst_head;
    int64_t n_slots_cache;              // slots the cache holds
    int64_t n_tokens;
    int32_t page, heads, chunks;        // chunks: 16-byte pieces of one head's row
    uint32_t *status;
};

// One kernel's share of bsm_paged_attention: which requests it takes, how their
// rows are tiled and how the work is split over its units (warps or CTAs).
struct PagedArgs {
    const void *q, *k, *v;
    void *out;
    float *lse;                                     // may be null
    int64_t q_token, q_head, out_token, out_head;   // strides, elements
    int64_t kv_page, kv_token, kv_head;
    const int32_t *starts, *lengths, *tables;
    int64_t table_stride;
    int32_t n, n_tokens, heads_q, heads_kv, d, page, n_pages, width;
    int32_t causal, window;                         // window 0: none
    float scale_log2;                               // scale * log2(e)
    // the split
    int32_t group;                                  // query heads of a key/value head
    int32_t subs, sub;                              // head groups of one key/value head, heads of each
    int32_t tok;                                    // tokens of a tile
    int32_t units, min_steps;                       // units at most; key steps of a unit at least
    float *part_o;                                  // units x 2 x tile rows x kPagedMaxDim
    float *part_ml;                                 // units x 2 x tile rows x 2
    struct PagedJoin *join;                         // units
    uint32_t *status;
};

// A tile whose keys were split over units u .. u + count - 1: the first one's
// second partial and the others' first are joined.
struct PagedJoin {
    int32_t token, head, tokens, heads;             // first token, first query head, tokens, heads of the tile
    int32_t count;                                  // 0: nothing to join
    // of the whole unit: the first tile that it starts, the tiles that it has whole from there
    uint32_t flags;                                 // kPaged*
    int32_t r, head0, tile, whole;
    int32_t pad[2];
};
constexpr uint32_t kPagedGone = 1;                  // it met a key whose page is not there
constexpr uint32_t kPagedOdd = 2;                   // an output that it stored is not finite

constexpr int32_t kPagedMostKeys = INT32_MAX - 255; // of a request: a step past them is still a 32-bit number
constexpr int32_t kPagedMostCount = INT32_MAX - 4095;   // requests, and tokens of attention: a block past them likewise
constexpr int kPagedWarps = 8;                      // of the row kernel
constexpr int kPagedRowTile = 16;                   // most rows of its tiles
constexpr int kPagedMaxDim = 128;
constexpr int kPagedTileRows = 256;                 // of the tile kernel: two blocks of 128
constexpr int kPagedTileKeys = 128;                 // keys of its steps

int launch_paged_tables(const PagedTablesArgs &a, int n_sm, void *stream);
int launch_paged_write(const PagedWriteArgs &a, int n_sm, void *stream);
int launch_paged_rows(const PagedArgs &a, bool f16, int grid, void *stream);
// maps: CUtensorMaps of q, k, v (host); box: rows of one copy of k and v (below 8:
// those maps are not used); per_page: 0, or whole rows a copy, with the maps' fourth
// dimension counting groups of eight rows, per_page of them from page to page
int launch_paged_tiles(const void *maps, const PagedArgs &a, bool f16, int box, int per_page, void *stream);
int paged_set_smem_limit();

}  // namespace bsm
