// bsm_paged_host.h -- what the host sides of the paged-cache and beam operators
// share: the device's state, spans of strided arrays and their overlaps.  Not
// part of the public ABI.
#pragma once

#include <algorithm>
#include <cstdint>

#include "../../include/bsm.h"

namespace bsm {

struct PagedDev {
    bool ready = false;
    int n_sm = 0;
    uint32_t *status = nullptr;
    bool clusters = false;              // the beam selection's clusters can be placed (see beam_cut)
};

int device_status_word(int device, uint32_t **out);

// The state of `device` (-1: current), set up on its first call.
int paged_device(int device, PagedDev **out);

inline bool misaligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// [address, end) of a strided array (non-negative strides).
struct Span {
    uintptr_t lo = 0, hi = 0;
    bool meets(const Span &o) const { return lo < o.hi && o.lo < hi; }
};

inline Span span(const void *p, int64_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes}; }

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
inline bool share_a_place(const Dim *d, int k, int64_t row, int64_t delta)
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

// The same for two arrays of tokens x heads rows of `row` elements, heads na and nb; true too
// where their strides differ (whoever asks has seen that their spans meet).
inline bool heads_share_a_place(int64_t tokens, int64_t token_a, int64_t head_a, int64_t na, int64_t token_b,
                                int64_t head_b, int64_t nb, int64_t row, int64_t delta)
{
    if ((tokens > 1 && token_a != token_b) || (na > 1 && nb > 1 && head_a != head_b))
        return true;
    // (differences of indices: i of a less j of b)
    struct Range {
        int64_t lo, hi, stride;
    } d[2] = {{1 - nb, na - 1, na > 1 ? head_a : head_b}, {1 - tokens, tokens - 1, token_a}};
    if (tokens > 1 && (na > 1 || nb > 1) && d[1].stride < d[0].stride)
        std::swap(d[0], d[1]);
    // of the larger stride only the two multiples around delta come within reach
    auto near_ = [](const Range &r, int64_t x, int64_t *out) {
        if (r.lo == 0 && r.hi == 0) {
            out[0] = out[1] = x;
            return 1;
        }
        const int64_t at = x / r.stride - (x % r.stride < 0);
        int n = 0;
        for (int64_t i = at; i <= at + 1; ++i)
            if (i >= r.lo && i <= r.hi)
                out[n++] = x - i * r.stride;
        return n;
    };
    int64_t a[2], b[2];
    for (int n = near_(d[1], delta, a); n > 0; --n)
        for (int m = near_(d[0], a[n - 1], b); m > 0; --m)
            if (b[m - 1] < row && -b[m - 1] < row)
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

inline int elem_size(int dtype) { return dtype == BSM_F32 ? 4 : 2; }

}  // namespace bsm
