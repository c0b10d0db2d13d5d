// bsm_paged_rotary.cu -- new keys and values to their slots of a paged cache,
// the keys (and the queries beside them) rotated by their positions on the way.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotHeads = 8;            // heads of a thread, where there are threads enough

// CTAs of an instance on an SM, as its registers allow.
template <int kBytes, bool kSide> constexpr int fit() { return kBytes < 16 ? 4 : kSide ? 3 : 2; }

template <int kBytes> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<2> { using type = uint16_t; };

// W values of a type and the fp32 numbers they stand for.
template <int kType, int kBytes> struct Values {
    static constexpr int W = kBytes / (kType == BSM_F32 ? 4 : 2);
    using Raw = typename RawOf<kBytes>::type;
    union Bits {
        Raw raw;
        float f[W];
        __nv_bfloat16 b[W];
        __half h[W];
        __device__ Bits() {}
    };
    static __device__ __forceinline__ void get(const Raw &r, float (&x)[W])
    {
        Bits v;
        v.raw = r;
#pragma unroll
        for (int i = 0; i < W; ++i)
            x[i] = kType == BSM_F32 ? v.f[i] : kType == BSM_BF16 ? __bfloat162float(v.b[i]) : __half2float(v.h[i]);
    }
    static __device__ __forceinline__ Raw put(const float (&x)[W])
    {
        Bits v;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (kType == BSM_F32)
                v.f[i] = x[i];
            else if (kType == BSM_BF16)
                v.b[i] = __float2bfloat16_rn(x[i]);
            else
                v.h[i] = __float2half_rn(x[i]);
        }
        return v.raw;
    }
};

// A unit of `pairs` pairs side by side of which the first `turned` are taken from x and the others
// from `as_it_was`, bit for bit (a NaN would not come back from fp32 with its own bits).
__device__ __forceinline__ uint4 first_pairs(const uint4 &x, const uint4 &as_it_was, int turned, int pairs)
{
    const int words = turned * 4 / pairs;               // (a pair is one word or two)
    return make_uint4(words > 0 ? x.x : as_it_was.x, words > 1 ? x.y : as_it_was.y, words > 2 ? x.z : as_it_was.z,
                      words > 3 ? x.w : as_it_was.w);
}

template <int N> __device__ __forceinline__ void load_floats(const float *p, bool wide, float (&x)[N])
{
    if (N % 4 == 0 && wide) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 v = reinterpret_cast<const float4 *>(p)[i];
            x[4 * i] = v.x;
            x[4 * i + 1] = v.y;
            x[4 * i + 2] = v.z;
            x[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = p[i];
    }
}

// (x1, x2) of a pair becomes (x1 cos - x2 sin, x2 cos + x1 sin), in fp32, rounded once.
// A thread takes one unit (W columns; with the pairs half a head apart, W and their
// partners) of kHeads heads of one tensor and token: it reads its cosines and sines once
// for all of them and has all their loads in flight.  Bound by the bytes.  40 thousand tokens of 32 + 8 + 8
// heads of 128, bf16, 1.13 GB: 168 us, 6.7 TB/s, 0.99 of a copy's rate (2 heads a thread 208, 4 186; a third more
// CTAs than two whole waves 181, a block each 249).  Few tokens take a head a thread: one token 1.9 us
// of GPU time, 256 tokens 2.8.
template <int kType, int kBytes, bool kSide, int kHeads>
__global__ void __launch_bounds__(kRotThreads, fit<kBytes, kSide>()) paged_rotary(const PagedRotaryArgs a)
{
    using V = Values<kType, kBytes>;
    using Raw = typename V::Raw;
    constexpr int W = V::W, kEs = kBytes / W;
    grid_dependency_wait();
    grid_launch_dependents();
    const uint64_t all = static_cast<uint64_t>(a.n_tokens) * a.per_token;
    for (uint64_t x = static_cast<uint64_t>(blockIdx.x) * kRotThreads + threadIdx.x; x < all;
         x += static_cast<uint64_t>(gridDim.x) * kRotThreads) {
        const uint32_t t = static_cast<uint32_t>(__umul64hi(x, a.by_token));
        uint32_t y = static_cast<uint32_t>(x - static_cast<uint64_t>(t) * a.per_token);
        const int32_t pos = a.positions[t];
        const int64_t slot = a.slots[t];
        if (pos < 0)
            continue;
        if (pos >= a.n_positions || slot >= a.n_slots_cache)
            atomicOr(a.status, BSM_DEV_BOUNDS);
        if (pos >= a.n_positions)
            continue;
        const bool value = y >= a.of_qk;
        if (value)
            y -= a.of_qk;
        const uint32_t per = value ? a.units_v : a.units;
        uint32_t g = __umulhi(y, value ? a.by_units_v : a.by_units);
        if (per == 1)
            g = y;
        const int32_t u = static_cast<int32_t>(y - g * per);
        const bool query = !value && g < static_cast<uint32_t>(a.groups_q);
        const int which = value ? 2 : query ? 0 : 1;
        if (!value && !query)
            g -= a.groups_q;
        const int32_t head = static_cast<int32_t>(g) * kHeads;
        const int32_t n = min(kHeads, (query ? a.heads_q : a.heads_kv) - head);
        const int64_t sh = which == 0 ? a.src_head[0] : which == 1 ? a.src_head[1] : a.src_head[2];
        const unsigned char *src = (which == 0 ? a.src[0] : which == 1 ? a.src[1] : a.src[2]) +
                                   t * (which == 0 ? a.src_token[0] : which == 1 ? a.src_token[1] : a.src_token[2]) +
                                   head * sh;
        unsigned char *dst;
        const int64_t dh = query ? a.out_head : a.dst_head;
        if (query) {
            dst = a.dst[0] + t * a.out_token + head * dh;
        } else {
            if (slot < 0 || slot >= a.n_slots_cache)
                continue;
            const int64_t page = pg_div(slot, a.page);
            dst = (value ? a.dst[2] : a.dst[1]) + page * a.dst_page + (slot - page * a.page) * a.dst_token + head * dh;
        }
        Raw lo[kHeads];
        if (value || u >= a.turned) {
            // as it is, bit for bit
            const int32_t col = value || kSide ? u * W : 2 * a.half + (u - a.turned) * W;
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                if (i < n)
                    lo[i] = *reinterpret_cast<const Raw *>(src + i * sh + col * kEs);
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                if (i < n)
                    *reinterpret_cast<Raw *>(dst + i * dh + col * kEs) = lo[i];
            continue;
        }
        const float *row = a.table + pos * a.table_stride;
        if constexpr (kSide) {
            const int32_t col = u * W;
            constexpr int N = W > 1 ? W / 2 : 1;
            float c[N], s[N];
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                if (i < n)
                    lo[i] = *reinterpret_cast<const Raw *>(src + i * sh + col * kEs);
            const int32_t first = u * N;
            if (first + N <= a.half) {
                load_floats<N>(row + first, a.wide_table, c);
                load_floats<N>(row + a.half + first, a.wide_table, s);
            } else {
                // the last unit: its columns past the rotated ones stay (see first_pairs)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    c[i] = first + i < a.half ? row[first + i] : 1.0f;
                    s[i] = first + i < a.half ? row[a.half + first + i] : 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < kHeads; ++i) {
                if (i >= n)
                    continue;
                float v[W], r[W];
                V::get(lo[i], v);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float p = v[2 * j], q = v[(2 * j + 1) % W];
                    r[2 * j] = __fmaf_rn(p, c[j], -(q * s[j]));
                    r[(2 * j + 1) % W] = __fmaf_rn(q, c[j], p * s[j]);
                }
                *reinterpret_cast<Raw *>(dst + i * dh + col * kEs) = first_pairs(V::put(r), lo[i], a.half - first, N);
            }
        } else {
            Raw hi[kHeads];
            const int32_t col = u * W, far = a.half + col;
            float c[W], s[W];
#pragma unroll
            for (int i = 0; i < kHeads; ++i)
                if (i < n) {
                    lo[i] = *reinterpret_cast<const Raw *>(src + i * sh + col * kEs);
                    hi[i] = *reinterpret_cast<const Raw *>(src + i * sh + far * kEs);
                }
            load_floats<W>(row + col, a.wide_table, c);
            load_floats<W>(row + far, a.wide_table, s);
#pragma unroll
            for (int i = 0; i < kHeads; ++i) {
                if (i >= n)
                    continue;
                float p[W], q[W], r[W];
                V::get(lo[i], p);
                V::get(hi[i], q);
#pragma unroll
                for (int j = 0; j < W; ++j)
                    r[j] = __fmaf_rn(p[j], c[j], -(q[j] * s[j]));
                *reinterpret_cast<Raw *>(dst + i * dh + col * kEs) = V::put(r);
#pragma unroll
                for (int j = 0; j < W; ++j)
                    r[j] = __fmaf_rn(q[j], c[j], p[j] * s[j]);
                *reinterpret_cast<Raw *>(dst + i * dh + far * kEs) = V::put(r);
            }
        }
    }
}

uint32_t reciprocal(uint32_t d) { return static_cast<uint32_t>(((uint64_t(1) << 32) + d - 1) / d); }    // d > 1

template <int kType, int kBytes, bool kSide> int launch(PagedRotaryArgs a, int n_sm, void *stream)
{
    constexpr int W = Values<kType, kBytes>::W;
    a.units_v = a.dim / W;
    a.units = kSide ? a.dim / W : a.half / W + (a.dim - 2 * a.half) / W;
    a.turned = kSide ? (2 * a.half + W - 1) / W : a.half / W;
    a.by_units = a.units > 1 ? reciprocal(a.units) : 0;
    a.by_units_v = a.units_v > 1 ? reciprocal(a.units_v) : 0;
    auto deal = [&](int heads) {
        a.groups_q = (a.heads_q + heads - 1) / heads;
        a.groups_kv = (a.heads_kv + heads - 1) / heads;
        a.of_qk = static_cast<uint32_t>(a.groups_q + a.groups_kv) * a.units;
        a.per_token = a.of_qk + static_cast<uint32_t>(a.groups_kv) * a.units_v;
        a.by_token = ~uint64_t(0) / a.per_token + 1;
        return static_cast<int64_t>(a.n_tokens) * a.per_token;
    };
    // two whole waves: a third wave that is not full costs as much as a full one
    const int64_t most = static_cast<int64_t>(n_sm) * 2 * fit<kBytes, kSide>();
    auto grid = [&](int64_t threads) {
        const int64_t want = (threads + kRotThreads - 1) / kRotThreads;
        return dim3(static_cast<unsigned>(want < most ? want : most));
    };
    int64_t threads = deal(kRotHeads);
    if (threads >= static_cast<int64_t>(n_sm) * kRotThreads)
        return launch_early(paged_rotary<kType, kBytes, kSide, kRotHeads>, grid(threads), kRotThreads, 0,
                            static_cast<cudaStream_t>(stream), a);
    threads = deal(1);
    return launch_early(paged_rotary<kType, kBytes, kSide, 1>, grid(threads), kRotThreads, 0,
                        static_cast<cudaStream_t>(stream), a);
}

// Pairs side by side come 16 bytes at a time; pairs half a head apart too, where the half is
// whole pieces of 16 bytes.
template <int kType> int launch_type(const PagedRotaryArgs &a, bool interleaved, int n_sm, void *stream)
{
    constexpr int kEs = kType == BSM_F32 ? 4 : 2;
    if (interleaved)
        return launch<kType, 16, true>(a, n_sm, stream);
    if (a.half * kEs % 16 == 0)
        return launch<kType, 16, false>(a, n_sm, stream);
    if (kEs == 4 || a.half * kEs % 4 == 0)
        return launch<kType, 4, false>(a, n_sm, stream);
    return launch<kType, kEs, false>(a, n_sm, stream);
}

}  // namespace

int launch_paged_rotary(PagedRotaryArgs a, int dtype, bool interleaved, int n_sm, void *stream)
{
    a.wide_table = reinterpret_cast<uintptr_t>(a.table) % 16 == 0 && a.table_stride % 4 == 0 && a.half % 4 == 0;
    return dtype == BSM_F32    ? launch_type<BSM_F32>(a, interleaved, n_sm, stream)
           : dtype == BSM_BF16 ? launch_type<BSM_BF16>(a, interleaved, n_sm, stream)
                               : launch_type<BSM_F16>(a, interleaved, n_sm, stream);
}

}  // namespace bsm
