// bsm_paged_tiles.cu -- attention of many new tokens over a paged cache, on
// the 5th-generation tensor cores.
//
//   s = scale q k^T,  p = exp(s - m),  o = sum p v / sum p   (m a running reference)
//
// Bound: the tensor cores (4 D operations a pair of a query row and a key) and,
// close behind, the exponentials.  One persistent CTA per SM, 10 warps:
//   warps 0-3, 4-7  softmax of one 128-row block each: a thread owns a row, reads
//                   its 128 scores from tensor memory, writes the probabilities
//                   back over them as 16-bit pairs, and at the end scales and
//                   stores its row of the output;
//   warp 8          producer: walks its share of the work line, copies the two
//                   query blocks and then blocks of 128 keys and values, page by
//                   page, with TMA (128-byte swizzle) into a ring of stages;
//   warp 9          issues tcgen05.mma: scores (both operands in shared memory),
//                   then probabilities (tensor memory) times values (shared memory,
//                   rows of head columns: the "N-major" form).
// The two row blocks share every stage, which halves what an SM reads from L2,
// and alternate on the tensor cores: while one block's scores become
// probabilities, the other's products run.  The output stays in tensor memory;
// it is rescaled only when a row's maximum has grown by more than 2^8 since
// its reference was taken (any reference gives the same quotient, and 2^8 is
// far from the range of fp32 sums), so nearly all blocks skip that pass.
// Every wait is bounded as in the batched product.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kTileThreads = 320;
constexpr int kPrefixThreads = 256;
constexpr int kKeys = kPagedTileKeys;
constexpr int kHalfBytes = 128 * 128;                   // 128 rows of 64 columns
constexpr int kTileHeader = 1024;
constexpr uint32_t kTileTmemCols = 512;
constexpr int kMaxStages = 8;
constexpr float kLag = 8.0f;                            // log2 of how far a maximum may pass its reference

// columns of the tensor memory: scores of the two blocks (probabilities over
// them), outputs of the two
__device__ __forceinline__ constexpr uint32_t s_col(int sub) { return static_cast<uint32_t>(sub * 128); }
__device__ __forceinline__ constexpr uint32_t o_col(int sub) { return static_cast<uint32_t>(256 + sub * 128); }

template <int DP> struct TileShape {
    static constexpr int kHalves = DP / 64;
    static constexpr int kStageBytes = kHalves * kHalfBytes;
    static constexpr int kStages = DP == 128 ? 5 : 8;
    static constexpr int kQBytes = 2 * kStageBytes;
    static constexpr int kSmem = 1024 + kTileHeader + kQBytes + kStages * kStageBytes;
};

// What the producer tells the other warps of a piece.
struct TilePiece {
    int32_t blocks;                     // key blocks; 0: no more pieces
    int32_t subs;                       // row blocks with rows (1 or 2)
    int32_t first;                      // first key block
    int32_t lo, hi, pos;                // keys of the tile; position of its first token
    int32_t token, tokens, head, heads;
    int32_t slot;                       // of its partial output; -1: the tile is whole
    int32_t join;                       // units that share the tile, if this one is the first
};

struct TileSmem {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t qfull, qempty;
    uint64_t sfull[2], pfull[2], odone[2], ofree[2];
    uint64_t pcfull[2], pcempty[2];
    uint64_t tail, drain;
    TilePiece piece[2];
    uint32_t tmem_base;
    int32_t abort_flag;
};
static_assert(sizeof(TileSmem) <= kTileHeader, "tile header");

__device__ __forceinline__ void tma_load_3d_q(void *dst, const CUtensorMap *map, int32_t c0, int32_t c1, int32_t c2,
                                              uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(saddr(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(saddr(bar))
        : "memory");
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1, int32_t c2,
                                            int32_t c3, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, "
        "%5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(saddr(bar))
        : "memory");
}

// Descriptor of a tile whose rows are the reduction dimension and whose
// columns (64 of them a 128-byte row) are N: groups of 8 rows 1024 bytes apart,
// the next 64 columns kHalfBytes on; 128-byte swizzle.
__device__ __forceinline__ uint64_t smem_desc_n(uint32_t addr)
{
    const uint64_t a = (addr & 0x3FFFFu) >> 4;
    return a | (uint64_t(kHalfBytes >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// kind::f16, fp32 accumulator, A and B both f16 or both bf16, M = 128.
template <bool kF16, int N, bool kBRows> __device__ __forceinline__ constexpr uint32_t tile_idesc()
{
    return (1u << 4) | (kF16 ? 0u : (1u << 7) | (1u << 10)) | (kBRows ? 1u << 16 : 0u) | (uint32_t(N >> 3) << 17) |
           (uint32_t(128 >> 4) << 24);
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Every lane waits; true in all lanes only if none gave up.
__device__ __forceinline__ bool warp_wait(uint64_t *b, uint32_t parity, const volatile int32_t *abort)
{
    return __all_sync(0xffffffffu, bar_spin(b, parity, abort));
}

// The same for what is waited for whether or not another warp gave up.
__device__ __forceinline__ bool warp_drain(uint64_t *b, uint32_t parity)
{
    return __all_sync(0xffffffffu, bar_wait(b, parity, nullptr));
}

// ------------------------------------------------------------- producer
// Copies stage after stage in the order the products read them: K and V of one
// block after another.  Lane c looks up the page of the block's c-th piece (a
// box of `box` rows lies in one page); the copies themselves are issued by one
// elected lane.
template <int DP>
__device__ bool produce(const PagedArgs &a, const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv, int box,
                        TileSmem &h, unsigned char *qs, unsigned char *stages, const PagedLine<kKeys> &line,
                        PagedWalk<kKeys> &walk, const PagedCut &cut, int32_t unit, uint32_t &loaded, uint32_t &qloads)
{
    using Shape = TileShape<DP>;
    const int lane = threadIdx.x & 31;
    const int boxes = kKeys / box;
    RingPos pos;
    uint32_t npc = 0, tails = 0;
    for (;; ++npc) {
        PagedPiece p{};
        const bool more = walk.next(p);
        if (!warp_wait(&h.pcempty[npc & 1u], ((npc >> 1) & 1u) ^ 1u, &h.abort_flag))
            return false;
        if (!more) {
            if (elect_one()) {
                h.piece[npc & 1u].blocks = 0;
                bar_arrive(&h.pcfull[npc & 1u]);
            }
            __syncwarp();
            return true;
        }
        const PagedSeq &s = walk.s;
        const int32_t kvh = p.head / a.subs, sub = p.head - kvh * a.subs, half_tok = a.tok / 2;
        TilePiece t;
        t.blocks = p.steps;
        t.first = p.first;
        t.lo = p.keys.lo;
        t.hi = p.keys.hi;
        t.token = s.t0 + p.tile * a.tok;
        t.tokens = s.m - p.tile * a.tok < a.tok ? s.m - p.tile * a.tok : a.tok;
        t.pos = s.L - s.m + p.tile * a.tok;
        t.subs = t.tokens > half_tok ? 2 : 1;
        t.head = kvh * a.group + sub * a.sub;
        t.heads = a.group - sub * a.sub < a.sub ? a.group - sub * a.sub : a.sub;
        t.slot = p.starts && p.ends ? -1 : 2 * unit + (p.starts ? 1 : 0);
        t.join = p.starts && !p.ends ? cut.owner(p.tile_end - 1) - unit + 1 : 0;
        if (elect_one()) {
            h.piece[npc & 1u] = t;
            bar_arrive(&h.pcfull[npc & 1u]);
        }
        __syncwarp();
        if (!warp_wait(&h.qempty, (npc & 1u) ^ 1u, &h.abort_flag))
            return false;
        if (elect_one()) {
            bar_expect(&h.qfull, static_cast<uint32_t>(t.subs * Shape::kHalves * half_tok * a.sub * 128));
            for (int sb = 0; sb < t.subs; ++sb)
                for (int hf = 0; hf < Shape::kHalves; ++hf)
                    tma_load_3d_q(qs + (sb * Shape::kHalves + hf) * kHalfBytes, &tq, hf * 64, t.head,
                                  t.token + sb * half_tok, &h.qfull);
        }
        __syncwarp();
        ++qloads;
        // keys that some token of the request sees: the others are not read
        int32_t keep = 0;
        if (a.window && s.L - s.m - a.window + 1 > 0)
            keep = s.L - s.m - a.window + 1;
        const int64_t row = p.r * a.table_stride;
        // page of this lane's piece of block b: (page, row in it); n_pages: not there, filled with zeros
        auto page_of = [&](int32_t b, int32_t &in) -> int32_t {
            const int32_t key = b * kKeys + lane * box;
            if (lane >= boxes || key >= s.L || key + box <= keep)
                return -1;
            const int32_t e = key / a.page;
            in = key - e * a.page;
            const int32_t page = a.tables[row + e];
            if (page < 0 || page >= a.n_pages) {
                atomicOr(a.status, BSM_DEV_BOUNDS);
                return a.n_pages;
            }
            return page;
        };
        int32_t in = 0;
        int32_t page = page_of(p.first, in);
        for (int32_t i = 0; i < p.steps; ++i) {
            const int32_t key0 = (p.first + i) * kKeys;
            const uint32_t have = __ballot_sync(0xffffffffu, page >= 0);
            // rows of the block that hold no key of the request: zeros for the values (0 times
            // whatever lies there may be NaN); their scores are masked
            const int32_t v0 = keep > key0 ? keep - key0 : 0;
            const int32_t v1 = s.L - key0 < kKeys ? (s.L > key0 ? s.L - key0 : 0) : kKeys;
            const bool ragged = v0 > 0 || v1 < kKeys;
            int32_t nin = 0, npage = -1;
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
                if (!warp_wait(&h.empty[pos.s], pos.ph ^ 1u, &h.abort_flag))
                    return false;
                const uint32_t st = saddr(stages) + static_cast<uint32_t>(pos.s * Shape::kStageBytes);
                const bool hold = kv == 1 && ragged;
                uint64_t *bar = hold ? &h.tail : &h.full[pos.s];
                if (elect_one())
                    bar_expect(bar, static_cast<uint32_t>(__popc(have) * box * 128 * Shape::kHalves));
                __syncwarp();
                for (int c = 0; c < boxes; ++c) {
                    const int32_t pg = __shfl_sync(0xffffffffu, page, c), rw = __shfl_sync(0xffffffffu, in, c);
                    if (!((have >> c) & 1u))
                        continue;
                    if (elect_one()) {
#pragma unroll
                        for (int hf = 0; hf < Shape::kHalves; ++hf)
                            tma_load_4d(st + hf * kHalfBytes + c * box * 128, kv ? &tv : &tk, hf * 64, rw, kvh, pg, bar);
                    }
                    __syncwarp();
                }
                if (kv == 0 && i + 1 < p.steps)
                    npage = page_of(p.first + i + 1, nin);
                if (hold) {
                    if (!warp_drain(&h.tail, tails & 1u))
                        return false;
                    ++tails;
                    for (int x = lane; x < 8 * kKeys; x += 32) {
                        const int r = x >> 3;
                        if (r < v0 || r >= v1) {
#pragma unroll
                            for (int hf = 0; hf < Shape::kHalves; ++hf)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(
                                                 st + hf * kHalfBytes + r * 128 + (x & 7) * 16),
                                             "r"(0)
                                             : "memory");
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (elect_one())
                        bar_arrive(&h.full[pos.s]);
                    __syncwarp();
                }
                ++loaded;
                pos.step(Shape::kStages);
            }
            page = npage;
            in = nin;
        }
    }
}

// ------------------------------------------------------------- tensor cores
template <int DP, bool kF16>
__device__ bool multiply(TileSmem &h, unsigned char *qs, unsigned char *stages, uint32_t tmem)
{
    using Shape = TileShape<DP>;
    constexpr uint32_t kScores = tile_idesc<kF16, kKeys, false>(), kOut = tile_idesc<kF16, DP, true>();
    RingPos pos;                        // next stage: K of the next block, then V of this one
    uint32_t nblk[2] = {0, 0}, npiece[2] = {0, 0};
    for (uint32_t npc = 0;; ++npc) {
        if (!warp_wait(&h.pcfull[npc & 1u], (npc >> 1) & 1u, &h.abort_flag))
            return false;
        const int32_t blocks = __shfl_sync(0xffffffffu, h.piece[npc & 1u].blocks, 0);
        const int32_t subs = __shfl_sync(0xffffffffu, h.piece[npc & 1u].subs, 0);
        __syncwarp();
        if (elect_one())
            bar_arrive(&h.pcempty[npc & 1u]);
        __syncwarp();
        if (blocks == 0)
            return true;
        if (!warp_wait(&h.qfull, npc & 1u, &h.abort_flag))
            return false;
        auto scores = [&](int sub, int stage) {
            const uint64_t ad = smem_desc(qs + sub * Shape::kStageBytes);
            const uint64_t bd = smem_desc(stages + stage * Shape::kStageBytes);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                const uint64_t off = static_cast<uint64_t>((k / 4) * (kHalfBytes >> 4) + (k % 4) * 2);
                mma_ss(tmem + s_col(sub), ad + off, bd + off, kScores, k != 0);
            }
            mma_commit(&h.sfull[sub]);
        };
        // K of the first block
        if (!warp_wait(&h.full[pos.s], pos.ph, &h.abort_flag))
            return false;
        tc_fence_after();
        if (elect_one()) {
            for (int sub = 0; sub < subs; ++sub)
                scores(sub, pos.s);
            mma_commit(&h.empty[pos.s]);
            if (blocks == 1)
                mma_commit(&h.qempty);
        }
        __syncwarp();
        pos.step(Shape::kStages);
        for (int32_t j = 0; j < blocks; ++j) {
            const bool next = j + 1 < blocks;
            const int vs = pos.s;
            const uint32_t vph = pos.ph;
            pos.step(Shape::kStages);
            const int ks = pos.s;
            const uint32_t kph = pos.ph;
            if (next)
                pos.step(Shape::kStages);
            for (int sub = 0; sub < subs; ++sub) {
                if (sub == 0 && !warp_wait(&h.full[vs], vph, &h.abort_flag))
                    return false;
                if (!warp_wait(&h.pfull[sub], nblk[sub] & 1u, &h.abort_flag))
                    return false;
                ++nblk[sub];
                // the previous piece's output has been read
                if (j == 0) {
                    if (!warp_wait(&h.ofree[sub], (npiece[sub] & 1u) ^ 1u, &h.abort_flag))
                        return false;
                    ++npiece[sub];
                }
                if (sub == 0 && next && !warp_wait(&h.full[ks], kph, &h.abort_flag))
                    return false;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t bd = smem_desc_n(saddr(stages) + vs * Shape::kStageBytes);
#pragma unroll
                    for (int k = 0; k < kKeys / 16; ++k)
                        mma_ts(tmem + o_col(sub), tmem + s_col(sub) + k * 8, bd + k * (2048 >> 4), kOut, (j | k) != 0);
                    mma_commit(&h.odone[sub]);
                    if (sub == subs - 1)
                        mma_commit(&h.empty[vs]);
                    if (next) {
                        scores(sub, ks);
                        if (sub == subs - 1) {
                            mma_commit(&h.empty[ks]);
                            if (j + 2 == blocks)
                                mma_commit(&h.qempty);
                        }
                    }
                }
                __syncwarp();
            }
        }
    }
}

// ------------------------------------------------------------- softmax
template <int DP, bool kF16>
__device__ bool softmax(const PagedArgs &a, TileSmem &h, uint32_t tmem, int sub, int32_t unit)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quarter = warp & 3;
    const int row = quarter * 32 + lane;                // of the row block
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const int32_t tt = row / a.sub, hh = row - tt * a.sub, half_tok = a.tok / 2;
    uint32_t nblk = 0;
    for (uint32_t npc = 0;; ++npc) {
        if (!warp_wait(&h.pcfull[npc & 1u], (npc >> 1) & 1u, &h.abort_flag))
            return false;
        const TilePiece t = h.piece[npc & 1u];
        __syncwarp();
        if (lane == 0)
            bar_arrive(&h.pcempty[npc & 1u]);
        if (t.blocks == 0)
            return true;
        if (sub >= t.subs)
            continue;
        const int32_t tok = sub * half_tok + tt;        // of the tile
        const bool live = tt < half_tok && tok < t.tokens && hh < t.heads;
        // keys this row sees; rows that are not stored compute whatever comes
        int32_t lo = 0, hi = INT32_MAX;
        if (live) {
            hi = t.hi;
            if (a.causal) {
                hi = t.pos + tok + 1 < t.hi ? t.pos + tok + 1 : t.hi;
                if (a.window && t.pos + tok - a.window + 1 > 0)
                    lo = t.pos + tok - a.window + 1;
            }
        }
        float ref = -INFINITY, sum = 0.0f;              // reference (log2), sum of probabilities
        for (int32_t j = 0; j < t.blocks; ++j, ++nblk) {
            if (!warp_wait(&h.sfull[sub], nblk & 1u, &h.abort_flag))
                return false;
            tc_fence_after();
            uint32_t r[128];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                tmem_ld32_nowait(lanes + s_col(sub) + c * 32, r + c * 32);
            tmem_wait_ld();
            float x[128];
#pragma unroll
            for (int c = 0; c < 128; ++c)
                x[c] = __uint_as_float(r[c]);
            const int32_t key0 = (t.first + j) * kKeys;
            if (!__all_sync(0xffffffffu, lo <= key0 && hi - kKeys >= key0)) {
                const int32_t c0 = lo - key0, c1 = hi - key0;
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    x[c] = c >= c0 && c < c1 ? x[c] : -INFINITY;
            }
            float top4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int c = 4; c < 128; ++c)
                top4[c & 3] = fmaxf(top4[c & 3], x[c]);
            const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * a.scale_log2;
            // (a maximum of -inf moves nothing; NaN neither: it comes out in the sum)
            const bool move = top > ref + kLag;
            if (__any_sync(0xffffffffu, move)) {
                const float f = !move ? 1.0f : pg_exp2(ref - top);
                ref = move ? top : ref;
                sum *= f;
                if (j > 0) {
                    // the product of the previous block still adds to the output
                    if (!warp_wait(&h.odone[sub], (nblk & 1u) ^ 1u, &h.abort_flag))
                        return false;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < DP / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32_nowait(lanes + o_col(sub) + c * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st32(lanes + o_col(sub) + c * 32, o);
                    }
                }
            }
            const float base = ref == -INFINITY ? 0.0f : ref - pg_shift<kF16>(kLag);
            float s4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            uint32_t pr[64];
#pragma unroll
            for (int c = 0; c < 128; c += 2) {
                const float p0 = pg_exp2(fmaf(x[c], a.scale_log2, -base));
                const float p1 = pg_exp2(fmaf(x[c + 1], a.scale_log2, -base));
                s4[c & 2] += p0;
                s4[(c & 2) + 1] += p1;
                pr[c / 2] = pg_pack<kF16>(p0, p1);
            }
            sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
            tmem_st32(lanes + s_col(sub), pr);
            tmem_st32(lanes + s_col(sub) + 32, pr + 32);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                bar_arrive(&h.pfull[sub]);
        }
        // ---- the row's output
        if (!warp_wait(&h.odone[sub], (nblk & 1u) ^ 1u, &h.abort_flag))
            return false;
        tc_fence_after();
        const float base = ref - pg_shift<kF16>(kLag);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int64_t token = t.token + tok;
        unsigned char *dst = static_cast<unsigned char *>(a.out) + 2 * (token * a.out_token + (t.head + hh) * a.out_head);
        float *part = a.part_o + static_cast<int64_t>(t.slot) * (256 * kPagedMaxDim) + (sub * 128 + row) * 4;
#pragma unroll 1
        for (int c = 0; c < DP / 32; ++c) {
            uint32_t o[32];
            tmem_ld32_nowait(lanes + o_col(sub) + c * 32, o);
            tmem_wait_ld();
            const float *f = reinterpret_cast<const float *>(o);
            if (t.slot < 0) {
                if (live) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (c * 32 + i * 8 < a.d) {
                            uint4 w;
                            w.x = pg_pack<kF16>(f[8 * i] * inv, f[8 * i + 1] * inv);
                            w.y = pg_pack<kF16>(f[8 * i + 2] * inv, f[8 * i + 3] * inv);
                            w.z = pg_pack<kF16>(f[8 * i + 4] * inv, f[8 * i + 5] * inv);
                            w.w = pg_pack<kF16>(f[8 * i + 6] * inv, f[8 * i + 7] * inv);
                            *reinterpret_cast<uint4 *>(dst + (c * 32 + i * 8) * 2) = w;
                        }
                    }
                }
            } else {
                // four columns of a row together, rows side by side: a warp stores 512 bytes at once
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<float4 *>(part + static_cast<int64_t>(c * 8 + i) * (256 * 4)) =
                        make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0)
            bar_arrive(&h.ofree[sub]);
        if (t.slot < 0) {
            if (live && a.lse)
                a.lse[token * a.heads_q + t.head + hh] =
                    sum == 0.0f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f;
        } else {
            *reinterpret_cast<float2 *>(a.part_ml + (static_cast<int64_t>(t.slot) * 256 + sub * 128 + row) * 2) =
                make_float2(base, sum);
        }
        if (t.join > 0 && sub == 0 && threadIdx.x == 0) {
            PagedJoin j{};
            j.token = t.token;
            j.head = t.head;
            j.tokens = t.tokens;
            j.heads = t.heads;
            j.count = t.join;
            a.join[unit] = j;
        }
    }
}

template <int DP, bool kF16>
__global__ void __launch_bounds__(kTileThreads, 1)
    paged_tiles(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                const __grid_constant__ CUtensorMap tv, const PagedArgs a, const int box)
{
    using Shape = TileShape<DP>;
    extern __shared__ __align__(1024) unsigned char raw[];
    unsigned char *smem = raw + ((1024u - (saddr(raw) & 1023u)) & 1023u);
    TileSmem &h = *reinterpret_cast<TileSmem *>(smem);
    unsigned char *qs = smem + kTileHeader, *stages = qs + Shape::kQBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int32_t unit = blockIdx.x;
    if (threadIdx.x == 0) {
        for (int s = 0; s < Shape::kStages; ++s) {
            bar_init(&h.full[s], 1);
            bar_init(&h.empty[s], 1);
        }
        bar_init(&h.qfull, 1);
        bar_init(&h.qempty, 1);
        for (int s = 0; s < 2; ++s) {
            bar_init(&h.sfull[s], 1);
            bar_init(&h.pfull[s], 4);
            bar_init(&h.odone[s], 1);
            bar_init(&h.ofree[s], 4);
            bar_init(&h.pcfull[s], 1);
            bar_init(&h.pcempty[s], 9);
        }
        bar_init(&h.tail, 1);
        bar_init(&h.drain, 1);
        h.abort_flag = 0;
        a.join[unit].count = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // the line of work; its prefix lies where the stages will be
    PagedPrefix<kPrefixThreads> &prefix = *reinterpret_cast<PagedPrefix<kPrefixThreads> *>(stages);
    const PagedLine<kKeys> line(a);
    paged_prefix<kKeys, kPrefixThreads>(line, prefix, blockIdx.x == 0);
    const int64_t W = prefix.pre[kPrefixThreads];
    const PagedCut cut(a, W);
    if (W == 0 || unit >= cut.units)
        return;                                         // (the whole CTA)
    PagedWalk<kKeys> walk(line, prefix, cut.begin(unit), warp == 8 ? cut.begin(unit + 1) : 0);
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(saddr(&h.tmem_base)),
                     "r"(kTileTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // the prefix has been read: the stages may be written over it by the copies
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = h.tmem_base;

    bool ok;
    if (warp == 8) {
        uint32_t loaded = 0, qloads = 0;
        ok = produce<DP>(a, tq, tk, tv, box, h, qs, stages, line, walk, cut, unit, loaded, qloads);
        if (!ok) {
            if (elect_one()) {
                atomicOr(a.status, BSM_DEV_TIMEOUT);
                h.abort_flag = 1;
            }
            __syncwarp();
        }
        // copies in flight land before the CTA leaves
        const uint32_t S = Shape::kStages;
        for (uint32_t j = loaded > S ? loaded - S : 0u; j < loaded; ++j)
            warp_drain(&h.full[j % S], (j / S) & 1u);
        if (qloads)
            warp_drain(&h.qfull, (qloads - 1) & 1u);
    } else if (warp == 9) {
        ok = multiply<DP, kF16>(h, qs, stages, tmem);
        if (elect_one()) {
            if (!ok) {
                atomicOr(a.status, BSM_DEV_TIMEOUT);
                h.abort_flag = 1;
            }
            mma_commit(&h.drain);
        }
        __syncwarp();
        // every product has finished before the tensor memory is freed
        warp_drain(&h.drain, 0);
    } else {
        ok = softmax<DP, kF16>(a, h, tmem, warp >> 2, unit);
        if (!ok) {
            if ((threadIdx.x & 31) == 0) {
                atomicOr(a.status, BSM_DEV_TIMEOUT);
                h.abort_flag = 1;
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTileTmemCols) : "memory");
    }
}

// Joins the parts of every cut tile (see paged_join of the row kernel): a
// thread a row, eight columns a CTA.
constexpr int kTileJoinThreads = 128;

template <bool kF16> __global__ void __launch_bounds__(kTileJoinThreads) paged_tile_join(const PagedArgs a)
{
    const int unit = blockIdx.x, sub = blockIdx.y;
    const PagedJoin j = a.join[unit];
    if (j.count <= 0)
        return;
    const int half_tok = a.tok / 2;
    const int tt = threadIdx.x / a.sub, h = threadIdx.x - tt * a.sub, tok = sub * half_tok + tt;
    if (tt >= half_tok || tok >= j.tokens || h >= j.heads)
        return;
    const int row = sub * 128 + threadIdx.x;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
    const float4 *po = reinterpret_cast<const float4 *>(a.part_o);
    float top = -INFINITY;
    for (int i = 0; i < j.count; ++i) {
        const int64_t slot = i == 0 ? 2 * unit + 1 : 2 * (unit + i);
        top = fmaxf(top, ml[slot * 256 + row].x);
    }
    const float ref = top == -INFINITY ? 0.0f : top;
    float acc[8] = {};
    float sum = 0.0f;
    const int c = blockIdx.z * 2;
#pragma unroll 4
    for (int i = 0; i < j.count; ++i) {
        const int64_t slot = i == 0 ? 2 * unit + 1 : 2 * (unit + i);
        const float2 m = ml[slot * 256 + row];
        const float4 u = po[(slot * (kPagedMaxDim / 4) + c) * 256 + row];
        const float4 v = po[(slot * (kPagedMaxDim / 4) + c + 1) * 256 + row];
        const float f = pg_exp2(m.x - ref);
        sum += f * m.y;
        acc[0] += f * u.x;
        acc[1] += f * u.y;
        acc[2] += f * u.z;
        acc[3] += f * u.w;
        acc[4] += f * v.x;
        acc[5] += f * v.y;
        acc[6] += f * v.z;
        acc[7] += f * v.w;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint4 w;
    w.x = pg_pack<kF16>(acc[0] * inv, acc[1] * inv);
    w.y = pg_pack<kF16>(acc[2] * inv, acc[3] * inv);
    w.z = pg_pack<kF16>(acc[4] * inv, acc[5] * inv);
    w.w = pg_pack<kF16>(acc[6] * inv, acc[7] * inv);
    const int64_t token = j.token + tok;
    *reinterpret_cast<uint4 *>(static_cast<unsigned char *>(a.out) +
                               2 * (token * a.out_token + (j.head + h) * a.out_head + blockIdx.z * 8)) = w;
    if (a.lse && blockIdx.z == 0)
        a.lse[token * a.heads_q + j.head + h] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

template <int DP, bool kF16>
int launch(const CUtensorMap *m, const PagedArgs &a, int box, cudaStream_t st)
{
    paged_tiles<DP, kF16><<<a.units, kTileThreads, TileShape<DP>::kSmem, st>>>(m[0], m[1], m[2], a, box);
    if (int e = static_cast<int>(cudaGetLastError()))
        return e;
    paged_tile_join<kF16><<<dim3(a.units, 2, a.d / 8), kTileJoinThreads, 0, st>>>(a);
    return static_cast<int>(cudaGetLastError());
}

}  // namespace

int launch_paged_tiles(const void *maps, const PagedArgs &a, bool f16, int box, void *stream)
{
    const CUtensorMap *m = static_cast<const CUtensorMap *>(maps);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.d <= 64)
        return f16 ? launch<64, true>(m, a, box, st) : launch<64, false>(m, a, box, st);
    return f16 ? launch<128, true>(m, a, box, st) : launch<128, false>(m, a, box, st);
}

int paged_tiles_set_smem()
{
    int e = 0;
    auto set = [&](const void *f, int bytes) {
        if (!e)
            e = static_cast<int>(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    };
    set(reinterpret_cast<const void *>(&paged_tiles<64, false>), TileShape<64>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<64, true>), TileShape<64>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, false>), TileShape<128>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, true>), TileShape<128>::kSmem);
    return e;
}

}  // namespace bsm
