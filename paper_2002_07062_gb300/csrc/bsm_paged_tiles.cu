// bsm_paged_tiles.cu -- attention of many new tokens over a paged cache, on
// the 5th-generation tensor cores.
//
//   s = scale q k^T,  p = exp(s - m),  o = sum p v / sum p   (m a running reference)
//
// Bound: the tensor cores (4 D operations a pair of a query row and a key) and,
// close behind, the softmax between a row block's two products.  One persistent
// CTA per SM, 12 warps:
//   warps 0-3, 4-7  two softmax groups, each with one block of 128 rows: a thread
//                   owns a row, reads its 128 scores of a step from tensor memory,
//                   writes the probabilities back over them as 16-bit pairs, and at
//                   the end scales and stores its row of the output;
//   warp 8          walks its CTA's share of the work line and copies steps of 128
//                   keys and values, page by page, with TMA (128-byte swizzle) into a
//                   ring of stages;
//   warps 9, 10     issue tcgen05.mma, one for each group: scores (both operands in
//                   shared memory), then probabilities (tensor memory) times values
//                   (shared memory, rows of head columns: the "N-major" form);
//   warp 11         copies each tile's query blocks.
// The row blocks share every stage, which halves what an SM reads from L2.  They
// take turns at the tensor cores: while one block's scores become
// probabilities, the other's products run.  A tile of one row block takes both
// groups all the same: one has the even key steps, the other the odd ones, each
// with its own output and reference, and the two are added at the end.
// Outputs stay in tensor memory; one is rescaled only when a row's maximum has
// grown by more than 2^8 since its reference was taken (any reference gives the
// same quotient, and probabilities are held 2^8 lower for it), so nearly all
// steps skip that pass.
//
// GB300: two prompts of 8192 tokens, 32/8 heads of 128: 714 to 780 us (1.54 to 1.41
// PFLOP/s; a plain bf16 product of the library's 1.95), the longer the more power the values
// draw; tensor pipe 71 % active on 2048 tokens over 6100; 2 x 4 tokens over up to 131 thousand
// keys, 1.02 GB: 171 us.  Without the softmax between the products the first runs in 548 us
// (2.0 PFLOP/s).  Every instance has 168 registers a thread and spills 4 to 8 bytes.  Tried and slower for it: steps of 64 keys with two score
// buffers a block, which never wait for scores (963 us: a product of 128 x 64 x 16
// takes 52 cycles instead of 32, the bytes of its operands in shared memory);
// probabilities in two parts, the first one's product beside the second's
// exponentials (787); two softmax warps a row (917 to 922: 96 registers, and the two
// have to meet every step); one issuing warp (924 and more); a warp each for keys and
// values (759).
// Every wait is bounded as in the batched product.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "bsm_paged_again.h"
#include "bsm_paged_dev.h"
#include "bsm_tc.h"

namespace bsm {
namespace {

constexpr int kTileThreads = 384;
constexpr int kPieces = 4;                              // told ahead at most
constexpr int kPrefixThreads = 256;
constexpr int kKeys = kPagedTileKeys;
constexpr int kQHalf = 128 * 128;                       // 128 query rows of 64 columns
constexpr int kHalfBytes = kKeys * 128;                 // a step's keys, 64 columns
constexpr int kStore = 8 * 32 * 64;                     // a warp's 32 rows of 32 columns on their way out
constexpr int kTileHeader = 4096;
constexpr uint32_t kTileTmemCols = 512;
constexpr int kMaxStages = 8;
constexpr float kLag = 8.0f;                            // log2 of how far a maximum may pass its reference

// columns of the tensor memory: scores of the two blocks (the probabilities
// over them), outputs of the two
__device__ __forceinline__ constexpr uint32_t s_col(int sub) { return static_cast<uint32_t>(sub * 128); }
__device__ __forceinline__ constexpr uint32_t o_col(int sub) { return static_cast<uint32_t>(256 + sub * 128); }

template <int DP> struct TileShape {
    static constexpr int kHalves = DP / 64;
    static constexpr int kStageBytes = kHalves * kHalfBytes;    // keys, or values, of a step
    static constexpr int kStages = DP == 128 ? 4 : 8;
    static constexpr int kQBytes = 2 * kHalves * kQHalf;
    static constexpr int kSmem = 1024 + kTileHeader + kStore + kQBytes + kStages * kStageBytes;
};

// How the stages are filled: by TMA, the two halves of the columns apart (a copy each);
// by TMA with whole rows a copy, the halves of eight rows side by side; row by row.
// (An instance of the kernel each: descriptors stay constants, and the last one's
// registers cost the others nothing.)  Whole rows halve the copies: two prompts of 8192
// tokens in pages of 16 take 757 us, 770 with halves apart; in pages of 8 876 and 926;
// a chunk of 2048 over 6100 keys in pages of 64 161 and 164.
enum Fill { kByHalves, kByRows, kOddPages };

template <int kFill> struct StageSteps {
    static constexpr int kHalf = kFill == kByRows ? 1024 : kHalfBytes;  // bytes to the other 64 columns
    static constexpr int kGroup = kFill == kByRows ? 2048 : 1024;       // to the next eight rows
};

// What the producer tells the other warps of a piece.
struct TilePiece {
    int32_t blocks;                     // key steps; 0: no more pieces
    int32_t subs;                       // softmax groups with work (1 or 2)
    int32_t dual;                       // one row block: key steps dealt to the two groups in turn
    int32_t first;                      // first key step
    int32_t hi, pos;                    // end of the tile's keys; position of its first token
    int32_t token, tokens, head, heads;
    int32_t r, kvh, keep, len;          // request, key/value head; keys [keep, len) may be read
    int32_t slot;                       // of its partial output; -1: the tile is whole
    int32_t join;                       // units that share the tile, if this one is the first
};

struct TileSmem {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t qfull, qempty;
    uint64_t sfull[2], pfull[2], olast[2], ofree[2];
    uint64_t pcfull[kPieces], pcempty[kPieces];
    uint64_t turn[2];                   // the group may issue its next scores
    uint64_t tail, drain, xfull;
    TilePiece piece[kPieces];
    float2 other[128];                  // reference and sum of the second group's rows (dual)
    int64_t where[2][kKeys];            // of odd pages: byte offset of a step's rows (-1: not read)
    uint32_t tmem_base;
    int32_t abort_flag, no_abort;       // (the second stays 0)
    int32_t odd;                        // an output that was stored is not finite
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
                                            int32_t c3, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, "
        "%5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1, int32_t c2,
                                            int32_t c3, int32_t c4, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, "
        "%5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar)
        : "memory");
}

// Descriptors of a stage, 128-byte swizzle.  Keys: the columns are the reduction
// dimension; groups of eight rows kGroup bytes apart.  Values: the rows are, and the
// columns (64 of them a 128-byte row) are N; the next 64 kHalf bytes on.
template <int kFill> __device__ __forceinline__ uint64_t stage_desc_k(uint32_t addr)
{
    const uint64_t a = (addr & 0x3FFFFu) >> 4;
    return a | (1ull << 16) | (uint64_t(StageSteps<kFill>::kGroup >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
template <int kFill> __device__ __forceinline__ uint64_t stage_desc_v(uint32_t addr)
{
    const uint64_t a = (addr & 0x3FFFFu) >> 4;
    return a | (uint64_t(StageSteps<kFill>::kHalf >> 4) << 16) | (uint64_t(StageSteps<kFill>::kGroup >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
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

// 16 columns
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Whether the phase is over, without waiting.
__device__ __forceinline__ bool bar_done(uint64_t *b, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(saddr(b)), "r"(parity)
        : "memory");
    return ok != 0;
}

// Every lane waits; true in all lanes only if none gave up.
__device__ __forceinline__ bool warp_wait(uint64_t *b, uint32_t parity, const volatile int32_t *abort)
{
    return __all_sync(0xffffffffu, bar_spin(b, parity, abort));
}

// The same for what is waited for whether or not another warp gave up.
__device__ __forceinline__ bool warp_drain(TileSmem &h, uint64_t *b, uint32_t parity)
{
    return __all_sync(0xffffffffu, bar_spin(b, parity, &h.no_abort));
}

__device__ TilePiece tile_piece(const PagedArgs &a, const PagedSeq &s, const PagedPiece &p, const PagedCut &cut, int32_t unit)
{
    const int32_t kvh = p.head / a.subs, sub = p.head - kvh * a.subs;
    TilePiece t;
    t.blocks = p.steps;
    t.first = p.first;
    t.hi = p.keys.hi;
    t.token = s.t0 + p.tile * a.tok;
    t.tokens = s.m - p.tile * a.tok < a.tok ? s.m - p.tile * a.tok : a.tok;
    t.pos = s.L - s.m + p.tile * a.tok;
    const int32_t blocks_q = t.tokens > a.tok / 2 ? 2 : 1;
    t.dual = blocks_q == 1 && p.steps > 1;
    t.subs = t.dual ? 2 : blocks_q;
    t.r = p.r;
    t.kvh = kvh;
    t.len = s.L;
    // (keys before the first that some token of the request sees are not read)
    t.keep = a.window && s.L - s.m >= a.window ? s.L - s.m - a.window + 1 : 0;
    t.head = kvh * a.group + sub * a.sub;
    t.heads = a.group - sub * a.sub < a.sub ? a.group - sub * a.sub : a.sub;
    t.slot = p.starts && p.ends ? -1 : 2 * unit + (p.starts ? 1 : 0);
    t.join = p.starts && !p.ends ? cut.owner(p.tile_end - 1) - unit + 1 : 0;
    return t;
}

// The same value in every lane, for the compiler too: what addresses an MMA, a tensor
// copy or tensor memory has to lie in uniform registers, and moving it there costs more
// than the MMA.  (In the softmax groups too: two prompts of 8192 tokens 714 us, 741
// without; prompts under a window 138 and 145; a mixed step 104 and 109.)
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_max_sync(0xffffffffu, x); }

// ------------------------------------------------------------- producer
// Copies stage after stage in the order the products read them: K and V of one
// block after another.  Lane c looks up the page of the block's c-th piece (a
// box of `box` rows lies in one page); the copies themselves are issued by one
// elected lane.  The warp's instructions bound the small pages: with coordinates the
// compiler does not know to be uniform, two prompts of 8192 tokens in pages of 16 take
// 829 us, 770 so; in pages of 8 1106 and 928.
template <int DP, int kFill>
__device__ bool produce(const PagedArgs &a, const CUtensorMap &tk, const CUtensorMap &tv, int box, int per_page, TileSmem &h,
                        unsigned char *stages, PagedWalk<kKeys> &walk, const PagedCut &cut, int32_t unit, uint32_t &loaded,
                        PagedSeen &seen)
{
    using Shape = TileShape<DP>;
    const int lane = threadIdx.x & 31;
    const int boxes = kKeys / box;
    RingPos pos;
    uint32_t npc = 0, tails = 0;
    for (;; ++npc) {
        PagedPiece p{};
        const bool more = walk.next(p);
        if (!warp_wait(&h.pcempty[npc % kPieces], ((npc / kPieces) & 1u) ^ 1u, &h.abort_flag))
            return false;
        if (!more) {
            if (elect_one()) {
                h.piece[npc % kPieces].blocks = 0;
                bar_arrive(&h.pcfull[npc % kPieces]);
            }
            __syncwarp();
            return true;
        }
        const PagedSeq &s = walk.s;
        const TilePiece t = tile_piece(a, s, p, cut, unit);
        seen.note(p);
        if (elect_one()) {
            h.piece[npc % kPieces] = t;
            bar_arrive(&h.pcfull[npc % kPieces]);
        }
        __syncwarp();
        const int32_t kvh = static_cast<int32_t>(uniform(t.kvh)), keep = t.keep;
        const int64_t row = p.r * a.table_stride;
        // page of this lane's piece of block b: (page, row in it); n_pages: not there, filled with zeros (see the join)
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
        // one stage: keys (side 0) or values of step i, whose pieces lie in the pages given
        auto load = [&](int32_t i, int side, int32_t page, int32_t in) -> bool {
            seen.gone |= page == a.n_pages;
            const uint32_t have = __ballot_sync(0xffffffffu, page >= 0);
            // rows of the values that belong to no key of the request: zeros (0 times whatever
            // lies there may be NaN); their scores are masked
            const int32_t key0 = (p.first + i) * kKeys;
            const int32_t v0 = keep > key0 ? keep - key0 : 0;
            const int32_t v1 = s.L - key0 < kKeys ? (s.L > key0 ? s.L - key0 : 0) : kKeys;
            const bool hold = side == 1 && (v0 > 0 || v1 < kKeys);
            if (!warp_wait(&h.empty[pos.s], pos.ph ^ 1u, &h.abort_flag))
                return false;
            const uint32_t st = uniform(saddr(stages) + static_cast<uint32_t>(pos.s * Shape::kStageBytes));
            const uint32_t bar = uniform(saddr(hold ? &h.tail : &h.full[pos.s]));
            if (elect_one())
                bar_expect(hold ? &h.tail : &h.full[pos.s], static_cast<uint32_t>(__popc(have) * box * 128 * Shape::kHalves));
            __syncwarp();
            const int32_t at = kFill == kByRows ? page * per_page + in / 8 : page;  // (of this lane's piece)
            for (int c = 0; c < boxes; ++c) {
                if (!((have >> c) & 1u))
                    continue;
                const int32_t pg = static_cast<int32_t>(uniform(lane == c ? at : 0));
                const int32_t rw = kFill == kByRows ? 0 : static_cast<int32_t>(uniform(lane == c ? in : 0));
                if (elect_one()) {
                    if (kFill == kByRows) {
                        tma_load_5d(st + c * box * 256, side ? &tv : &tk, 0, 0, 0, pg, kvh, bar);
                    } else {
#pragma unroll
                        for (int hf = 0; hf < Shape::kHalves; ++hf)
                            tma_load_4d(st + hf * kHalfBytes + c * box * 128, side ? &tv : &tk, hf * 64, rw, kvh, pg, bar);
                    }
                }
                __syncwarp();
            }
            if (hold) {
                if (!warp_drain(h, &h.tail, tails & 1u))
                    return false;
                ++tails;
                for (int x = lane; x < 8 * kKeys; x += 32) {
                    const int r = x >> 3;
                    if (r < v0 || r >= v1) {
#pragma unroll
                        for (int hf = 0; hf < Shape::kHalves; ++hf)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(
                                             st + hf * StageSteps<kFill>::kHalf + (r >> 3) * StageSteps<kFill>::kGroup +
                                             (r & 7) * 128 + (x & 7) * 16),
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
            return true;
        };
        // in the order of the products: K0 V0 K1 V1 .., dual K0 K1 V0 K2 V1 ..: the keys of step i,
        // then the values of step i - lag
        const int32_t lag = t.dual ? 1 : 0;
        int32_t in = 0, page = page_of(p.first, in), in1 = 0, page1 = -1;
        for (int32_t i = 0; i < p.steps + lag; ++i) {
            int32_t nin = 0, npage = -1;
            if (i + 1 < p.steps)
                npage = page_of(p.first + i + 1, nin);      // (read a step ahead)
            if (i < p.steps && !load(i, 0, page, in))
                return false;
            if (i >= lag && !load(i - lag, 1, lag ? page1 : page, lag ? in1 : in))
                return false;
            page1 = page;
            in1 = in;
            page = npage;
            in = nin;
        }
    }
}

// The query blocks of piece npc, once the one before it has its scores.
template <int DP>
__device__ bool load_q(const PagedArgs &a, const CUtensorMap &tq, TileSmem &h, unsigned char *qs, const TilePiece &t, uint32_t npc)
{
    using Shape = TileShape<DP>;
    const int32_t half_tok = a.tok / 2, blocks_q = t.tokens > half_tok ? 2 : 1;
    if (!warp_wait(&h.qempty, (npc & 1u) ^ 1u, &h.abort_flag))
        return false;
    if (elect_one()) {
        bar_expect(&h.qfull, static_cast<uint32_t>(blocks_q * Shape::kHalves * half_tok * a.sub * 128));
        for (int sb = 0; sb < blocks_q; ++sb)
            for (int hf = 0; hf < Shape::kHalves; ++hf)
                tma_load_3d_q(qs + (sb * Shape::kHalves + hf) * kQHalf, &tq, hf * 64, t.head, t.token + sb * half_tok,
                              &h.qfull);
    }
    __syncwarp();
    return true;
}

// The query blocks of each piece, as soon as the one before it has its scores
// (in a warp of its own, so that keys and values of the next piece come
// meanwhile).
template <int DP>
__device__ bool produce_q(const PagedArgs &a, const CUtensorMap &tq, TileSmem &h, unsigned char *qs, uint32_t &loaded)
{
    for (uint32_t npc = 0;; ++npc) {
        if (!warp_wait(&h.pcfull[npc % kPieces], (npc / kPieces) & 1u, &h.abort_flag))
            return false;
        const TilePiece t = h.piece[npc % kPieces];
        __syncwarp();
        if (elect_one())
            bar_arrive(&h.pcempty[npc % kPieces]);
        __syncwarp();
        if (t.blocks == 0)
            return true;
        if (!load_q<DP>(a, tq, h, qs, t, npc))
            return false;
        ++loaded;
    }
}

// Pages that are no whole groups of eight rows (the swizzle of the copies above):
// 16 bytes a lane by plain asynchronous copies, to the swizzled places, rows that
// are not read filled with zeros.  Up to three stages of this warp's are in flight;
// a stage is handed on when its copies have landed, at the latest before this warp
// waits for anything (so no one waits for a stage that only this warp could hand
// on).  Warp 8 fills the stages of keys, warp 11 those of values: bound by their
// instructions.  Two prompts of 8192 tokens in pages of 1: 1.66 ms (2.18 with one
// warp, 12.1 on the row kernel; in pages of 64, by TMA, 0.72).
struct Pending {
    int count = 0;                      // stages not handed on yet
    int at[3];                          // which, the oldest first
};

template <int kLeft> __device__ __forceinline__ void hand_on(TileSmem &h, Pending &q)
{
    if (q.count <= kLeft)
        return;
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    while (q.count > kLeft) {
        if (elect_one())
            bar_arrive(&h.full[q.at[0]]);
        __syncwarp();
        q.at[0] = q.at[1];
        q.at[1] = q.at[2];
        --q.count;
    }
}

template <int DP>
__device__ bool produce_odd(const PagedArgs &a, const CUtensorMap &tq, TileSmem &h, unsigned char *qs, unsigned char *stages,
                            PagedWalk<kKeys> &walk, const PagedCut &cut, int32_t unit, int side, uint32_t &queries, PagedSeen &seen)
{
    using Shape = TileShape<DP>;
    constexpr int S = Shape::kStages;
    const int lane = threadIdx.x & 31;
    const unsigned char *base = static_cast<const unsigned char *>(side ? a.v : a.k);
    RingPos pos;
    Pending q;
    for (uint32_t npc = 0;; ++npc) {
        TilePiece t;
        if (side == 0) {
            PagedPiece p{};
            const bool more = walk.next(p);
            t.blocks = 0;
            if (more) {
                t = tile_piece(a, walk.s, p, cut, unit);
                seen.note(p);
            }
            hand_on<0>(h, q);
            if (!warp_wait(&h.pcempty[npc % kPieces], ((npc / kPieces) & 1u) ^ 1u, &h.abort_flag))
                return false;
            if (elect_one()) {
                h.piece[npc % kPieces] = t;
                bar_arrive(&h.pcfull[npc % kPieces]);
            }
            __syncwarp();
        } else {
            hand_on<0>(h, q);
            if (!warp_wait(&h.pcfull[npc % kPieces], (npc / kPieces) & 1u, &h.abort_flag))
                return false;
            t = h.piece[npc % kPieces];
            __syncwarp();
            if (elect_one())
                bar_arrive(&h.pcempty[npc % kPieces]);
            __syncwarp();
        }
        if (t.blocks == 0)
            return true;
        if (side == 1) {
            if (!load_q<DP>(a, tq, h, qs, t, npc))
                return false;
            ++queries;
        }
        const int64_t row0 = t.r * a.table_stride, head = t.kvh * a.kv_head;
        // byte offsets of the rows of step i, four a lane: read a step ahead
        int64_t off[kKeys / 32];
        auto locate = [&](int32_t i) {
#pragma unroll
            for (int x = 0; x < kKeys / 32; ++x) {
                const int32_t key = (t.first + i) * kKeys + x * 32 + lane;
                off[x] = -1;
                if (i < t.blocks && key >= t.keep && key < t.len) {
                    const int32_t e = key / a.page, page = a.tables[row0 + e];
                    const bool in = page >= 0 && page < a.n_pages;
                    if (in)
                        off[x] = 2 * (page * a.kv_page + (key - e * a.page) * a.kv_token + head);
                    else
                        atomicOr(a.status, BSM_DEV_BOUNDS);
                    seen.gone |= !in;
                }
            }
        };
        auto load = [&]() -> bool {
            if (!__all_sync(0xffffffffu, bar_done(&h.empty[pos.s], pos.ph ^ 1u))) {
                hand_on<0>(h, q);
                if (!warp_wait(&h.empty[pos.s], pos.ph ^ 1u, &h.abort_flag))
                    return false;
            }
            const uint32_t st = saddr(stages) + static_cast<uint32_t>(pos.s * Shape::kStageBytes);
            const int c = lane & 7;
#pragma unroll 4
            for (int r4 = 0; r4 < kKeys; r4 += 4) {
                const int row = r4 + (lane >> 3);
                const int64_t at = h.where[side][row];
#pragma unroll
                for (int hf = 0; hf < Shape::kHalves; ++hf) {
                    const bool in = at >= 0 && hf * 64 + c * 8 < a.d;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                     st + hf * kHalfBytes + row * 128 + ((c ^ (row & 7)) << 4)),
                                 "l"(base + (in ? at + (hf * 64 + c * 8) * 2 : 0)), "r"(in ? 16u : 0u)
                                 : "memory");
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            q.at[q.count == 0 ? 0 : q.count == 1 ? 1 : 2] = pos.s;
            ++q.count;
            hand_on<2>(h, q);
            return true;
        };
        // K0 V0 K1 V1 .., dual K0 K1 V0 K2 V1 ..
        const int32_t lag = t.dual ? 1 : 0;
        locate(0);
        for (int32_t i = 0; i < t.blocks + lag; ++i) {
            for (int sd = 0; sd < 2; ++sd) {
                const int32_t step = sd ? i - lag : i;
                if (step < 0 || step >= t.blocks)
                    continue;
                if (sd == side) {
                    __syncwarp();           // the rows of the step before have been read
#pragma unroll
                    for (int x = 0; x < kKeys / 32; ++x)
                        h.where[side][x * 32 + lane] = off[x];
                    __syncwarp();
                    locate(step + 1);
                    if (!load())
                        return false;
                }
                pos.step(S);
            }
        }
    }
}

// ------------------------------------------------------------- tensor cores
// One warp per softmax group.  Both go through all stages; of a stage that is
// the other group's alone it only takes note.
template <int DP, bool kF16, int kFill>
__device__ bool multiply(TileSmem &h, unsigned char *qs, unsigned char *stages, uint32_t tmem_, uint32_t sub_)
{
    using Shape = TileShape<DP>;
    using Steps = StageSteps<kFill>;
    constexpr uint32_t kScores = tile_idesc<kF16, kKeys, false>(), kOut = tile_idesc<kF16, DP, true>();
    const uint32_t tmem = uniform(tmem_);
    const int sub = static_cast<int>(uniform(sub_));
    RingPos pos;
    uint32_t np = 0, used = 0, turns = 0;   // steps' outputs issued; pieces with work; turns taken
    for (uint32_t npc = 0;; ++npc) {
        if (!warp_wait(&h.pcfull[npc % kPieces], (npc / kPieces) & 1u, &h.abort_flag))
            return false;
        const int32_t blocks = static_cast<int32_t>(uniform(static_cast<uint32_t>(h.piece[npc % kPieces].blocks)));
        const int32_t subs = static_cast<int32_t>(uniform(static_cast<uint32_t>(h.piece[npc % kPieces].subs)));
        const bool dual = uniform(static_cast<uint32_t>(h.piece[npc % kPieces].dual)) != 0;
        __syncwarp();
        if (elect_one())
            bar_arrive(&h.pcempty[npc % kPieces]);
        __syncwarp();
        if (blocks == 0)
            return true;
        if (!warp_wait(&h.qfull, npc & 1u, &h.abort_flag))
            return false;
        const bool active = sub < subs;
        const int32_t lead = dual ? 2 : 1;
        const int32_t from = dual ? sub : 0;            // this group's steps: from, from + lead .. last
        const int32_t last = dual ? blocks - 1 - ((blocks - 1 - sub) & 1) : blocks - 1;
        const uint64_t ad = smem_desc(qs + (dual ? 0 : sub) * (Shape::kHalves * kQHalf));
        if (!active && elect_one())
            bar_arrive(&h.qempty);
        __syncwarp();
        const uint32_t to_s = tmem + s_col(sub), to_o = tmem + o_col(sub);
        auto scores = [&](int32_t i, int stage) {
            const uint64_t kd = stage_desc_k<kFill>(saddr(stages) + static_cast<uint32_t>(stage * Shape::kStageBytes));
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
                mma_ss(to_s, ad + (d / 4) * (kQHalf >> 4) + (d % 4) * 2, kd + (d / 4) * (Steps::kHalf >> 4) + (d % 4) * 2,
                       kScores, d != 0);
            mma_commit(&h.sfull[sub]);
            mma_commit(&h.empty[stage]);
            if (i == last)
                mma_commit(&h.qempty);
        };
        // scores of the first steps
        for (int32_t i = 0; i < lead; ++i) {
            if (!warp_wait(&h.full[pos.s], pos.ph, &h.abort_flag))
                return false;
            tc_fence_after();
            const bool mine = active && (!dual || i == sub);
            if (elect_one()) {
                if (mine)
                    scores(i, pos.s);
                else
                    bar_arrive(&h.empty[pos.s]);
            }
            __syncwarp();
            pos.step(Shape::kStages);
        }
        // then the output of step j and the scores of step j + lead, whose keys are waited for
        // before the probabilities, so that nothing lies between the last product and them
        for (int32_t j = 0; j < blocks; ++j) {
            const bool mine = active && (!dual || (j & 1) == sub), more = j + lead < blocks;
            if (!warp_wait(&h.full[pos.s], pos.ph, &h.abort_flag))
                return false;
            const int vs = pos.s;
            pos.step(Shape::kStages);
            if (!mine) {
                if (elect_one())
                    bar_arrive(&h.empty[vs]);
                __syncwarp();
            } else {
                // the previous piece's output has been read
                if (j == from && !warp_wait(&h.ofree[sub], (used++ & 1u) ^ 1u, &h.abort_flag))
                    return false;
            }
            const uint64_t vd = stage_desc_v<kFill>(saddr(stages) + static_cast<uint32_t>(vs * Shape::kStageBytes));
            const int ks = pos.s;
            if (more) {
                if (!warp_wait(&h.full[ks], pos.ph, &h.abort_flag))
                    return false;
                pos.step(Shape::kStages);
            }
            // The groups take turns: products of both, issued at once, would be done at once, and
            // the groups' exponentials and products would go on at the same time, each leaving
            // the other's unit idle.  (The first group's turn at the start has no barrier.)
            if (mine && subs == 2) {
                if ((sub == 1 || turns > 0) && !warp_wait(&h.turn[sub], (turns - (sub == 0 ? 1u : 0u)) & 1u, &h.abort_flag))
                    return false;
                ++turns;
            }
            if (mine && !warp_wait(&h.pfull[sub], np++ & 1u, &h.abort_flag))
                return false;
            tc_fence_after();
            if (elect_one()) {
                if (mine) {
#pragma unroll
                    for (int k = 0; k < kKeys / 16; ++k)
                        mma_ts(to_o, to_s + k * 8, vd + k * (2 * Steps::kGroup >> 4), kOut, j != from || k != 0);
                    if (j == last)
                        mma_commit(&h.olast[sub]);
                    mma_commit(&h.empty[vs]);
                    if (more)
                        scores(j + lead, ks);
                    if (subs == 2)
                        bar_arrive(&h.turn[dual ? (j + 1 < blocks ? 1 - sub : 0) : 1 - sub]);
                } else if (more) {
                    bar_arrive(&h.empty[ks]);
                }
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------- softmax
__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Waits for this thread's loads from tensor memory; r[0 .. N-1] are used after it.
template <int N> __device__ __forceinline__ void tmem_landed(uint32_t *r)
{
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < N; ++i)
        asm volatile("" : "+r"(r[i]));
}

template <int DP, bool kF16>
__device__ bool softmax(const PagedArgs &a, TileSmem &h, unsigned char *store, uint32_t tmem, int sub_, int32_t unit)
{
    const int sub = static_cast<int>(uniform(static_cast<uint32_t>(sub_)));
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quarter = warp & 3;
    const int row = quarter * 32 + lane;                // of the row block
    const uint32_t lanes = uniform(tmem + (static_cast<uint32_t>(quarter * 32) << 16));
    const int32_t tt = row / a.sub, hh = row - tt * a.sub, half_tok = a.tok / 2;
    const uint64_t scale2 = pair(a.scale_log2, a.scale_log2);
    unsigned char *mine = store + warp * (32 * 64);
    uint32_t n = 0, pieces = 0, pieces1 = 0, duals = 0; // steps and pieces so far; pieces of the second group
    for (uint32_t npc = 0;; ++npc) {
        if (!warp_wait(&h.pcfull[npc % kPieces], (npc / kPieces) & 1u, &h.abort_flag))
            return false;
        TilePiece t = h.piece[npc % kPieces];
        __syncwarp();
        if (lane == 0)
            bar_arrive(&h.pcempty[npc % kPieces]);
        t.blocks = static_cast<int32_t>(uniform(static_cast<uint32_t>(t.blocks)));
        t.dual = static_cast<int32_t>(uniform(static_cast<uint32_t>(t.dual)));
        t.slot = static_cast<int32_t>(uniform(static_cast<uint32_t>(t.slot + 1))) - 1;
        t.first = static_cast<int32_t>(uniform(static_cast<uint32_t>(t.first)));
        if (t.blocks == 0)
            return true;
        if (sub >= t.subs)
            continue;
        const int32_t tok = (t.dual ? 0 : sub * half_tok) + tt;     // of the tile
        const bool live = tt < half_tok && tok < t.tokens && hh < t.heads;
        const bool idle = !__any_sync(0xffffffffu, live);
        // keys this row sees; rows that are not stored compute whatever comes
        int32_t lo = 0, hi = INT32_MAX;
        if (live) {
            hi = t.hi;
            if (a.causal) {
                hi = t.pos + tok + 1 < t.hi ? t.pos + tok + 1 : t.hi;
                if (a.window && t.pos + tok >= a.window)
                    lo = t.pos + tok - a.window + 1;
            }
        }
        float ref = -INFINITY, sum = 0.0f;              // reference (log2), sum of probabilities
        const int32_t j0 = t.dual ? sub : 0, dj = t.dual ? 2 : 1;
        for (int32_t j = j0; j < t.blocks; j += dj, ++n) {
            if (!warp_wait(&h.sfull[sub], n & 1u, &h.abort_flag))
                return false;
            tc_fence_after();
            if (idle) {
                // no row of this warp is stored: whatever lies there will do
                __syncwarp();
                if (lane == 0) {
                    bar_arrive(&h.pfull[sub]);
                }
                continue;
            }
            const uint32_t sc = lanes + s_col(sub);
            uint32_t r[kKeys];
            tmem_ld32_nowait(sc, r);
            tmem_ld32_nowait(sc + 32, r + 32);
            const int32_t key0 = (t.first + j) * kKeys;
            const bool masked = !__all_sync(0xffffffffu, lo <= key0 && hi - kKeys >= key0);
            const int32_t c0 = lo - key0, c1 = hi - key0;
            float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int q = 0; q < kKeys; q += 64) {
                tmem_landed<64>(r + q);
                if (q == 0) {
                    tmem_ld32_nowait(sc + 64, r + 64);
                    tmem_ld32_nowait(sc + 96, r + 96);
                }
                if (masked) {
                    // 32 columns at a time, and only the side that cuts them
#pragma unroll
                    for (int g = q; g < q + 64; g += 32) {
                        if (__any_sync(0xffffffffu, c1 < g + 32)) {
#pragma unroll
                            for (int c = g; c < g + 32; ++c)
                                r[c] = c < c1 ? r[c] : 0xFF800000u;
                        }
                        if (__any_sync(0xffffffffu, c0 > g)) {
#pragma unroll
                            for (int c = g; c < g + 32; ++c)
                                r[c] = c >= c0 ? r[c] : 0xFF800000u;
                        }
                    }
                }
#pragma unroll
                for (int c = q; c < q + 64; c += 2)
                    top4[(c >> 1) & 3] =
                        fmaxf(fmaxf(top4[(c >> 1) & 3], __uint_as_float(r[c])), __uint_as_float(r[c + 1]));
            }
            const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * a.scale_log2;
            // (a maximum of -inf moves nothing; NaN neither: it comes out in the sum)
            const bool move = top > ref + kLag;
            if (__any_sync(0xffffffffu, move)) {
                const float f = !move ? 1.0f : pg_exp2(ref - top);
                ref = move ? top : ref;
                sum *= f;
                if (j != j0) {
                    // the products of earlier steps are done: this step's scores were issued behind them
#pragma unroll 1
                    for (int c = 0; c < DP / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld16(lanes + o_col(sub) + c * 16, o);
                        tmem_landed<16>(o);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st16(lanes + o_col(sub) + c * 16, o);
                    }
                }
            }
            const float base = ref == -INFINITY ? 0.0f : ref - pg_shift<kF16>(kLag);
            const uint64_t base2 = pair(-base, -base);
            uint64_t s2[2] = {0, 0};
#pragma unroll
            for (int q = 0; q < kKeys; q += 32) {
                uint32_t pr[16];
#pragma unroll
                for (int c = q; c < q + 32; c += 2) {
                    float p0, p1;
                    unpair(fma2(pair(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), scale2, base2), p0, p1);
                    p0 = pg_exp2(p0);
                    p1 = pg_exp2(p1);
                    s2[(c >> 1) & 1] = add2(s2[(c >> 1) & 1], pair(p0, p1));
                    pr[(c - q) / 2] = pg_pack<kF16>(p0, p1);
                }
                tmem_st16(sc + q / 2, pr);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                bar_arrive(&h.pfull[sub]);
            float e0, e1;
            unpair(add2(s2[0], s2[1]), e0, e1);
            sum += e0 + e1;
        }
        // ---- the row's output
        if (!warp_wait(&h.olast[sub], pieces++ & 1u, &h.abort_flag))
            return false;
        pieces1 += t.subs == 2 ? 1 : 0;
        float base = ref - pg_shift<kF16>(kLag), f0 = 1.0f, f1 = 0.0f;
        if (t.dual) {
            if (sub == 1) {
                // the first group adds and stores both outputs
                h.other[row] = make_float2(base, sum);
                __syncwarp();
                if (lane == 0)
                    bar_arrive(&h.xfull);
                continue;
            }
            if (!warp_wait(&h.xfull, duals & 1u, &h.abort_flag) ||
                !warp_wait(&h.olast[1], (pieces1 & 1u) ^ 1u, &h.abort_flag))
                return false;
            ++duals;
            const float2 x = h.other[row];
            const float both = fmaxf(base, x.x), at = both == -INFINITY ? 0.0f : both;
            f0 = pg_exp2(base - at);
            f1 = pg_exp2(x.x - at);
            sum = f0 * sum + f1 * x.y;
            base = both;
        }
        tc_fence_after();
        const int64_t token = t.token + tok;
        const int64_t off = 2 * (token * a.out_token + (t.head + hh) * a.out_head);
        const int srow = (t.dual ? 0 : sub) * 128 + row;
        float *part = a.part_o + static_cast<int64_t>(t.slot) * (kPagedTileRows * kPagedMaxDim) + srow * 4;
        if (t.slot < 0) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            f0 *= inv;
            f1 *= inv;
        }
        uint64_t odd[2] = {0, 0};                       // sums of the outputs: not finite if one of them is not
#pragma unroll 1
        for (int c = 0; c < DP / 32 && !idle; ++c) {
            uint32_t o[32];
            float f[32];
            tmem_ld32_nowait(lanes + o_col(sub) + c * 32, o);
            tmem_landed<32>(o);
#pragma unroll
            for (int i = 0; i < 32; ++i)
                f[i] = __uint_as_float(o[i]) * f0;
            if (t.dual) {
                tmem_ld32_nowait(lanes + o_col(1) + c * 32, o);
                tmem_landed<32>(o);
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    f[i] = fmaf(__uint_as_float(o[i]), f1, f[i]);
            }
            if (t.slot < 0) {
#pragma unroll
                for (int i = 0; i < 32; i += 2)
                    odd[(i >> 1) & 1] = add2(odd[(i >> 1) & 1], pair(f[i], f[i + 1]));
                // through shared memory, so that four lanes store 64 bytes of a row (a lane storing
                // its own row touches 32 lines at once); 16-byte pieces swizzled over the banks
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4 w;
                    w.x = pg_pack<kF16>(f[8 * i], f[8 * i + 1]);
                    w.y = pg_pack<kF16>(f[8 * i + 2], f[8 * i + 3]);
                    w.z = pg_pack<kF16>(f[8 * i + 4], f[8 * i + 5]);
                    w.w = pg_pack<kF16>(f[8 * i + 6], f[8 * i + 7]);
                    *reinterpret_cast<uint4 *>(mine + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = w;
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = i * 8 + (lane >> 2), k = lane & 3;
                    const int64_t to = __shfl_sync(0xffffffffu, off, r);
                    const bool ok = __shfl_sync(0xffffffffu, live ? 1 : 0, r) != 0;
                    const uint4 w = *reinterpret_cast<const uint4 *>(mine + r * 64 + ((k ^ ((r >> 1) & 3)) << 4));
                    if (ok && c * 32 + k * 8 < a.d)
                        *reinterpret_cast<uint4 *>(static_cast<unsigned char *>(a.out) + to + (c * 32 + k * 8) * 2) = w;
                }
                __syncwarp();
            } else {
                // four columns of a row together, rows side by side: a warp stores 512 bytes at once
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<float4 *>(part + static_cast<int64_t>(c * 8 + i) * (kPagedTileRows * 4)) =
                        make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            bar_arrive(&h.ofree[sub]);
            if (t.dual)
                bar_arrive(&h.ofree[1]);
        }
        float odd0, odd1;
        unpair(add2(odd[0], odd[1]), odd0, odd1);
        if (live && !pg_finite(odd0 + odd1))
            *static_cast<volatile int32_t *>(&h.odd) = 1;
        if (t.slot < 0) {
            if (live && a.lse)
                a.lse[token * a.heads_q + t.head + hh] =
                    sum == 0.0f ? -INFINITY : (base + log2f(sum)) * kPagedLn2;
        } else {
            *reinterpret_cast<float2 *>(a.part_ml + (static_cast<int64_t>(t.slot) * kPagedTileRows + srow) * 2) =
                make_float2(base, sum);
        }
        if (t.join > 0 && sub == 0 && threadIdx.x == 0) {
            PagedJoin &j = a.join[unit];                // (its flags are others')
            j.token = t.token;
            j.head = t.head;
            j.tokens = t.tokens;
            j.heads = t.heads;
            j.count = t.join;
        }
    }
}

template <int DP, bool kF16, int kFill>
__global__ void __launch_bounds__(kTileThreads, 1)
    paged_tiles(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                const __grid_constant__ CUtensorMap tv, const PagedArgs a, const int box, const int per_page)
{
    using Shape = TileShape<DP>;
    extern __shared__ __align__(1024) unsigned char raw[];
    unsigned char *smem = raw + ((1024u - (saddr(raw) & 1023u)) & 1023u);
    TileSmem &h = *reinterpret_cast<TileSmem *>(smem);
    unsigned char *store = smem + kTileHeader, *qs = store + kStore, *stages = qs + Shape::kQBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int32_t unit = blockIdx.x;
    if (threadIdx.x == 0) {
        for (int s = 0; s < Shape::kStages; ++s) {
            bar_init(&h.full[s], 1);
            bar_init(&h.empty[s], 2);
        }
        bar_init(&h.qfull, 1);
        bar_init(&h.qempty, 2);
        for (int s = 0; s < 2; ++s) {
            bar_init(&h.sfull[s], 1);
            bar_init(&h.pfull[s], 4);
            bar_init(&h.olast[s], 1);
            bar_init(&h.ofree[s], 4);
            bar_init(&h.turn[s], 1);
        }
        for (int s = 0; s < kPieces; ++s) {
            bar_init(&h.pcfull[s], 1);
            bar_init(&h.pcempty[s], 11);
        }
        bar_init(&h.tail, 1);
        bar_init(&h.drain, 2);
        bar_init(&h.xfull, 4);
        h.abort_flag = h.no_abort = h.odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_dependency_wait();
    grid_launch_dependents();
    if (threadIdx.x == 0) {
        a.join[unit].count = 0;
        a.join[unit].flags = 0;
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
    const uint32_t tmem = __shfl_sync(0xffffffffu, h.tmem_base, 0);

    bool ok;
    if (warp == 8) {
        uint32_t loaded = 0;
        uint32_t none = 0;
        PagedSeen seen;
        if (kFill == kOddPages)
            ok = produce_odd<DP>(a, tq, h, qs, stages, walk, cut, unit, 0, none, seen);
        else
            ok = produce<DP, kFill>(a, tk, tv, box, per_page, h, stages, walk, cut, unit, loaded, seen);
        seen.store(a.join[unit]);
        __syncwarp();
        if (!ok) {
            if (elect_one()) {
                atomicOr(a.status, BSM_DEV_TIMEOUT);
                h.abort_flag = 1;
            }
            __syncwarp();
        }
        // copies in flight land before the CTA leaves
        if (kFill == kOddPages)
            asm volatile("cp.async.wait_all;" ::: "memory");
        const uint32_t S = Shape::kStages;
        for (uint32_t j = loaded > S ? loaded - S : 0u; j < loaded; ++j)
            warp_drain(h, &h.full[j % S], (j / S) & 1u);
    } else if (warp == 11) {
        uint32_t loaded = 0;
        PagedSeen seen;                 // (the warp of the keys tells)
        if (kFill == kOddPages)
            ok = produce_odd<DP>(a, tq, h, qs, stages, walk, cut, unit, 1, loaded, seen);
        else
            ok = produce_q<DP>(a, tq, h, qs, loaded);
        if (!ok) {
            if (elect_one()) {
                atomicOr(a.status, BSM_DEV_TIMEOUT);
                h.abort_flag = 1;
            }
            __syncwarp();
        }
        if (kFill == kOddPages)
            asm volatile("cp.async.wait_all;" ::: "memory");
        if (loaded)
            warp_drain(h, &h.qfull, (loaded - 1) & 1u);
    } else if (warp >= 9) {
        ok = multiply<DP, kF16, kFill>(h, qs, stages, tmem, warp - 9);
        if (elect_one()) {
            if (!ok) {
                atomicOr(a.status, BSM_DEV_TIMEOUT);
                h.abort_flag = 1;
            }
            mma_commit(&h.drain);
        }
        __syncwarp();
        // every product has finished before the tensor memory is freed
        warp_drain(h, &h.drain, 0);
    } else {
        ok = softmax<DP, kF16>(a, h, store, tmem, warp >> 2, unit);
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
    if (threadIdx.x == 0 && h.odd)
        atomicOr(&a.join[unit].flags, kPagedOdd);
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTileTmemCols) : "memory");
    }
}

// Joins the parts of every cut tile (the sums of the row kernel's RowSum): a
// thread a row and kCols columns, kShares threads a row where there are many parts
// (few tiles), each with its share of them.
// Whether an output of this thread is not finite comes back.
template <bool kF16, int kCols, int kShares>
__device__ __forceinline__ bool tile_join(const PagedArgs &a, const PagedJoin &j, int unit, int sub, float *other)
{
    const int half_tok = a.tok / 2, lane_row = threadIdx.x & 127, share = threadIdx.x >> 7;
    const int tt = lane_row / a.sub, h = lane_row - tt * a.sub, tok = sub * half_tok + tt;
    const bool live = tt < half_tok && tok < j.tokens && h < j.heads;
    const int row = sub * 128 + lane_row;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
    const float4 *po = reinterpret_cast<const float4 *>(a.part_o);
    auto slot = [&](int i) { return static_cast<int64_t>(i == 0 ? 2 * unit + 1 : 2 * (unit + i)); };
    const int from = j.count * share / kShares, to = j.count * (share + 1) / kShares;
    float4 acc[kCols / 4] = {};
    float sum = 0.0f, top = -INFINITY;
    if (live) {
#pragma unroll 8
        for (int i = from; i < to; ++i)
            top = fmaxf(top, ml[slot(i) * kPagedTileRows + row].x);
        const float ref = top == -INFINITY ? 0.0f : top;
        const int c = blockIdx.z * (kCols / 4);
#pragma unroll(kCols == 32 ? 2 : 8)
        for (int i = from; i < to; ++i) {
            const float2 m = ml[slot(i) * kPagedTileRows + row];
            const float f = pg_exp2(m.x - ref);
            sum += f * m.y;
#pragma unroll
            for (int k = 0; k < kCols / 4; ++k) {
                const float4 v = po[(slot(i) * (kPagedMaxDim / 4) + c + k) * kPagedTileRows + row];
                acc[k].x += f * v.x;
                acc[k].y += f * v.y;
                acc[k].z += f * v.z;
                acc[k].w += f * v.w;
            }
        }
    }
    if (kShares > 1) {
        // [share - 1][column, then sum and top][row]
        float *mine = other + (share - 1) * 128 * (kCols + 2) + lane_row;
        if (share > 0) {
#pragma unroll
            for (int k = 0; k < kCols / 4; ++k) {
                mine[(4 * k) * 128] = acc[k].x;
                mine[(4 * k + 1) * 128] = acc[k].y;
                mine[(4 * k + 2) * 128] = acc[k].z;
                mine[(4 * k + 3) * 128] = acc[k].w;
            }
            mine[kCols * 128] = sum;
            mine[(kCols + 1) * 128] = top;
        }
        __syncthreads();
        if (share > 0)
            return false;
        float all = top;
        for (int s = 0; s < kShares - 1; ++s)
            all = fmaxf(all, other[(s * (kCols + 2) + kCols + 1) * 128 + lane_row]);
        const float ref = all == -INFINITY ? 0.0f : all;
        const float f0 = pg_exp2(top - ref);
        sum *= f0;
#pragma unroll
        for (int k = 0; k < kCols / 4; ++k) {
            acc[k].x *= f0;
            acc[k].y *= f0;
            acc[k].z *= f0;
            acc[k].w *= f0;
        }
        for (int s = 0; s < kShares - 1; ++s) {
            const float *o = other + s * 128 * (kCols + 2) + lane_row;
            const float f = pg_exp2(o[(kCols + 1) * 128] - ref);
            sum += f * o[kCols * 128];
#pragma unroll
            for (int k = 0; k < kCols / 4; ++k) {
                acc[k].x += f * o[(4 * k) * 128];
                acc[k].y += f * o[(4 * k + 1) * 128];
                acc[k].z += f * o[(4 * k + 2) * 128];
                acc[k].w += f * o[(4 * k + 3) * 128];
            }
        }
        top = all;
    }
    if (!live)
        return false;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    float odd = 0.0f;
    const int64_t token = j.token + tok;
    unsigned char *out = static_cast<unsigned char *>(a.out) + 2 * (token * a.out_token + (j.head + h) * a.out_head);
#pragma unroll
    for (int k = 0; k < kCols / 4; k += 2) {
        const int col = blockIdx.z * kCols + k * 4;
        uint4 w;
        w.x = pg_pack<kF16>(acc[k].x * inv, acc[k].y * inv);
        w.y = pg_pack<kF16>(acc[k].z * inv, acc[k].w * inv);
        w.z = pg_pack<kF16>(acc[k + 1].x * inv, acc[k + 1].y * inv);
        w.w = pg_pack<kF16>(acc[k + 1].z * inv, acc[k + 1].w * inv);
        odd += pg_total(acc[k]) + pg_total(acc[k + 1]);
        if (col < a.d)
            *reinterpret_cast<uint4 *>(out + col * 2) = w;
    }
    if (a.lse && blockIdx.z == 0)
        a.lse[token * a.heads_q + j.head + h] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kPagedLn2;
    return !pg_finite(odd);
}

// The join, then what the units' flags ask for: rows once more.
// (CTAs an SM: with what the compiler takes by itself the join's loads go through spilled
// addresses; 2 x 4 tokens over 131 thousand keys 179 us, 170 so.)
template <bool kF16, int kCols, int kShares>
__global__ void __launch_bounds__(128 * kShares, kShares > 1 ? 2 : 5) paged_tile_join(const PagedArgs a)
{
    __shared__ float other[kShares > 1 ? (kShares - 1) * 128 * (kCols + 2) : 1];
    const int unit = blockIdx.x, sub = blockIdx.y;
    grid_dependency_wait();
    grid_launch_dependents();
    const PagedJoin j = a.join[unit];
    uint32_t flags = 0;                                 // a page missing in a part of the cut tile; its own rows odd
    for (int i = threadIdx.x; i < j.count; i += 128 * kShares)
        flags |= a.join[unit + i].flags & kPagedGone;
    if (j.count > 0 && tile_join<kF16, kCols, kShares>(a, j, unit, sub, other))
        flags |= kPagedOdd;
    const bool parts = __syncthreads_or(flags != 0);
    if (parts || j.flags) {
        const bool gone = __syncthreads_or((flags | j.flags) & kPagedGone);
        constexpr int kWarps = 4 * kShares;
        const int warp = threadIdx.x >> 5, half_tok = a.tok / 2;
        paged_unit_again<kF16>(a, j, j.flags != 0, parts, gone, (blockIdx.z * gridDim.y + sub) * kWarps + warp,
                               gridDim.z * gridDim.y * kWarps, blockIdx.z * kCols, (blockIdx.z + 1) * kCols,
                               [&](int32_t t, int32_t h) { return t / half_tok == sub && (t * a.sub + h) % kWarps == warp; });
    }
}

template <bool kF16, int kCols, int kShares> int launch_join(const PagedArgs &a, cudaStream_t st)
{
    return launch_early(paged_tile_join<kF16, kCols, kShares>, dim3(a.units, 2, (a.d + kCols - 1) / kCols), 128 * kShares, 0,
                        st, a);
}

template <int DP, bool kF16>
int launch(const CUtensorMap *m, const PagedArgs &a, int box, int per_page, int64_t tiles, cudaStream_t st)
{
    // (halves side by side: heads of 128 only)
    const auto kernel = box < 8 ? paged_tiles<DP, kF16, kOddPages>
                        : DP == 128 && per_page ? paged_tiles<DP, kF16, DP == 128 ? kByRows : kByHalves>
                                                : paged_tiles<DP, kF16, kByHalves>;
    if (int e = launch_early(kernel, dim3(a.units), kTileThreads, TileShape<DP>::kSmem, st, m[0], m[1], m[2], a, box,
                             per_page))
        return e;
    // Tiles of ten parts and more: more CTAs, four threads to a row's parts.  16 tokens
    // over 100 thousand keys, one key/value head: 41.6 us in all, 112 the other way; 64
    // tokens over 8000 keys, 8 key/value heads: 28 and 33.
    return tiles * 10 <= a.units ? launch_join<kF16, 8, 4>(a, st) : launch_join<kF16, 32, 1>(a, st);
}

}  // namespace

int launch_paged_tiles(const void *maps, const PagedArgs &a, bool f16, int box, int per_page, void *stream)
{
    const CUtensorMap *m = static_cast<const CUtensorMap *>(maps);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // tiles of the batch, each request having one at least
    const int64_t tiles = static_cast<int64_t>(a.n > a.n_tokens / a.tok ? a.n : a.n_tokens / a.tok) * a.heads_kv * a.subs;
    if (a.d <= 64)
        return f16 ? launch<64, true>(m, a, box, per_page, tiles, st) : launch<64, false>(m, a, box, per_page, tiles, st);
    return f16 ? launch<128, true>(m, a, box, per_page, tiles, st) : launch<128, false>(m, a, box, per_page, tiles, st);
}

int paged_tiles_set_smem()
{
    int e = 0;
    auto set = [&](const void *f, int bytes) {
        if (!e)
            e = static_cast<int>(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    };
    set(reinterpret_cast<const void *>(&paged_tiles<64, false, kByHalves>), TileShape<64>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<64, true, kByHalves>), TileShape<64>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<64, false, kOddPages>), TileShape<64>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<64, true, kOddPages>), TileShape<64>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, false, kByHalves>), TileShape<128>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, true, kByHalves>), TileShape<128>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, false, kByRows>), TileShape<128>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, true, kByRows>), TileShape<128>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, false, kOddPages>), TileShape<128>::kSmem);
    set(reinterpret_cast<const void *>(&paged_tiles<128, true, kOddPages>), TileShape<128>::kSmem);
    return e;
}

}  // namespace bsm
