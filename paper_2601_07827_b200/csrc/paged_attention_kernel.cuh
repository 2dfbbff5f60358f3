// Attention of one new token per sequence over a paged key-value cache.
//
//   o[h] = sum_j softmax_j(scale q[h] . k_j) v_j   over the visible tokens j of the sequence
//
// Every visible key and value is read once and used by the query heads that share it: 2 * group
// multiply-adds per element, far below what the tensor cores need to be busy, so the pass is bound by
// HBM and everything here serves to keep copies in flight:
//   * a warp is a pipeline of its own: it copies tiles of 16 tokens (keys and values of one key head) into
//     a ring of `STAGES` buffers with 16-byte cp.async and consumes them without any CTA barrier.  Eight
//     warps with two tiles of 8 KB in flight each are 128 KB per SM.
//   * S^T = K Q^T and O^T = V^T P^T with mma.sync: tokens are the M side of the first product and head
//     elements that of the second, so 8 query heads fill the N side (with the heads on the M side half
//     of each product would be padding for groups of 8), and P needs only a transpose of 8 x 8 blocks.
//     The products are a few percent of the time; mma.sync keeps them in registers of the warp that
//     copied the tile, where tcgen05's 128-row tiles would be 15/16 empty.
//   * 16-bit types: P is split in two (p = hi + lo, products with both): f16 then holds 22 bits of it, bf16 16,
//     2^-17 of a probability left out at most, a 256th of what the output's own rounding leaves out (a third part
//     would be half as many products again).  fp32: each product is formed from three TF32 products
//     (x = hi + lo; lo * lo is dropped, at most 2^-22 of the product), as in the contractions.
//   * running maximum, sum and output in fp32 (the flash form); the output is rescaled only when a maximum moved.
//     The tensor core adds up the tokens of one tile; tiles are added in fp32, rounded to nearest.  The tensor core cuts
//     its sums off, always towards zero: over the 7000 tiles of a warp whole outputs fell short by 4e-4 (f16 and
//     bf16), as much as f16's own rounding.  The additions cost 0 to 3 % (heads of 128: 64 ragged requests 79.3 -> 79.5 us,
//     with groups of 16 109 -> 113 us).
// Work.  The tiles of all (sequence, key head) pairs form one list; CTAs and in them warps take equal
// contiguous shares of it, whatever the lengths are, found on the device from a prefix sum of the tile
// counts (the host never reads a length).  What a warp cannot finish is merged in shared memory by its
// CTA, what a CTA cannot finish goes to the workspace and a second small kernel joins it, in a fixed order.
// Measured (replayed graphs): 8 x 128 Ki tokens of f16 (4.3 GB) 650 us = 6.6 TB/s, the measured copy bandwidth; 64 requests of 64 to
// 8192 tokens (0.44 GB) 79 us; one request of 1500 tokens 11.8 us, nearly all of it latency.
#pragma once

#include "../../include/btc.h"
#include "decoder_common.cuh"

#include <type_traits>

namespace btc {

constexpr int kAttnTok = 16;                 // tokens per tile
constexpr int kAttnMaxDim = 256;
// What beginning and ending an item (a sequence's key head) costs, in tiles: about 2 us, when a tile takes 1.3.  The list
// of tiles is cut into equal shares of tiles plus this for every item; counted by tiles alone, the CTA with
// the shortest sequences of a ragged batch ran 17 us longer than the others' 68.
constexpr int kAttnItemTiles = 2;
constexpr int kAttnMaxSequences = 1 << 23;   // tiles and sequences are counted in one 64-bit prefix sum

struct AttentionParams {
    const void *q, *k, *v;
    void *o;
    const int32_t *table, *lengths;
    float *lse;                              // [sequences][query heads] or NULL
    int32_t *flags;
    float *partial;                          // workspace: [CTA][2][8 NT heads x DP values, then maxima, then sums]
    int32_t *partial_item;                   // workspace: [CTA][2] item, -1: none
    int64_t q_n, q_h, q_d, o_n, o_h, o_d;
    int64_t k_page, k_slot, k_head, k_d, v_page, v_slot, v_head, v_d;
    int64_t table_n, table_j;
    int32_t sequences, heads, key_heads, group, blocks;   // blocks: groups of 8 NT query heads per key head
    int32_t dim_k, dim_v, pages, columns;
    int32_t window;                          // 0: everything up to the length is visible
    int32_t room;                            // tokens a table row can hold
    int32_t whole_tiles;                     // vec_k and vec_v, and pages of whole tiles (16) or half tiles (8); 0: neither
    int32_t vec_k, vec_v, vec_q;             // 16-byte copies of keys / values, 4-byte loads of queries
    FastDiv page;
    float scale_log2;                        // scale * log2(e)
    // trees of drafted tokens (TREE): `group` counts the rows that share a key head, drafts * sharing of them: row r is draft r / sharing
    const int32_t *masks;                    // [sequences][drafts][words]
    int64_t q_t, o_t, m_n, m_t, m_w;
    int32_t drafts, words;
    FastDiv sharing;                         // query heads of a draft that share a key head
};

// Per-warp ring and warps of a CTA: as many as 224 KB of shared memory hold.  fp32 tiles of 12 KB and more take
// two stages and more warps instead of three (a tile is then 1000 instructions of products; what is
// in flight, one tile of every warp, is still 96 KB).
template <typename T, int DP, int NT> struct AttentionShape {
    static constexpr int ROW = DP * int(sizeof(T));              // bytes of a token's row of one tensor
    static constexpr int STAGE = 2 * kAttnTok * ROW;             // keys and values
    static constexpr int DEPOSIT = 8 * NT * DP * 4;              // an unfinished item's output
    static constexpr int STAGES = STAGE <= 4096 ? 6 : (sizeof(T) == 4 && STAGE > 8192 ? 2 : 3);
    static constexpr int RING = STAGES * STAGE;
    static constexpr int FIT = 224 * 1024 / (RING + DEPOSIT);
    static constexpr int WARPS = FIT < 8 ? FIT : 8;
    static constexpr int SMEM = WARPS * (RING + DEPOSIT);
    static_assert(RING >= DEPOSIT, "the last item's deposit takes the warp's ring");
    static_assert(WARPS * DEPOSIT >= (WARPS * 32 + 1) * 8, "the prefix sum takes the first items' place");
};

template <typename T> struct AttentionBias { static constexpr float value = 0.f, factor = 1.f; };
// f16 products: probabilities are kept 2^10 times larger (they cancel against the sum), so that values down to
// 2^-24 of the largest stay normal numbers.  The factor is applied to the probability, which is exact: as an addend to
// the score it would be rounded where scores are large (beyond 2^25 it changed from maximum to maximum, at 2^27 the
// largest probability became 2^16, more than f16 holds).
template <> struct AttentionBias<__half> { static constexpr float value = 10.f, factor = 1024.f; };

// The code of a kernel that runs for a few microseconds is fetched as it goes: a jump over code that is not needed costs
// about a third of a microsecond.  What is rarely needed is marked so that it is put out of the way.
__device__ __forceinline__ bool rare(bool x) { return __builtin_expect(x, 0); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma8_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x = hi + lo with hi rounded to TF32's 11 significant bits, so that |lo| <= 2^-11 |x|; of lo the tensor core takes
// the leading 11 bits (it ignores the low 13 of what it is given): at most 2^-21 |x| is left out
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t &hi, uint32_t &lo)
{
    hi = (x + 0x1000u) & 0xffffe000u;
    lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(hi));
}
// the products with x0, x1: lo * hi, hi * lo and hi * hi, each into an accumulator
__device__ __forceinline__ void mma8_split(float (&c_lh)[4], float (&c_hl)[4], float (&c_hh)[4], const uint32_t (&ah)[4],
                                           const uint32_t (&al)[4], uint32_t x0, uint32_t x1)
{
    uint32_t h0, l0, h1, l1;
    split_tf32(x0, h0, l0);
    split_tf32(x1, h1, l1);
    mma8_tf32(c_lh, al, h0, h1);
    mma8_tf32(c_hl, ah, l0, l1);
    mma8_tf32(c_hh, ah, h0, h1);
}
// copies `bytes` (0..16) and fills the rest of the 16 with zeros
__device__ __forceinline__ void cp_async_part(unsigned dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait_group() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// visible tokens [begin, end) of a sequence, and its tiles, which start at multiples of 16 tokens.  TREE: those that any draft
// may see; the drafts lie behind the `cached` tokens.
template <bool TREE> struct AttentionSpan {
    int32_t begin, end, first_tile, tiles, cached;
    __device__ __forceinline__ void set(const AttentionParams &p, int32_t length)
    {
        const int32_t room = p.room;
        end = length < 0 ? 0 : (length > room ? room : length);
        if constexpr (TREE) {
            cached = end;
            begin = p.window > 0 && cached >= p.window ? cached + 1 - p.window : 0;
            end = min(cached + p.drafts, room);
        } else {
            cached = 0;
            begin = p.window > 0 && end > p.window ? end - p.window : 0;
        }
        first_tile = begin / kAttnTok;
        tiles = end / kAttnTok + (end % kAttnTok != 0) - first_tile;
    }
    __device__ __forceinline__ static bool bad(const AttentionParams &p, int32_t length) { return length < 0 || length > p.room; }
    // Is it an error by itself that token t has no page?  (Drafts: see report_drafts.)
    __device__ __forceinline__ bool needs_page(int32_t t) const { return !TREE || t < cached; }
};

// TREE: a warp reports drafts without a page or without room, of every gridDim.x-th sequence, where a row sees them: what no row sees
// needs neither.  Apart from the loops that look pages up, which have no registers to spare for the masks, and at their end.
__device__ __forceinline__ void report_drafts(const AttentionParams &p, int lane)
{
    if (!p.flags) return;
#pragma unroll 1
    for (int s = blockIdx.x; s < p.sequences; s += gridDim.x) {
        AttentionSpan<true> span;
        span.set(p, p.lengths[s]);
#pragma unroll 1
        for (int d = lane; d < p.drafts; d += 32) {
            const int32_t t = span.cached + d;
            int32_t page = -1;
            if (t < span.end) page = p.table[s * p.table_n + int64_t(p.page.div(uint32_t(t))) * p.table_j];
            if (page >= 0 && page < p.pages) continue;
            uint32_t seen = 0;
            const int32_t *mask = p.masks + s * p.m_n + (d >> 5) * p.m_w;
#pragma unroll 4
            for (int i = 0; i < p.drafts; ++i, mask += p.m_t) seen |= uint32_t(*mask);
            if ((seen >> (d & 31)) & 1u) atomicOr(p.flags, int(t < span.end ? BTC_FLAG_BAD_PAGE : BTC_FLAG_BAD_LENGTH));
        }
    }
}

// n / d for n >= 0 and d > 0; a 64-bit division is several times as long as a 32-bit one
__device__ __forceinline__ int64_t divide(int64_t n, int32_t d)
{
    if (__builtin_expect(n >= (int64_t(1) << 31), 0)) return n / d;
    return int64_t(uint32_t(n) / uint32_t(d));
}

// Where row `r` of a key head's group lies: TREE: which draft it is of, and which query head
template <bool TREE> __device__ __forceinline__ int32_t attention_row(const AttentionParams &p, int32_t key_head, int32_t r, int32_t &draft)
{
    if constexpr (!TREE) {
        draft = 0;
        return key_head * p.group + r;
    }
    draft = int32_t(p.sharing.div(uint32_t(r)));
    return key_head * int32_t(p.sharing.d) + r - draft * int32_t(p.sharing.d);
}

// A place in the list of tiles: sequence, head block, tile; the same in every lane.
template <bool TREE> struct AttentionCursor {
    int32_t seq, hb, tile;                   // tile counted from the span's first
    int32_t key_head, block;                 // hb = key_head * blocks + block
    AttentionSpan<TREE> span;
    __device__ __forceinline__ void next(const AttentionParams &p)
    {
        if (++tile < span.tiles) return;
        tile = 0;
        ++hb;
        if (++block < p.blocks) return;
        block = 0;
        if (++key_head < p.key_heads) return;
        hb = key_head = 0;
        span.tiles = 0;
        while (span.tiles == 0 && ++seq < p.sequences) span.set(p, p.lengths[seq]);
    }
};

template <typename T, int DP, int NT, bool TREE> struct AttentionWarp {
    typedef AttentionShape<T, DP, NT> Shape;
    typedef AttentionCursor<TREE> Cursor;
    static constexpr int ROW = Shape::ROW;
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int KSTEPS = F32 ? DP / 8 : DP / 16;
    static constexpr int MT = DP / 16;
    // fp32: even within a tile the tensor core's cut-off sums are the largest error.  Scores leave it after so many
    // steps, outputs after every step, and are added in fp32: errors of
    // 3e-7 to 4e-7 instead of 7e-7 to 3e-6 (heads of 64 to 256, 2700 to 131072 tokens; plain fp32 8e-7 to 1e-6), for
    // 2 to 3 % of the time.
    static constexpr int kExactSteps = 2;

    const AttentionParams &p;
    unsigned ring;                           // shared-memory address of the warp's ring
    int lane;
    uint32_t q[NT][KSTEPS][2];               // the queries as N-side operand
    float o[MT][NT][4];                      // O^T: rows head elements, columns query heads
    float m[NT][2], l[NT][2];                // running maximum (of scale * score * log2 e) and this thread's part of the sum
    int seen_drafts[NT][2];                  // TREE: see drafts_seen()

    __device__ __forceinline__ AttentionWarp(const AttentionParams &params, unsigned ring_addr, int lane_)
        : p(params), ring(ring_addr), lane(lane_) {}

    __device__ __forceinline__ static unsigned swizzled(int row, int chunk) { return unsigned(row * ROW + ((chunk ^ (row & 7)) << 4)); }

    // page number and row in the page of token `tile * 16 + lane % 16`; -1 where the token is not visible or has no page
    __device__ __forceinline__ int32_t look_up(const Cursor &c, int32_t &row) const
    {
        const int32_t t = (c.span.first_tile + c.tile) * kAttnTok + (lane & 15);
        if (t < c.span.begin || t >= c.span.end) { row = 0; return -1; }
        const uint32_t j = p.page.div(uint32_t(t));
        row = t - int32_t(j * p.page.d);
        const int32_t page = p.table[c.seq * p.table_n + int64_t(j) * p.table_j];
        if (rare(page < 0 || page >= p.pages)) {
            if (p.flags && c.span.needs_page(t)) atomicOr(p.flags, int(BTC_FLAG_BAD_PAGE));
            return -1;
        }
        return page;
    }

    // Which chunks of 16 bytes of which rows this lane copies: a copy instruction of the warp covers STEP rows
    // (a part of one where a row has more than 32 chunks; rows of 24 chunks leave 8 lanes idle).
    static constexpr int CHUNKS = ROW / 16, PER = 16 / int(sizeof(T));
    static constexpr int STEP = CHUNKS >= 32 ? 1 : 32 / CHUNKS, COLS = CHUNKS >= 32 ? CHUNKS / 32 : 1;
    static_assert(CHUNKS % 32 == 0 || CHUNKS < 32, "whole copy instructions");
    __device__ __forceinline__ int my_sub() const { return STEP == 1 ? 0 : lane / CHUNKS; }
    __device__ __forceinline__ int my_chunk() const { return STEP == 1 ? lane : lane % CHUNKS; }
    __device__ __forceinline__ bool idle() const { return 32 % CHUNKS != 0 && CHUNKS < 32 && lane >= STEP * CHUNKS; }
    __device__ __forceinline__ static int chunk_bytes(int chunk, int dim)
    {
        const int left = (dim - chunk * PER) * int(sizeof(T));
        return left < 0 ? 0 : (left < 16 ? left : 16);
    }

    // start the copies of a tile whose 16 rows are all there, the first and the last 8 in one page each: an address step
    // and a copy per row
    __device__ __forceinline__ void copy_whole(unsigned dst, const T *src, const T *src8, int64_t s_slot, int dim) const
    {
        const int sub = my_sub();
#pragma unroll
        for (int c0 = 0; c0 < COLS; ++c0) {
            const int chunk = my_chunk() + 32 * c0, bytes = chunk_bytes(chunk, dim);
            const int64_t mine = sub * s_slot + (bytes ? chunk * PER : 0);
            const T *at = src + mine;
            const unsigned to = dst + sub * ROW + ((chunk ^ sub) << 4);       // = swizzled(sub, chunk): rows r0 + sub only flip bits 4 to 6
            if (!idle()) {
#pragma unroll
                for (int r0 = 0; r0 < kAttnTok; r0 += STEP) {
                    if (r0 == 8) at = src8 + mine;
                    cp_async_part((to ^ ((r0 & 7) << 4)) + r0 * ROW, at, bytes);
                    at += STEP * s_slot;
                }
            }
        }
    }
    // start the copies of any tile; rows without a token (bit clear in `mask`) are zeros
    __device__ __forceinline__ void copy_rows(unsigned dst, const T *base, int64_t s_page, int64_t s_slot, int64_t s_d,
                                              int dim, bool vec, int32_t page, int32_t row, uint32_t mask) const
    {
        const int64_t offset = page < 0 ? 0 : page * s_page + row * s_slot;      // of row lane % 16
        if (vec) {
            const int sub = my_sub();
#pragma unroll 4
            for (int r0 = 0; r0 < kAttnTok; r0 += STEP) {
                const int r = r0 + (idle() ? 0 : sub);
                const T *src = base + __shfl_sync(0xffffffffu, offset, r);
                const bool there = (mask >> r) & 1;
#pragma unroll
                for (int c0 = 0; c0 < COLS; ++c0) {
                    const int chunk = my_chunk() + 32 * c0;
                    const int bytes = there ? chunk_bytes(chunk, dim) : 0;
                    if (!idle()) cp_async_part(dst + swizzled(r, chunk), bytes ? src + chunk * PER : base, bytes);
                }
            }
        } else {
#pragma unroll 1
            for (int r = 0; r < kAttnTok; ++r) {
                const T *src = base + __shfl_sync(0xffffffffu, offset, r);
                const bool there = (mask >> r) & 1;
#pragma unroll 1
                for (int d = lane; d < DP; d += 32) {
                    T x = from_f32<T>(0.f);
                    if (there && d < dim) x = src[d * s_d];
                    const unsigned at = dst + swizzled(r, d / PER) + unsigned(d % PER) * unsigned(sizeof(T));
                    if constexpr (F32) asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
                    else asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(*reinterpret_cast<const unsigned short *>(&x)) : "memory");
                }
            }
        }
    }
    __device__ __forceinline__ void copy_tile(const Cursor &c, int stage, int32_t page, int32_t row, uint32_t mask) const
    {
        const unsigned dst = ring + unsigned(stage) * Shape::STAGE;
        const T *k = static_cast<const T *>(p.k) + c.key_head * p.k_head, *v = static_cast<const T *>(p.v) + c.key_head * p.v_head;
        if (p.whole_tiles && mask == 0xffffu) {
            // lanes 0 and 8 have the first row of each half; where pages hold a multiple of 16 tokens both are in one page
            const int64_t row0 = __shfl_sync(0xffffffffu, row, 0);
            int32_t page0 = page, page8 = page;
            int64_t row8 = row0 + 8;
            if (p.whole_tiles == 8) {
                page0 = __shfl_sync(0xffffffffu, page, 0);
                page8 = __shfl_sync(0xffffffffu, page, 8);
                row8 = __shfl_sync(0xffffffffu, row, 8);
            }
            copy_whole(dst, k + page0 * p.k_page + row0 * p.k_slot, k + page8 * p.k_page + row8 * p.k_slot, p.k_slot, p.dim_k);
            copy_whole(dst + kAttnTok * ROW, v + page0 * p.v_page + row0 * p.v_slot, v + page8 * p.v_page + row8 * p.v_slot, p.v_slot, p.dim_v);
            return;
        }
        copy_rows(dst, k, p.k_page, p.k_slot, p.k_d, p.dim_k, p.vec_k, page, row, mask);
        copy_rows(dst + kAttnTok * ROW, v, p.v_page, p.v_slot, p.v_d, p.dim_v, p.vec_v, page, row, mask);
    }

    // the item's first row in its key head's group, and how many rows it has
    __device__ __forceinline__ int first_row(const Cursor &c, int &count) const
    {
        count = min(8 * NT, p.group - c.block * 8 * NT);
        return c.block * 8 * NT;
    }
    __device__ __forceinline__ static const T *query(const AttentionParams &p, const Cursor &c, int row)
    {
        int32_t draft;
        const int64_t head = attention_row<TREE>(p, c.key_head, row, draft);
        return static_cast<const T *>(p.q) + c.seq * p.q_n + head * p.q_h + (TREE ? draft * p.q_t : 0);
    }
    // TREE: how many drafts the row sees (0: it holds none, and sees nothing)
    __device__ __forceinline__ int drafts_seen(const Cursor &c, int row) const
    {
        int32_t draft;
        attention_row<TREE>(p, c.key_head, row, draft);
        const int32_t *m = p.masks + c.seq * p.m_n + draft * p.m_t;
        int n = 0;
        for (int w = 0; w < p.words; ++w) {
            uint32_t x = uint32_t(m[w * p.m_w]);
            if (p.drafts - 32 * w < 32) x &= (1u << (p.drafts - 32 * w)) - 1u;
            n += __popc(x);
        }
        return n;
    }
    // TREE: does the row, which sees `count` drafts, see token t of the sequence?
    __device__ __forceinline__ bool sees(const Cursor &c, int row, int count, int t) const
    {
        const int d = t - c.span.cached;
        if (d < 0) return p.window == 0 || t >= c.span.cached + count - p.window;
        int32_t draft;
        attention_row<TREE>(p, c.key_head, row, draft);
        return (uint32_t(p.masks[c.seq * p.m_n + draft * p.m_t + (d >> 5) * p.m_w]) >> (d & 31)) & 1u;
    }

    __device__ __forceinline__ void begin_item(const Cursor &c)
    {
        int count;
        const int h0 = first_row(c, count);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int h = nt * 8 + lane / 4;
            const T *src = query(p, c, h0 + (h < count ? h : 0));
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t x = 0;
                    if constexpr (F32) {
                        const int d = ks * 8 + half * 4 + lane % 4;
                        if (h < count && d < p.dim_k) x = __float_as_uint(src[d * p.q_d]);
                    } else {
                        const int d = ks * 16 + half * 8 + 2 * (lane % 4);
                        if (h < count && d < p.dim_k) {
                            if (p.vec_q) {
                                x = *reinterpret_cast<const uint32_t *>(src + d);
                            } else {
                                x = *reinterpret_cast<const unsigned short *>(src + d * p.q_d);
                                if (d + 1 < p.dim_k) x |= uint32_t(*reinterpret_cast<const unsigned short *>(src + (d + 1) * p.q_d)) << 16;
                            }
                        }
                    }
                    q[nt][ks][half] = x;
                }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[nt][j] = -INFINITY;
                l[nt][j] = 0.f;
                const int column = nt * 8 + 2 * (lane & 3) + j;
                if constexpr (TREE) seen_drafts[nt][j] = column < count ? drafts_seen(c, h0 + column) : 0;
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[mt][nt][j] = 0.f;
        }
    }

    // The scores of a tile by plain fp32 products.  A split infinity is inf + NaN, so a tile with a score that is not
    // a number is computed again here, where infinite keys give infinite scores.
    __device__ __noinline__ static void plain_scores(const AttentionParams &p, const Cursor &c, int h0, int count,
                                                     unsigned keys, int lane, float (*s)[4])
    {
        for (int nt = 0; nt < NT; ++nt)
            for (int j = 0; j < 2; ++j) {
                const int h = nt * 8 + 2 * (lane & 3) + j;
                const T *src = query(p, c, h0 + (h < count ? h : 0));
                float x = 0.f, y = 0.f;
                for (int d = 0; d < p.dim_k; ++d) {
                    float k0, k1;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(k0) : "r"(keys + swizzled(lane >> 2, d >> 2) + unsigned(d & 3) * 4u) : "memory");
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(k1) : "r"(keys + swizzled((lane >> 2) + 8, d >> 2) + unsigned(d & 3) * 4u) : "memory");
                    const float qd = to_f32(src[d * p.q_d]);
                    x = fmaf(k0, qd, x);
                    y = fmaf(k1, qd, y);
                }
                s[nt][j] = x;
                s[nt][j + 2] = y;
            }
    }

    // Does a tile of values hold an infinity or NaN?  (A product with a probability of zero would be NaN: in a tree such a
    // token may be invisible to this row and visible to the next.)
    __device__ __forceinline__ bool odd_values(unsigned values) const
    {
        bool odd = false;
#pragma unroll 4
        for (int i = lane; i < kAttnTok * ROW / 16; i += 32) {
            uint32_t x[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(values + 16u * unsigned(i)) : "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (F32) {
                    odd |= (x[j] & 0x7f800000u) == 0x7f800000u;
                } else {
                    constexpr uint32_t e = sizeof(T) == 2 && std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
                    odd |= (x[j] & e) == e || ((x[j] >> 16) & e) == e;
                }
            }
        }
        return __any_sync(0xffffffffu, odd);
    }
    // O += V^T P with plain fp32 products, without the tokens whose probability is zero
    __device__ __forceinline__ void plain_values(unsigned values, const float (&s)[NT][4])
    {
#pragma unroll 1
        for (int tk = 0; tk < kAttnTok; ++tk) {
            float pr[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int src = (tk & 7) * 4 + (lane & 3);
                    const float a = __shfl_sync(0xffffffffu, s[nt][j], src), b = __shfl_sync(0xffffffffu, s[nt][j + 2], src);
                    pr[nt][j] = tk < 8 ? a : b;
                }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int d = element(mt, half);
                    const unsigned at = values + swizzled(tk, d / PER) + unsigned(d % PER) * unsigned(sizeof(T));
                    float x;
                    if constexpr (F32) {
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
                    } else {
                        unsigned short h;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at) : "memory");
                        x = to_f32(*reinterpret_cast<const T *>(&h));
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (pr[nt][j] != 0.f) o[mt][nt][2 * half + j] = fmaf(pr[nt][j], x, o[mt][nt][2 * half + j]);
                }
        }
    }

    // one tile; bit r of `seen`: token r counts
    __device__ __forceinline__ void tile(const Cursor &cur, int stage, uint32_t seen)
    {
        const unsigned ks_base = ring + unsigned(stage) * Shape::STAGE, vs_base = ks_base + kAttnTok * ROW;
        // the products of even and odd steps (fp32: the three kinds of partial products) go to accumulators of their
        // own: one chain of dependent MMAs would cost more time than everything else in a tile
        constexpr int CHAINS = F32 ? 3 : 2;
        float s[NT][4], part[NT][CHAINS][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[nt][j] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < CHAINS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) part[nt][i][j] = 0.f;
        {
            // the next pair of chunks flips address bits 5 and 6, the next 128 bytes of the row are a step
            const unsigned at = ks_base + swizzled(((lane >> 3) & 1) * 8 + (lane & 7), lane >> 4);
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                uint32_t a[4];
                ldsm4(a, (at ^ ((ks & 3) << 5)) + (ks >> 2) * 128);
                if constexpr (F32) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) split_tf32(a[j], hi[j], lo[j]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma8_split(part[nt][0], part[nt][1], part[nt][2], hi, lo, q[nt][ks][0], q[nt][ks][1]);
                    if (ks % kExactSteps == kExactSteps - 1)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                s[nt][j] += part[nt][2][j];
                                part[nt][2][j] = 0.f;
                            }
                } else {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16(part[nt][ks & 1], a, q[nt][ks][0], q[nt][ks][1], T());
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[nt][j] += part[nt][1][j] + part[nt][0][j];
                }
        }
        if constexpr (F32) {
            bool odd = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= s[nt][j] != s[nt][j];
            if (rare(__any_sync(0xffffffffu, odd))) {
                int count;
                const int h0 = first_row(cur, count);
                float again[NT][4];
                plain_scores(p, cur, h0, count, ks_base, lane, again);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[nt][j] = again[nt][j];
            }
        }
        const bool ok0 = (seen >> (lane >> 2)) & 1, ok1 = (seen >> ((lane >> 2) + 8)) & 1;
        float alpha[NT][2];
        bool moved = false;
        // TREE: tiles of tokens that every draft sees need no look at the masks
        const int token0 = (cur.span.first_tile + cur.tile) * kAttnTok;
        const bool masked = TREE && (token0 + kAttnTok > cur.span.cached || (p.window > 0 && token0 < cur.span.cached + p.drafts - p.window));
        int rows_here = 0, row0 = 0;
        if constexpr (TREE) row0 = first_row(cur, rows_here);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float &s0 = s[nt][j], &s1 = s[nt][j + 2];
                s0 = ok0 ? s0 * p.scale_log2 : -INFINITY;
                s1 = ok1 ? s1 * p.scale_log2 : -INFINITY;
                if (TREE && masked) {
                    const int column = nt * 8 + 2 * (lane & 3) + j;
                    if (column < rows_here && seen_drafts[nt][j] > 0) {
                        if (ok0 && !sees(cur, row0 + column, seen_drafts[nt][j], token0 + (lane >> 2))) s0 = -INFINITY;
                        if (ok1 && !sees(cur, row0 + column, seen_drafts[nt][j], token0 + (lane >> 2) + 8)) s1 = -INFINITY;
                    }
                }
                float top = fmaxf(s0, s1);
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                top = fmaxf(top, m[nt][j]);
                // nothing seen yet (or every score is -inf): subtract 0, the probabilities are exp2(-inf) = 0
                const float base = top == -INFINITY ? 0.f : top;
                alpha[nt][j] = m[nt][j] == top ? 1.f : exp2f(m[nt][j] - top);
                moved |= alpha[nt][j] != 1.f;
                m[nt][j] = top;
                s0 = exp2f(s0 - base) * AttentionBias<T>::factor;
                s1 = exp2f(s1 - base) * AttentionBias<T>::factor;
                l[nt][j] = l[nt][j] * alpha[nt][j] + (s0 + s1);
            }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[mt][nt][j] *= alpha[nt][j & 1];
        }
        if (TREE && masked && rare(odd_values(vs_base))) {
            plain_values(vs_base, s);
            return;
        }
        if constexpr (F32) {
            // P (rows tokens, columns heads) -> N-side operand: token lane % 4 (+ 4, + 8, + 12) of head lane / 4
            uint32_t b[NT][2][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int src = (half * 4 + (lane & 3)) * 4 + (lane >> 3);
                        const float x = __shfl_sync(0xffffffffu, s[nt][2 * ks], src), y = __shfl_sync(0xffffffffu, s[nt][2 * ks + 1], src);
                        b[nt][ks][half] = __float_as_uint((lane >> 2) & 1 ? y : x);
                    }
            // The rows of the product may be any order of the head's elements.  They are taken so that a lane's four elements
            // of one token in two row tiles are neighbours (element()): one 16-byte read for them
#pragma unroll
            for (int pair = 0; pair < MT / 2; ++pair)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    uint32_t hi[2][4], lo[2][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t x[4];
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                                     : "r"(vs_base + swizzled(ks * 8 + j * 4 + (lane & 3), lane >> 2) + pair * 128) : "memory");
#pragma unroll
                        for (int e = 0; e < 4; ++e) split_tf32(x[e], hi[e >> 1][2 * j + (e & 1)], lo[e >> 1][2 * j + (e & 1)]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float f[4] = {0.f, 0.f, 0.f, 0.f};
                            mma8_split(f, f, f, hi[i], lo[i], b[nt][ks][0], b[nt][ks][1]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[2 * pair + i][nt][j] += f[j];
                        }
                }
        } else {
            uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float x = s[nt][2 * half], y = s[nt][2 * half + 1];
                    const float xh = to_f32(from_f32<T>(x)), yh = to_f32(from_f32<T>(y));
                    hi[nt][half] = transpose8x8(pack2(xh, yh, T()));
                    lo[nt][half] = transpose8x8(pack2(x - xh, y - yh, T()));
                }
            const unsigned at = vs_base + swizzled((lane >> 4) * 8 + (lane & 7), (lane >> 3) & 1);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                uint32_t a[4];
                ldsm4_trans(a, (at ^ ((mt & 3) << 5)) + (mt >> 2) * 128);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float f[4] = {0.f, 0.f, 0.f, 0.f};
                    mma16(f, a, lo[nt][0], lo[nt][1], T());
                    mma16(f, a, hi[nt][0], hi[nt][1], T());
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[mt][nt][j] += f[j];
                }
            }
        }
    }

    // which element of the head the accumulator row (lane / 4, + 8 when half) of row tile mt is
    __device__ __forceinline__ int element(int mt, int half) const
    {
        return F32 ? (mt >> 1) * 32 + (lane >> 2) * 4 + (mt & 1) * 2 + half : mt * 16 + half * 8 + (lane >> 2);
    }
    __device__ __forceinline__ void finish_sums()
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float &x = l[nt][j];
                x += __shfl_xor_sync(0xffffffffu, x, 4);
                x += __shfl_xor_sync(0xffffffffu, x, 8);
                x += __shfl_xor_sync(0xffffffffu, x, 16);
                // a row without a draft: as if every score were -inf
                if (TREE && seen_drafts[nt][j] == 0) { x = 0.f; m[nt][j] = -INFINITY; }
            }
    }
    __device__ __forceinline__ void write_out(const Cursor &c) const
    {
        int count;
        const int h0 = first_row(c, count);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = nt * 8 + 2 * (lane & 3) + j;
                if (h >= count) continue;
                int32_t draft;
                const int head = attention_row<TREE>(p, c.key_head, h0 + h, draft);
                const bool nothing = l[nt][j] == 0.f;          // every score is -inf: zeros, whatever V holds (0 * inf is NaN)
                const float inv = 1.f / l[nt][j];
                T *dst = static_cast<T *>(p.o) + c.seq * p.o_n + int64_t(head) * p.o_h + (TREE ? draft * p.o_t : 0);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int d = element(mt, half);
                        if (d < p.dim_v) dst[d * p.o_d] = from_f32<T>(nothing ? 0.f : o[mt][nt][2 * half + j] * inv);
                    }
                if (p.lse && lane < 4)
                    p.lse[(TREE ? int64_t(c.seq) * p.drafts + draft : int64_t(c.seq)) * p.heads + head] = nothing ? -INFINITY
                        : (m[nt][j] + (log2f(l[nt][j]) - AttentionBias<T>::value)) * 0.6931471805599453f;
            }
    }
    // an unfinished item: output, maxima and sums to shared memory
    __device__ __forceinline__ void deposit(float *out, float *stats) const
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = nt * 8 + 2 * (lane & 3) + j;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        out[h * DP + element(mt, half)] = o[mt][nt][2 * half + j];
                if (lane < 4) {
                    stats[h] = m[nt][j];
                    stats[8 * NT + h] = l[nt][j];
                }
            }
    }
};

// what a part with maximum m counts in a whole with maximum top >= m (a part that saw nothing has m = -inf and o = l = 0)
__device__ __forceinline__ float join_weight(float m, float top)
{
    const float w = exp2f(m - top);          // NaN where both are infinite
    return m == top ? 1.f : w;
}

// elements d..d+3 of head h of an item (8 NT = `per` heads) from its joined sums
template <typename T, bool TREE>
__device__ __forceinline__ void write_joined(const AttentionParams &p, int32_t item, int per, int h, int d, const float4 &o, float m, float l)
{
    const int head_blocks = p.key_heads * p.blocks;
    const int seq = item / head_blocks, hb = item - seq * head_blocks;
    const int kh = hb / p.blocks, in_group = (hb - kh * p.blocks) * per + h;
    if (in_group >= p.group) return;
    int32_t draft;
    const int head = attention_row<TREE>(p, kh, in_group, draft);
    const bool nothing = l == 0.f;             // as in write_out
    const float inv = 1.f / l;
    T *dst = static_cast<T *>(p.o) + seq * p.o_n + int64_t(head) * p.o_h + (TREE ? draft * p.o_t : 0);
    const float v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (d + j < p.dim_v) dst[(d + j) * p.o_d] = from_f32<T>(nothing ? 0.f : v[j] * inv);
    if (d == 0 && p.lse)
        p.lse[(TREE ? int64_t(seq) * p.drafts + draft : int64_t(seq)) * p.heads + head] = nothing ? -INFINITY : (m + (log2f(l) - AttentionBias<T>::value)) * 0.6931471805599453f;
}

template <typename T, int DP, int NT, bool TREE>
__global__ void __launch_bounds__(AttentionShape<T, DP, NT>::WARPS * 32, 1)
paged_attention_kernel(const __grid_constant__ AttentionParams p)
{
    typedef AttentionShape<T, DP, NT> Shape;
    constexpr int W = Shape::WARPS, THREADS = W * 32, STAGES = Shape::STAGES, H = 8 * NT;
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ float stats[2 * W][2 * H];
    __shared__ int32_t dep_item[2 * W];
    __shared__ int32_t first_item, last_item;                  // items of the CTA's range that it does not hold whole; -1: none
    int64_t *scan = reinterpret_cast<int64_t *>(smem + W * Shape::RING);     // until the ranges are known
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head_blocks = p.key_heads * p.blocks;

    early_begin();

    // tiles of all sequences: thread i sums sequences [i * per, (i + 1) * per), then a prefix sum over the threads
    const int per = (p.sequences + THREADS - 1) / THREADS;
    {
        int64_t mine = 0;                                       // tiles * 2^24 + sequences that have any
        for (int i = 0; i < per; ++i) {
            const int s = tid * per + i;
            if (s >= p.sequences) break;
            const int32_t length = p.lengths[s];
            AttentionSpan<TREE> span;
            span.set(p, length);
            mine += (int64_t(span.tiles) << 24) + (span.tiles > 0 ? 1 : 0);
            if (blockIdx.x == 0 && p.flags && rare(AttentionSpan<TREE>::bad(p, length))) atomicOr(p.flags, int(BTC_FLAG_BAD_LENGTH));
        }
        int64_t x = mine;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, k);
            if (lane >= k) x += y;
        }
        scan[tid + 1] = x;
        if (tid == 0) { scan[0] = 0; first_item = last_item = -1; }
        if (tid < 2 * W) dep_item[tid] = -1;
        __syncthreads();
        int64_t before = 0;
        for (int w = 0; w < warp; ++w) before += scan[(w + 1) * 32];
        __syncthreads();
        scan[tid + 1] = x + before;
        __syncthreads();
    }
    // equal shares of the list, at least one unit per warp of the CTAs that take part
    auto units = [&](int i) { return ((scan[i] >> 24) + (scan[i] & 0xffffff) * kAttnItemTiles) * head_blocks; };
    const int64_t total = units(THREADS);
    int64_t ctas = (total + W - 1) / W;
    if (ctas > gridDim.x) ctas = gridDim.x;
    // Lanes 0, 1 and 2 look up the places where the warp's share begins and ends and where the CTA's ends.
    AttentionCursor<TREE> cur;
    int64_t n = 0;                                              // tiles of this warp
    bool closes = false;                                        // its last tile is the CTA's last
    if (blockIdx.x < ctas) {
        const int64_t each = divide(total, int32_t(ctas)), more = total - each * ctas;
        const int64_t cta_lo = each * blockIdx.x + min(int64_t(blockIdx.x), more), in_cta = each + (int64_t(blockIdx.x) < more ? 1 : 0);
        const int64_t we = in_cta / W, wm = in_cta - we * W;
        const int64_t lo = cta_lo + we * warp + min(int64_t(warp), wm);
        const int64_t unit = lane == 1 ? lo + we + (warp < wm ? 1 : 0) : (lane == 2 ? cta_lo + in_cta : lo);
        cur.seq = p.sequences;
        cur.hb = cur.tile = 0;
        cur.span.begin = cur.span.end = cur.span.first_tile = cur.span.tiles = cur.span.cached = 0;
        int64_t tiles_before = (scan[THREADS] >> 24) * head_blocks;
        if (unit < total) {
            int a = 0, b = THREADS;                             // units(a) <= unit < units(b)
            while (b - a > 1) {
                const int c = (a + b) / 2;
                if (units(c) <= unit) a = c; else b = c;
            }
            int64_t at = unit - units(a);
            tiles_before = (scan[a] >> 24) * head_blocks;
            cur.seq = a * per;
            cur.span.set(p, p.lengths[cur.seq]);
            // a sequence's units: kAttnItemTiles and then its tiles, for each key head
            while (cur.seq + 1 < p.sequences) {
                const int64_t here = cur.span.tiles > 0 ? int64_t(cur.span.tiles + kAttnItemTiles) * head_blocks : 0;
                if (at < here) break;
                at -= here;
                tiles_before += int64_t(cur.span.tiles) * head_blocks;
                cur.span.set(p, p.lengths[++cur.seq]);
            }
            const int32_t item_units = cur.span.tiles + kAttnItemTiles;
            cur.hb = int32_t(divide(at, item_units));
            cur.tile = max(0, int32_t(at - int64_t(cur.hb) * item_units) - kAttnItemTiles);
            tiles_before += int64_t(cur.hb) * cur.span.tiles + cur.tile;
        }
        const int64_t from = __shfl_sync(0xffffffffu, tiles_before, 0), to = __shfl_sync(0xffffffffu, tiles_before, 1);
        n = to - from;
        closes = to == __shfl_sync(0xffffffffu, tiles_before, 2);
        cur.seq = __shfl_sync(0xffffffffu, cur.seq, 0);
        cur.hb = __shfl_sync(0xffffffffu, cur.hb, 0);
        cur.tile = __shfl_sync(0xffffffffu, cur.tile, 0);
        cur.span.begin = __shfl_sync(0xffffffffu, cur.span.begin, 0);
        cur.span.end = __shfl_sync(0xffffffffu, cur.span.end, 0);
        cur.span.first_tile = __shfl_sync(0xffffffffu, cur.span.first_tile, 0);
        cur.span.tiles = __shfl_sync(0xffffffffu, cur.span.tiles, 0);
        if constexpr (TREE) cur.span.cached = __shfl_sync(0xffffffffu, cur.span.cached, 0);
        cur.key_head = cur.hb / p.blocks;
        cur.block = cur.hb - cur.key_head * p.blocks;
        // does the CTA's share begin inside an item?  (Then its first unit is a tile, and warp 0 has it.)
        if (warp == 0 && cur.tile != 0 && lane == 0) first_item = cur.seq * head_blocks + cur.hb;
    }
    const unsigned ring = static_cast<unsigned>(__cvta_generic_to_shared(smem)) + unsigned(warp) * Shape::RING;
    float *deposit_first = reinterpret_cast<float *>(smem + W * Shape::RING) + warp * (Shape::DEPOSIT / 4);
    float *deposit_last = reinterpret_cast<float *>(smem + warp * Shape::RING);

    __syncthreads();

    if (n > 0) {
        AttentionWarp<T, DP, NT, TREE> w(p, ring, lane);
        AttentionCursor<TREE> ahead = cur;                            // the tile whose page numbers are in `page`, `row`
        int64_t issued = 0;
        int32_t row, page = w.look_up(ahead, row);
        // tokens that count: seen[k] belongs to the tile k steps ahead of the one being consumed
        uint32_t seen[STAGES];
#pragma unroll
        for (int k = 0; k < STAGES; ++k) seen[k] = 0;
        bool began_here = cur.tile == 0;                        // the current item's first tile is in this warp's range
        w.begin_item(cur);
        int stage = 0, into = 0;
        // one step: start the copies of tile i + STAGES - 1, consume tile i (the first STAGES - 1 steps only copy)
        for (int64_t i = 1 - STAGES; i < n; ++i) {
            cp_async_wait_group<STAGES - 2>();
            __syncwarp();                                       // every lane's copies have landed, the oldest stage is free
#pragma unroll
            for (int k = 0; k + 1 < STAGES; ++k) seen[k] = seen[k + 1];
            seen[STAGES - 1] = 0;
            if (issued < n) {
                seen[STAGES - 1] = __ballot_sync(0xffffffffu, page >= 0) & 0xffffu;
                w.copy_tile(ahead, into, page, row, seen[STAGES - 1]);
                if (++into == STAGES) into = 0;
                if (++issued < n) {
                    ahead.next(p);
                    page = w.look_up(ahead, row);
                }
            }
            cp_async_commit();
            if (i < 0) continue;
            w.tile(cur, stage, seen[0]);
            if (++stage == STAGES) stage = 0;
            const bool item_ends = cur.tile + 1 == cur.span.tiles;
            if (item_ends || i + 1 == n) {
                w.finish_sums();
                if (item_ends && began_here) {
                    w.write_out(cur);
                } else {
                    // an item that began in an earlier range goes to its own place; one that began here and is cut
                    // off is the last, so that it can have the ring, which nothing uses any more
                    const int slot = began_here ? 1 : 0;
                    if (slot) cp_async_wait_group<0>();
                    __syncwarp();
                    w.deposit(slot ? deposit_last : deposit_first, stats[2 * warp + slot]);
                    if (lane == 0) {
                        dep_item[2 * warp + slot] = cur.seq * head_blocks + cur.hb;
                        if (i + 1 == n && closes && !item_ends) last_item = cur.seq * head_blocks + cur.hb;
                    }
                }
                if (i + 1 < n) {
                    cur.next(p);
                    w.begin_item(cur);
                    began_here = true;
                }
            } else {
                ++cur.tile;
            }
        }
        cp_async_wait_group<0>();
    }
    __syncthreads();

    if (tid < 2) p.partial_item[2 * blockIdx.x + tid] = tid == 0 ? first_item : (last_item == first_item ? -1 : last_item);
    if (blockIdx.x < ctas) {
        // Join what the warps left, a warp to a head.  First a lane to a deposit (those of an item are neighbours): its
        // weight against the item's largest maximum; then a lane to four elements.
        for (int h = warp; h < H; h += W) {
            const int at = lane < 2 * W ? lane : 0;
            const int32_t item = lane < 2 * W ? dep_item[at] : -1;
            const bool mine = item >= 0;
            const float m = mine ? stats[at][h] : -INFINITY, l = mine ? stats[at][H + h] : 0.f;
            const uint32_t same = __match_any_sync(0xffffffffu, mine ? item : -1 - lane);
            float top = m;
#pragma unroll
            for (int j = 0; j < 2 * W; ++j) {
                const float x = __shfl_sync(0xffffffffu, m, j);
                if ((same >> j) & 1) top = fmaxf(top, x);
            }
            const float share = mine ? join_weight(m, top) : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 2 * W; ++j) {
                const float x = __shfl_sync(0xffffffffu, l * share, j);
                if ((same >> j) & 1) sum += x;
            }
            const uint32_t present = __ballot_sync(0xffffffffu, mine);
            uint32_t ends = __ballot_sync(0xffffffffu, mine && (same >> lane) == 1);    // the last deposit of its item
            int begin = 0;
            while (ends) {
                const int last = __ffs(int(ends)) - 1;
                ends &= ends - 1;
                const int32_t this_item = __shfl_sync(0xffffffffu, item, last);
                const float this_top = __shfl_sync(0xffffffffu, top, last), this_sum = __shfl_sync(0xffffffffu, sum, last);
#pragma unroll
                for (int q0 = 0; q0 < DP / 4; q0 += 32) {
                    const int quad = q0 + lane;
                    const bool here = quad < DP / 4;
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int i = begin; i <= last; ++i) {
                        const float weight = __shfl_sync(0xffffffffu, share, i);
                        if (((present >> i) & 1) && here) {
                            const unsigned char *src = (i & 1) ? smem + (i >> 1) * Shape::RING : smem + W * Shape::RING + (i >> 1) * Shape::DEPOSIT;
                            const float4 x = reinterpret_cast<const float4 *>(src)[h * (DP / 4) + quad];
                            o.x = fmaf(x.x, weight, o.x); o.y = fmaf(x.y, weight, o.y); o.z = fmaf(x.z, weight, o.z); o.w = fmaf(x.w, weight, o.w);
                        }
                    }
                    if (!here) continue;
                    if (this_item == first_item || this_item == last_item) {
                        float *out = p.partial + (2 * int64_t(blockIdx.x) + (this_item == first_item ? 0 : 1)) * (H * DP + 2 * H);
                        reinterpret_cast<float4 *>(out)[h * (DP / 4) + quad] = o;
                        if (quad == 0) { out[H * DP + h] = this_top; out[H * DP + H + h] = this_sum; }
                    } else {
                        write_joined<T, TREE>(p, this_item, H, h, 4 * quad, o, this_top, this_sum);
                    }
                }
                begin = last + 1;
            }
        }
    }
    if constexpr (TREE)
        if (warp == 0) report_drafts(p, lane);
    // sequences with nothing to see
    for (int s = blockIdx.x; s < p.sequences; s += gridDim.x) {
        AttentionSpan<TREE> span;
        span.set(p, p.lengths[s]);
        if (rare(span.tiles == 0)) {
            const int drafts = TREE ? p.drafts : 1;
            for (int e = tid; e < p.heads * p.dim_v; e += THREADS) {
                const int h = e / p.dim_v, d = e - h * p.dim_v;
                for (int t = 0; t < drafts; ++t)
                    static_cast<T *>(p.o)[s * p.o_n + (TREE ? t * p.o_t : 0) + int64_t(h) * p.o_h + d * p.o_d] = from_f32<T>(0.f);
            }
            if (p.lse)
                for (int h = tid; h < p.heads * drafts; h += THREADS) p.lse[int64_t(s) * p.heads * drafts + h] = -INFINITY;
        }
    }
}

// loads that stay where they are written: ahead of the branches and barriers that come before their use
__device__ __forceinline__ int32_t load_now(const int32_t *p)
{
    int32_t v;
    asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float load_now(const float *p)
{
    float v;
    asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float4 load_now(const float4 *p)
{
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}

// Items that span CTAs: the blocks (c, slice) join the item that begins in CTA c's range and ends in a later one's: CTA
// c's second slot, then the first slots of the CTAs after it while they carry the same item.  A block takes a quarter
// of the heads, a thread four elements of one; the threads beyond the elements split the parts among them, so
// that a long sequence alone (148 parts) is a few rounds of loads.
constexpr int kJoinThreads = 256, kJoinSlices = 4;
template <typename T, int DP, int NT, bool TREE>
__global__ void __launch_bounds__(kJoinThreads) paged_attention_join_kernel(const __grid_constant__ AttentionParams p, int ctas)
{
    constexpr int H = 8 * NT, HEADS = H / kJoinSlices, QUADS = HEADS * DP / 4, SPLIT = kJoinThreads / QUADS, AHEAD = 16 / SPLIT;
    constexpr int64_t slot_floats = H * DP + 2 * H;
    static_assert(QUADS * SPLIT <= kJoinThreads && SPLIT >= 2 && HEADS <= kJoinThreads / 32, "");
    __shared__ int32_t parts;
    __shared__ float tops[HEADS], totals[HEADS];
    __shared__ float4 sums[SPLIT - 1][QUADS];
    const int c = blockIdx.x, h0 = blockIdx.y * HEADS, tid = threadIdx.x, lane = tid & 31;
    early_begin();
    const int32_t item = load_now(p.partial_item + 2 * c + 1);
    if (item < 0) return;
    // Part 0 is CTA c's second slot, part i CTA c + i's first; the first CTA without the item ends it.  How many parts there
    // are is known one round trip to memory later: what the first 32 (a warp's maxima and sums) and the first 16
    // (a thread's elements) hold is loaded before that.
    const int left = ctas - c;
    const float *first = p.partial + 2 * int64_t(c) * slot_floats;
    auto part = [&](int i) { return first + (i == 0 ? slot_floats : 2 * int64_t(i) * slot_floats); };
    const int split = tid / QUADS, quad = tid - split * QUADS, k = quad * 4 / DP, h = h0 + k, d = quad * 4 - k * DP;
    const int32_t other = tid + 1 < left ? load_now(p.partial_item + 2 * (c + tid + 1)) : -1;
    float m0 = -INFINITY, l0 = 0.f;
    if (tid / 32 < HEADS && lane < left) {
        m0 = load_now(part(lane) + H * DP + h0 + tid / 32);
        l0 = load_now(part(lane) + H * DP + H + h0 + tid / 32);
    }
    float4 ahead[AHEAD];
    float ahead_m[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int i = split + j * SPLIT;
        ahead[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        ahead_m[j] = -INFINITY;
        if (split < SPLIT && i < left) {
            ahead[j] = load_now(reinterpret_cast<const float4 *>(part(i) + h0 * DP + quad * 4));
            ahead_m[j] = load_now(part(i) + H * DP + h);
        }
    }
    if (tid == 0) parts = left;
    __syncthreads();
    if (tid + 1 < left && other != item) atomicMin(&parts, tid + 1);
    if (rare(left > kJoinThreads))
        for (int i = tid + 1 + kJoinThreads; i < left; i += kJoinThreads)
            if (p.partial_item[2 * (c + i)] != item) atomicMin(&parts, i);
    __syncthreads();
    const int n = parts;
    // a warp takes a head's maxima and sums
    if (tid / 32 < HEADS) {
        const int at = H * DP + h0 + tid / 32;
        float top = lane < n ? m0 : -INFINITY;
        if (rare(n > 32)) {
#pragma unroll 1
            for (int i = lane + 32; i < n; i += 32) top = fmaxf(top, part(i)[at]);
        }
#pragma unroll
        for (int j = 1; j < 32; j <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, j));
        float l = lane < n ? l0 * join_weight(m0, top) : 0.f;
        if (rare(n > 32)) {
#pragma unroll 1
            for (int i = lane + 32; i < n; i += 32) l = fmaf(part(i)[at + H], join_weight(part(i)[at], top), l);
        }
#pragma unroll
        for (int j = 1; j < 32; j <<= 1) l += __shfl_xor_sync(0xffffffffu, l, j);
        if (lane == 0) { tops[tid / 32] = top; totals[tid / 32] = l; }
    }
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (split < SPLIT) {
        const float top = tops[k];
        auto add = [&](const float4 &x, float m) {
            const float share = join_weight(m, top);
            o.x = fmaf(x.x, share, o.x); o.y = fmaf(x.y, share, o.y); o.z = fmaf(x.z, share, o.z); o.w = fmaf(x.w, share, o.w);
        };
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (split + j * SPLIT < n) add(ahead[j], ahead_m[j]);
        if (rare(n > AHEAD * SPLIT)) {
#pragma unroll 4
            for (int i = split + AHEAD * SPLIT; i < n; i += SPLIT)
                add(*reinterpret_cast<const float4 *>(part(i) + h0 * DP + quad * 4), part(i)[H * DP + h]);
        }
        if (split > 0) sums[split - 1][quad] = o;
    }
    __syncthreads();
    if (split > 0) return;
#pragma unroll
    for (int j = 0; j < SPLIT - 1; ++j) {
        const float4 x = sums[j][quad];
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    write_joined<T, TREE>(p, item, H, h, d, o, tops[k], totals[k]);
}

}  // namespace btc
