// Attention of trees of drafted tokens in 16-bit types on the 5th-generation tensor cores.
//
// The rows of a key head (drafts x query heads that share it) are the M side of both products: S = Q K^T and F = P V, 128 rows and
// 128 tokens at a time, with S, P and F in tensor memory.  One read of the cache serves up to 256 rows.
//
// CTA (one per SM, 12 warps):
//   warps 0-7     softmax of S (tensor memory -> registers -> P in tensor memory, in the place of S), running maximum, sum and output in
//                 registers, F added to it in fp32.  Warps w and w + 4 share 32 rows: one takes the first 64 tokens of a tile and the
//                 first half of the head, the other the second; they exchange the maxima through shared memory.
//   warps 8-10    bring queries, keys and values into the swizzled layouts that the tensor core reads: bulk tensor copies where pages are
//                 whole boxes, 16-byte cp.async elsewhere (tiles with tokens that are not visible)
//   warp 11       issues the products (one lane)
// A step is a tile of tokens for 128 rows; items of more than 128 rows take two steps a tile.  Two sets of S and F alternate: the products
// of one step run while the softmax of the next is computed, and F is added a step later.
//
// Numbers as in the one-token kernels: P is split in two 16-bit parts (both products), S and F are sums over one tile of 128
// tokens, and tiles are added in fp32 outside the tensor core (it cuts its sums off towards zero), so F needs no
// rescaling in tensor memory.
//
// Work: the list of (sequence, key head, block of rows) items in tiles is cut into equal contiguous shares, one per CTA, found on the
// device from the lengths; what a CTA does not hold whole goes to the workspace and a second kernel joins it, in a fixed order.
// Every wait is bounded.  One that gives up ends the CTA, after its copies and products in flight; the rows of the items it had in hand become NaN, so that
// nobody takes an incomplete result for a whole one, and BTC_FLAG_TIMEOUT reports it.
//
// Measured (replayed graphs, heads of 128): 32 requests of 64 to 8192 tokens, 128 rows: 89 us (240 MB), 256 rows: 183 us; 4 x 64 Ki tokens, 32
// rows: 228 us in bf16, 243 in f16 (1.07 GB: 4.7 and 4.4 TB/s), 512 rows 1.06 ms (515 TFLOP/s of the two products), which under the power limit of
// a run of seconds becomes 1.2 ms (455 TFLOP/s).  What bounds it is the chain of a step in the softmax warps, about 4000 cycles (228 us are 111 steps):
// tensor memory to registers 600, the exchange of maxima 290, exponentials 1400 (64 a thread, 16 a cycle on an SM), F 700 to 1000.  A 128 x 128 x 16
// product takes 67 cycles, 24 of them a step.  The softmax warps have 216 registers and spill 224 to 248 bytes a thread; a pass executes 0.6 million
// local accesses of a warp (32 requests), 2 % of what the L1 could.
#pragma once

#include "paged_attention_kernel.cuh"
#include "umma16_common.cuh"

namespace btc {

constexpr int kTreeTok = 128, kTreeRows = 128;
// what beginning and ending an item costs, in tiles (1, 3, 5: 118.5, 104.5, 106.9 us for 32 requests of 64 to 8192 tokens, when a pass took 104)
constexpr int kTreeItemTiles = 3;
constexpr int kTreeThreads = 384;
constexpr int kTreeInfos = 8;                // tiles whose visible tokens are kept: more than the ring can be ahead of the softmax

template <int DP> struct TreeShape {
    static constexpr int PANELS = DP / 64;                       // of 64 elements = 128 bytes, the swizzle's width
    static constexpr int PANEL = kTreeTok * 128;
    static constexpr int TILE = PANELS * PANEL;                  // keys, values or queries of 128 tokens or rows
    static constexpr int SLOTS = DP == 128 ? 5 : 8;
    static constexpr int SMEM = (2 + SLOTS) * TILE;              // queries of up to 256 rows, ring
    static constexpr int64_t PART = int64_t(kTreeRows) * DP + 2 * kTreeRows;      // floats of an unfinished group of rows
};

struct TreeParams {
    AttentionParams a;                       // `group`: rows per key head; `blocks`: of 256 rows
    float *partial;                          // [CTA][2][2 groups][PART]: [element][row], maxima, sums
    int32_t *partial_item;                   // [CTA][2]
    int32_t vec_q, vec_o;                    // 16-byte accesses
    // bulk tensor copies: rows of a box of keys and values (they divide the page), drafts of a box of queries; 0: 16-byte copies
    int32_t box_kv, box_q;
    uint32_t k_page16, k_slot16, v_page16, v_slot16;       // strides of the cache in 16 bytes
    uint32_t poll_limit;                     // polls after which a wait gives up
};
constexpr int32_t kTreeLost = -2;            // in partial_item: a wait of this CTA gave up (-1: no such part)

// visible range of a sequence in tiles of 128 tokens
struct TreeSpan {
    int32_t begin, end, cached, first_tile, tiles;
    __device__ __forceinline__ void set(const AttentionParams &p, int32_t length)
    {
        AttentionSpan<true> s;
        s.set(p, length);
        begin = s.begin; end = s.end; cached = s.cached;
        first_tile = begin / kTreeTok;
        tiles = end > begin ? (end - 1) / kTreeTok + 1 - first_tile : 0;
    }
};

// an item and where this CTA's share of it begins; the same in all threads
struct TreeCursor {
    int32_t seq, hb, tile, key_head, block;
    TreeSpan span;
    __device__ __forceinline__ void next(const AttentionParams &p)
    {
        tile = 0;
        ++hb;
        if (++block < p.blocks) return;
        block = 0;
        if (++key_head < p.key_heads) return;
        hb = key_head = 0;
        span.tiles = 0;
        while (span.tiles == 0 && ++seq < p.sequences) span.set(p, p.lengths[seq]);
    }
    __device__ __forceinline__ int rows(const AttentionParams &p) const { return min(2 * kTreeRows, p.group - block * 2 * kTreeRows); }
};

// The order in which an item's n tiles of keys and values go through the ring: that in which they are used.  Two steps a tile: K0 V0 K1 V1
// ..; one step: scores run two tiles ahead, K0 K1 V0 K2 V1 .. (values that come with their keys hold a place for two steps, and
// the ring is then too short for the memory's latency).
__device__ __forceinline__ int tree_place_k(int j, bool two) { return two ? 2 * j : (j == 0 ? 0 : 2 * j - 1); }
__device__ __forceinline__ int tree_place_v(int j, int n, bool two) { return two || j == n - 1 ? 2 * j + 1 : 2 * j + 2; }
__device__ __forceinline__ int tree_placed(int i, int n, bool two, int &kv)
{
    if (two) { kv = i & 1; return i >> 1; }
    if (i == 0) { kv = 0; return 0; }
    if (i == 2 * n - 1) { kv = 1; return n - 1; }
    kv = (i & 1) ^ 1;
    return kv ? (i - 2) >> 1 : (i + 1) >> 1;
}

struct TreeBarriers {
    uint64_t full[8], empty[8];              // ring of keys and values
    uint64_t q_full[2], q_empty[2];          // two places for 128 rows of queries, taken in turn
    uint64_t s_full[2], p_full[2], f_full[2];
    uint64_t pair[4];                        // the two warps that share rows
    uint64_t drain;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Bit i: does a row see token first + i (of 32)?  `low`: the first cached token it sees; drafts by its mask words.
__device__ __forceinline__ uint32_t tree_visible(int first, int cached, int low, const uint32_t (&mask)[4])
{
    // cached tokens low .. cached - 1
    const int a = max(low - first, 0), b = min(cached - first, 32);
    uint32_t v = b <= a ? 0u : (b >= 32 ? ~0u : (1u << b) - 1u) & (a >= 32 ? 0u : ~0u << a);
    const int d = first - cached;            // draft of bit 0
    if (d > -32 && d < 128) {
        if (d < 0) {
            v |= mask[0] << (-d);
        } else {
            const int w = d >> 5, s = d & 31;
            const uint32_t lo = w == 0 ? mask[0] : w == 1 ? mask[1] : w == 2 ? mask[2] : mask[3];
            const uint32_t hi = w == 0 ? mask[1] : w == 1 ? mask[2] : w == 2 ? mask[3] : 0u;
            v |= __funnelshift_r(lo, hi, s);
        }
    }
    return v;
}

// May rows differ in what they see of the tile that begins at token0?  At its drafts, and at the window's edge, where rows that see
// more drafts begin later.
__device__ __forceinline__ bool tree_differs(const AttentionParams &p, int token0, int cached)
{
    return token0 + kTreeTok > cached || (p.window > 0 && token0 < cached + p.drafts - p.window);
}

// Elements d0 .. d0 + COUNT - 1 of F for one row and tile by plain products over what the row sees.  A value that is infinite or NaN makes
// the tensor core's F NaN in every row, its probability of zero included; where rows differ in what they see such a token may be invisible
// to this row and visible to the next, so those tiles are computed again here when their F is not finite.
template <typename T, int COUNT>
__device__ __noinline__ void tree_plain_values(const AttentionParams &p, const TreeCursor &cur, const uint32_t *seen, int token0, int low,
                                               uint32_t m0, uint32_t m1, uint32_t m2, uint32_t m3, int group_row, float base, int d0, float *out)
{
    const uint32_t mask[4] = {m0, m1, m2, m3};
    int32_t draft;
    const int64_t head = attention_row<true>(p, cur.key_head, group_row, draft);
    const T *q = static_cast<const T *>(p.q) + cur.seq * p.q_n + head * p.q_h + draft * p.q_t;
    for (int i = 0; i < COUNT; ++i) out[i] = 0.f;
    for (int i = 0; i < kTreeTok; ++i) {
        const uint32_t vis = tree_visible(token0 + (i & ~31), cur.span.cached, low, mask) & seen[i >> 5];
        if (!((vis >> (i & 31)) & 1)) continue;
        const uint32_t t = uint32_t(token0 + i), j = p.page.div(t);
        const int64_t page = p.table[cur.seq * p.table_n + int64_t(j) * p.table_j], row = t - j * p.page.d;
        const T *k = static_cast<const T *>(p.k) + cur.key_head * p.k_head + page * p.k_page + row * p.k_slot;
        const T *v = static_cast<const T *>(p.v) + cur.key_head * p.v_head + page * p.v_page + row * p.v_slot;
        float s = 0.f;
        for (int d = 0; d < p.dim_k; ++d) s = fmaf(to_f32(q[d * p.q_d]), to_f32(k[d * p.k_d]), s);
        const float e = ex2(fmaf(s, p.scale_log2, -base)) * AttentionBias<T>::factor;
        if (e == 0.f) continue;
        for (int d = 0; d < COUNT && d0 + d < p.dim_v; ++d) out[d] = fmaf(e, to_f32(v[(d0 + d) * p.v_d]), out[d]);
    }
}

// A wait gave up: NaN into all rows of the items of this CTA's share (256 threads; the joining kernel leaves what it has lost parts of NaN, too).
template <typename T> __device__ __noinline__ void tree_spoil(const TreeParams &tp, TreeCursor cur, int64_t left)
{
    const AttentionParams &p = tp.a;
    while (left > 0) {
        const int rows = cur.rows(p), row0 = cur.block * 2 * kTreeRows;
        for (int e = threadIdx.x; e < rows * p.dim_v; e += 256) {
            const int r = e / p.dim_v, d = e - r * p.dim_v;
            int32_t draft;
            const int64_t head = attention_row<true>(p, cur.key_head, row0 + r, draft);
            static_cast<T *>(p.o)[cur.seq * p.o_n + draft * p.o_t + head * p.o_h + d * p.o_d] = from_f32<T>(NAN);
            if (d == 0 && p.lse) p.lse[(int64_t(cur.seq) * p.drafts + draft) * p.heads + head] = NAN;
        }
        left -= min(int64_t(cur.span.tiles - cur.tile), left);
        cur.next(p);
    }
    if (threadIdx.x == 0) tp.partial_item[2 * blockIdx.x] = tp.partial_item[2 * blockIdx.x + 1] = kTreeLost;
}

// elements d0 .. d0 + N - 1 of an output row
template <typename T, int N>
__device__ __forceinline__ void tree_write(T *dst, int d0, int dim, int64_t stride, bool vec, const float (&o)[N], float scale, bool nothing)
{
    static_assert(N % 8 == 0, "");
#pragma unroll
    for (int d = 0; d < N; d += 8) {
        if (d0 + d >= dim) break;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = nothing ? 0.f : o[d + e] * scale;
        if (vec && d0 + d + 8 <= dim) {
            *reinterpret_cast<uint4 *>(dst + d0 + d) = pack_vector<T, 8>(x);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (d0 + d + e < dim) dst[(d0 + d + e) * stride] = from_f32<T>(x[e]);
        }
    }
}

// WIDE: items may have more than 128 rows; otherwise a thread keeps one output and has room for its scores
template <typename T, int DP, bool WIDE>
__global__ void __launch_bounds__(kTreeThreads, 1) tree_umma_kernel(const __grid_constant__ TreeParams tp, const __grid_constant__ CUtensorMap map_q,
                                                                    const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    typedef TreeShape<DP> Shape;
    constexpr int SLOTS = Shape::SLOTS, TILE = Shape::TILE, PANEL = Shape::PANEL, PANELS = Shape::PANELS;
    const AttentionParams &p = tp.a;
    extern __shared__ __align__(1024) unsigned char raw_smem[];   // (what is static beside it is less than 3 KB)
    __shared__ __align__(8) TreeBarriers bars;
    __shared__ uint32_t tmem_base_word;
    __shared__ int abort_word;
    __shared__ TreeCursor start;
    __shared__ int64_t share;
    __shared__ uint32_t infos[kTreeInfos][4];
    __shared__ float tops[2][2][kTreeRows];                     // [step's parity][half][row]
    __shared__ uint32_t filled[10];                             // 1 + phase of the last copies into a place of the ring (0..7) and of queries (8, 9); 0: none
    volatile int *abort_flag = &abort_word;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int64_t *scan = reinterpret_cast<int64_t *>(raw_smem);      // until the shares are known
    const unsigned smem = unsigned(__cvta_generic_to_shared(raw_smem));
    const unsigned q_at = smem, ring_at = smem + 2 * TILE;
    auto bar = [&](const uint64_t &b) { return unsigned(__cvta_generic_to_shared(&b)); };
    const int head_blocks = p.key_heads * p.blocks;
    // the same answer in all lanes: what follows are instructions of whole warps
    auto wait = [&](unsigned b, unsigned phase) -> bool { return __all_sync(0xffffffffu, mbar_wait_bounded(b, phase, abort_flag, nullptr, 0, tp.poll_limit)); };

    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(bar(bars.full[i]), 32); mbar_init(bar(bars.empty[i]), 1); }
        for (int w = 0; w < 2; ++w) { mbar_init(bar(bars.q_full[w]), 32); mbar_init(bar(bars.q_empty[w]), 1); mbar_init(bar(bars.s_full[w]), 1); mbar_init(bar(bars.p_full[w]), 256); mbar_init(bar(bars.f_full[w]), 1); }
        for (int i = 0; i < 4; ++i) mbar_init(bar(bars.pair[i]), 64);
        mbar_init(bar(bars.drain), 1);
        abort_word = 0;
        for (int i = 0; i < 10; ++i) filled[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 11) {
        tmem_alloc(unsigned(__cvta_generic_to_shared(&tmem_base_word)), 512);
        tmem_relinquish();
    }
    early_begin();

    // ---- this CTA's share ----
    const int per = (p.sequences + kTreeThreads - 1) / kTreeThreads;
    {
        int64_t mine = 0;                                       // tiles * 2^24 + sequences that have any
        for (int i = 0; i < per; ++i) {
            const int s = tid * per + i;
            if (s >= p.sequences) break;
            const int32_t length = p.lengths[s];
            TreeSpan span;
            span.set(p, length);
            mine += (int64_t(span.tiles) << 24) + (span.tiles > 0 ? 1 : 0);
            if (blockIdx.x == 0 && p.flags && rare(AttentionSpan<true>::bad(p, length))) atomicOr(p.flags, int(BTC_FLAG_BAD_LENGTH));
        }
        int64_t x = mine;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, k);
            if (lane >= k) x += y;
        }
        scan[tid + 1] = x;
        if (tid == 0) scan[0] = 0;
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        int64_t before = 0;
        for (int w = 0; w < warp; ++w) before += scan[(w + 1) * 32];
        __syncthreads();
        scan[tid + 1] = x + before;
        proxy_fence_async();                                    // bulk copies will write where these sums lie
        __syncthreads();
    }
    const unsigned tmem = *reinterpret_cast<volatile uint32_t *>(&tmem_base_word);
    if (warp == 0) {
        auto units = [&](int i) { return ((scan[i] >> 24) + (scan[i] & 0xffffff) * kTreeItemTiles) * head_blocks; };
        const int64_t total = units(kTreeThreads), ctas = min(total, int64_t(gridDim.x));
        int64_t tiles_before = (scan[kTreeThreads] >> 24) * head_blocks;
        TreeCursor cur;
        cur.seq = p.sequences;
        cur.hb = cur.tile = cur.key_head = cur.block = 0;
        cur.span.begin = cur.span.end = cur.span.cached = cur.span.first_tile = cur.span.tiles = 0;
        if (blockIdx.x < ctas) {
            // lanes 0 and 1 look up where the share begins and ends
            const int64_t each = total / ctas, more = total - each * ctas;
            const int64_t lo = each * blockIdx.x + min(int64_t(blockIdx.x), more), hi = lo + each + (int64_t(blockIdx.x) < more ? 1 : 0);
            const int64_t unit = lane == 1 ? hi : lo;
            if (unit < total) {
                int a = 0, b = kTreeThreads;                    // units(a) <= unit < units(b)
                while (b - a > 1) {
                    const int c = (a + b) / 2;
                    if (units(c) <= unit) a = c; else b = c;
                }
                int64_t at = unit - units(a);
                tiles_before = (scan[a] >> 24) * head_blocks;
                cur.seq = a * per;
                cur.span.set(p, p.lengths[cur.seq]);
                while (cur.seq + 1 < p.sequences) {
                    const int64_t here = cur.span.tiles > 0 ? int64_t(cur.span.tiles + kTreeItemTiles) * head_blocks : 0;
                    if (at < here) break;
                    at -= here;
                    tiles_before += int64_t(cur.span.tiles) * head_blocks;
                    cur.span.set(p, p.lengths[++cur.seq]);
                }
                const int32_t item_units = cur.span.tiles + kTreeItemTiles;
                cur.hb = int32_t(at / item_units);
                cur.tile = max(0, int32_t(at - int64_t(cur.hb) * item_units) - kTreeItemTiles);
                tiles_before += int64_t(cur.hb) * cur.span.tiles + cur.tile;
                cur.key_head = cur.hb / p.blocks;
                cur.block = cur.hb - cur.key_head * p.blocks;
            }
        }
        const int64_t to = __shfl_sync(0xffffffffu, tiles_before, 1);
        if (lane == 0) {
            start = cur;
            share = to - tiles_before;
        }
    }
    __syncthreads();
    int64_t left = share;
    TreeCursor cur = start;

    // 384 threads x 168 registers at launch hold 128 x 64 and 256 x 216
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;" ::: "memory");
    if (warp < 11) {
        // ---- loaders: a copy of 128 tokens' keys or values to a warp, in turn; the first one also brings the queries ----
        constexpr int CHUNKS = DP / 8, STEP = 32 / CHUNKS;       // chunks of a row; rows of a warp's copy
        const int lw = warp - 8, sub = lane / CHUNKS, chunk = lane % CHUNKS;
        const unsigned in_row = unsigned((chunk >> 3) * PANEL);
        int turn = 0, info = 0, q_slot = 0, slot = 0;            // copies so far modulo 3; the next one's place in the ring
        unsigned phase = 0, q_phase = 0;
        bool ok = true;
        while (ok && left > 0) {
            const int cnt = int(min(int64_t(cur.span.tiles - cur.tile), left)), rows = cur.rows(p), row0 = cur.block * 2 * kTreeRows;
            const bool two = WIDE && rows > kTreeRows;
#pragma unroll 1
            for (int w = 0; w < (two ? 2 : 1); ++w) {
                const unsigned full = bar(bars.q_full[q_slot]), to = q_at + unsigned(q_slot) * TILE;
                if (lw == 0) {
                    if (!(ok = wait(bar(bars.q_empty[q_slot]), q_phase ^ 1u))) break;
                    if (lane == 0) filled[8 + q_slot] = 1 + q_phase;
                    if (tp.box_q) {
                        // a box: the heads that share a key head x some drafts, in the order of the rows (zeros behind the last draft)
                        if (elect_one()) {
                            mbar_arrive_expect_tx(full, unsigned(PANELS * tp.box_q) * p.sharing.d * 128u);
#pragma unroll
                            for (int pn = 0; pn < PANELS; ++pn)
                                tma_load_box(to + unsigned(pn) * PANEL, &map_q, full, 64 * pn, 0, int(p.sharing.div(uint32_t(row0 + w * kTreeRows))), cur.key_head, cur.seq);
                        } else {
                            mbar_arrive(full);
                        }
                        __syncwarp();
                    } else {
                        const int bytes_k = max(0, min(16, (p.dim_k - chunk * 8) * 2));
#pragma unroll 1
                        for (int r = sub; r < kTreeRows; r += STEP) {
                            const int row = w * kTreeRows + r;
                            const T *src = static_cast<const T *>(p.q);
                            const bool there = row < rows;
                            if (there) {
                                int32_t draft;
                                const int64_t head = attention_row<true>(p, cur.key_head, row0 + row, draft);
                                src += cur.seq * p.q_n + head * p.q_h + draft * p.q_t;
                            }
                            const unsigned dst = to + in_row + unsigned(r) * 128u + unsigned(((chunk ^ r) & 7) << 4);
                            if (tp.vec_q) {
                                const int bytes = there ? bytes_k : 0;
                                cp_async_part(dst, bytes ? src + chunk * 8 : static_cast<const T *>(p.q), bytes);
                            } else {
#pragma unroll 1
                                for (int e = 0; e < 8; ++e) {
                                    unsigned short x = 0;
                                    if (there && chunk * 8 + e < p.dim_k) x = *reinterpret_cast<const unsigned short *>(src + (chunk * 8 + e) * p.q_d);
                                    asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst + 2u * unsigned(e)), "h"(x) : "memory");
                                }
                            }
                        }
                        if (tp.vec_q) mbar_arrive_on_copies(full); else mbar_arrive(full);
                    }
                }
                if ((q_slot ^= 1) == 0) q_phase ^= 1u;
            }
            if (!ok) break;
#pragma unroll 1
            for (int i = 0; i < 2 * cnt; ++i) {
                const bool my_turn = turn == lw;
                if (++turn == 3) turn = 0;
                const int here = slot;
                const unsigned here_phase = phase;
                if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
                if (!my_turn) continue;
                int kv;
                const int j = tree_placed(i, cnt, two, kv), token0 = (cur.span.first_tile + cur.tile + j) * kTreeTok;
                // pages of the tokens lane, lane + 32, ..: -1 where the token is not visible or its entry is no page
                int32_t page[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int t = token0 + 32 * g + lane;
                    page[g] = -1;
                    if (t >= cur.span.begin && t < cur.span.end) page[g] = p.table[cur.seq * p.table_n + int64_t(p.page.div(uint32_t(t))) * p.table_j];
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int t = token0 + 32 * g + lane;
                    if (rare(page[g] >= p.pages || (page[g] < 0 && t >= cur.span.begin && t < cur.span.end))) {
                        if (p.flags && t < cur.span.cached) atomicOr(p.flags, int(BTC_FLAG_BAD_PAGE));
                        page[g] = -1;
                    }
                }
                if (!(ok = wait(bar(bars.empty[here]), here_phase ^ 1u))) break;
                if (lane == 0) filled[here] = 1 + here_phase;
                if (kv == 0) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const uint32_t seen = __ballot_sync(0xffffffffu, page[g] >= 0);
                        if (lane == g) infos[(info + j) % kTreeInfos][g] = seen;
                    }
                }
                const unsigned dst = ring_at + unsigned(here) * TILE, full = bar(bars.full[here]);
                if (tp.box_kv && token0 >= cur.span.begin && token0 + kTreeTok <= cur.span.end) {
                    // all tokens are visible: boxes of a page's rows, zeros where the page is none (its number lies outside)
                    if (elect_one()) mbar_arrive_expect_tx(full, TILE);
                    else mbar_arrive(full);
                    __syncwarp();
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        // boxes that begin in these 32 tokens: one each 8, 16 or 32, or the first of 64 or 128
                        if (g & (max(tp.box_kv, 32) / 32 - 1)) continue;
#pragma unroll 1
                        for (int o = 0; o < 32; o += tp.box_kv) {
                            const int32_t n = __shfl_sync(0xffffffffu, page[g], o);
                            const int t = token0 + 32 * g + o, row = t - int32_t(p.page.div(uint32_t(t)) * p.page.d);
                            if (elect_one()) {
#pragma unroll
                                for (int pn = 0; pn < PANELS; ++pn)
                                    tma_load_box4(dst + unsigned(pn) * PANEL + unsigned(32 * g + o) * 128u, kv == 0 ? &map_k : &map_v, full, 64 * pn, row, cur.key_head, n);
                            }
                            __syncwarp();
                        }
                    }
                } else {
                    const T *base = static_cast<const T *>(kv == 0 ? p.k : p.v) + cur.key_head * (kv == 0 ? p.k_head : p.v_head) + chunk * 8;
                    const uint32_t s_page = kv == 0 ? tp.k_page16 : tp.v_page16, s_slot = kv == 0 ? tp.k_slot16 : tp.v_slot16;
                    const int bytes = max(0, min(16, ((kv == 0 ? p.dim_k : p.dim_v) - chunk * 8) * 2));
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        // in units of 16 bytes, so that 32 bits hold it: one exchange per row
                        const int t = token0 + 32 * g + lane;
                        const uint32_t at = page[g] < 0 ? ~0u : uint32_t(page[g]) * s_page + uint32_t(t - int32_t(p.page.div(uint32_t(t)) * p.page.d)) * s_slot;
#pragma unroll 4
                        for (int r = 0; r < 32; r += STEP) {
                            const uint32_t from = __shfl_sync(0xffffffffu, at, r + sub);
                            const int n16 = from == ~0u ? 0 : bytes;
                            cp_async_part(dst + in_row + unsigned(32 * g + r + sub) * 128u + unsigned(((chunk ^ (r + sub)) & 7) << 4),
                                          base + (n16 ? int64_t(from) * 8 : -chunk * 8), n16);
                        }
                    }
                    mbar_arrive_on_copies(full);
                }
            }
            info = (info + cnt) % kTreeInfos;
            left -= cnt;
            cur.next(p);
        }
        cp_async_wait_all();
        if (lw == 2) report_drafts(p, lane);
    } else {
        // ---- products ----
        const unsigned idesc_s = umma16_instr_desc<T>(kTreeTok, false), idesc_f = umma16_instr_desc<T>(DP, true);
        const unsigned full0 = bar(bars.full[0]), empty0 = bar(bars.empty[0]);
        int base_slot = 0;                                       // place and round of the item's first keys in the ring
        unsigned base_phase = 0, q_phase = 0, p_phase[2] = {0, 0};
        int parity = 0, q_slot = 0;                              // of the item's first step; next place of queries
        bool ok = true;
        auto place = [&](int i, unsigned &phase) {               // of the i-th tile copied since base
            int s = base_slot + i;
            phase = base_phase ^ (unsigned(s / SLOTS) & 1u);
            return s % SLOTS;
        };
        while (ok && left > 0) {
            const int cnt = int(min(int64_t(cur.span.tiles - cur.tile), left)), shift = WIDE && cur.rows(p) > kTreeRows ? 1 : 0, steps = cnt << shift;
            int q_slots[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (w > shift) break;
                q_slots[w] = q_slot;
                ok = ok && wait(bar(bars.q_full[q_slot]), q_phase);
                if ((q_slot ^= 1) == 0) q_phase ^= 1u;
            }
            if (!ok) break;
            auto scores = [&](int i) -> bool {
                const int w = shift ? i & 1 : 0, b = (parity + i) & 1;
                unsigned phase;
                const int s = place(tree_place_k(i >> shift, shift), phase);
                if (!wait(full0 + 8u * s, phase)) return false;
                tc_fence_after();
                proxy_fence_async();
                if (elect_one()) {
                    const unsigned qs = q_at + unsigned(w ? q_slots[1] : q_slots[0]) * TILE, ks = ring_at + unsigned(s) * TILE;
#pragma unroll
                    for (int pn = 0; pn < PANELS; ++pn)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma16(tmem + unsigned(b) * 256u, umma_smem_desc(qs + pn * PANEL + k * 32, 16, 1024, 2),
                                   umma_smem_desc(ks + pn * PANEL + k * 32, 16, 1024, 2), idesc_s, pn || k ? 1u : 0u);
                    umma_commit(bar(bars.s_full[b]));
                    if (w == shift) umma_commit(empty0 + 8u * s);
                    if (i + shift + 1 >= steps) umma_commit(bar(bars.q_empty[w ? q_slots[1] : q_slots[0]]));
                }
                __syncwarp();
                return true;
            };
            for (int i = 0; ok && i < 2 && i < steps; ++i) ok = scores(i);
            for (int i = 0; ok && i < steps; ++i) {
                const int w = shift ? i & 1 : 0, b = (parity + i) & 1;
                unsigned phase;
                const int s = place(tree_place_v(i >> shift, cnt, shift), phase);
                if (!(ok = wait(full0 + 8u * s, phase))) break;
                if (!(ok = wait(bar(bars.p_full[b]), p_phase[b]))) break;
                p_phase[b] ^= 1u;
                tc_fence_after();
                proxy_fence_async();
                if (elect_one()) {
                    const unsigned ps = tmem + unsigned(b) * 256u, f = ps + 128u, vs = ring_at + unsigned(s) * TILE;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint64_t db = umma_smem_desc(vs + k * 2048, PANEL, 1024, 2);
                        const unsigned pa = ps + 16u * unsigned(k);
                        umma16_ts(f, pa + 8u, db, idesc_f, k ? 1u : 0u);
                        umma16_ts(f, pa, db, idesc_f, 1u);
                    }
                    umma_commit(bar(bars.f_full[b]));
                    if (w == shift) umma_commit(empty0 + 8u * s);
                }
                __syncwarp();
                if (i + 2 < steps) ok = scores(i + 2);
            }
            parity = (parity + steps) & 1;
            {
                const int64_t n = int64_t(base_slot) + 2 * int64_t(cnt);
                base_phase ^= unsigned(n / SLOTS) & 1u;
                base_slot = int(n % SLOTS);
            }
            left -= cnt;
            cur.next(p);
        }
    }
    } else {
        // ---- softmax ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;" ::: "memory");
        constexpr int HALF = DP / 2;                             // elements of the head that a thread keeps
        const int half = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        const unsigned lanes = unsigned(quarter * 32) << 16;
        unsigned s_phase[2] = {0, 0}, f_phase[2] = {0, 0}, pair_phase = 0;
        int info = 0, parity = 0;
        int32_t parts[2] = {-1, -1};                             // items that the CTA does not hold whole: one that began earlier, one that goes on
        bool ok = true;
        auto pair_wait = [&]() -> bool {
            mbar_arrive(bar(bars.pair[quarter]));
            const bool good = wait(bar(bars.pair[quarter]), pair_phase);
            pair_phase ^= 1u;
            return good;
        };
        while (ok && left > 0) {
            const int cnt = int(min(int64_t(cur.span.tiles - cur.tile), left)), rows = cur.rows(p), shift = WIDE && rows > kTreeRows ? 1 : 0, steps = cnt << shift;
            const int row0 = cur.block * 2 * kTreeRows;
            // the row's mask, and how many drafts it sees
            auto load_mask = [&](int row, uint32_t (&mask)[4]) -> int {
                int32_t draft;
                attention_row<true>(p, cur.key_head, row0 + row, draft);
                const int32_t *at = p.masks + cur.seq * p.m_n + draft * p.m_t;
                int drafts = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mask[i] = 0;
                    if (i < p.words) {
                        mask[i] = uint32_t(at[i * p.m_w]);
                        if (p.drafts - 32 * i < 32) mask[i] &= (1u << (p.drafts - 32 * i)) - 1u;
                        drafts += __popc(mask[i]);
                    }
                }
                return drafts;
            };
            // do the rows hold drafts?  (Asked here, where the first scores are still waited for.)
            bool empty0 = true, empty1 = true;
            {
                uint32_t mask[4];
                if (r < rows) empty0 = load_mask(r, mask) == 0;
                if (WIDE && kTreeRows + r < rows) empty1 = load_mask(kTreeRows + r, mask) == 0;
            }
            float o0[HALF], o1[WIDE ? HALF : 1], m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f, alpha = 1.f;
#pragma unroll
            for (int d = 0; d < HALF; ++d) o0[d] = 0.f;
#pragma unroll
            for (int d = 0; d < (WIDE ? HALF : 1); ++d) o1[d] = 0.f;
            // add F of step i, whose exponentials were taken against the maximum m, to the output
            auto add = [&](float (&o)[HALF], int i, float m) -> bool {
                const int b = (parity + i) & 1, w = shift ? i & 1 : 0;
                if (!wait(bar(bars.f_full[b]), f_phase[b])) return false;
                f_phase[b] ^= 1u;
                tc_fence_after();
                const bool mine = w * kTreeRows + r < rows;
                if (!__any_sync(0xffffffffu, mine)) return true;
                uint32_t v[HALF];
                const unsigned f_at = tmem + unsigned(b) * 256u + 128u + unsigned(half * HALF) + lanes;
                if constexpr (HALF == 64) tmem_load64(f_at, v); else tmem_load32(f_at, v);
                tmem_load_wait();
                const int j = i >> shift, token0 = (cur.span.first_tile + cur.tile + j) * kTreeTok;
                if (tree_differs(p, token0, cur.span.cached)) {
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < HALF; ++e) odd |= (v[e] & 0x7f800000u) == 0x7f800000u;
                    if (rare(__any_sync(0xffffffffu, odd && mine))) {
                        float again[HALF];
                        const int row = mine ? w * kTreeRows + r : 0;
                        uint32_t mask[4];
                        const int drafts = load_mask(row, mask);
                        tree_plain_values<T, HALF>(p, cur, infos[(info + j) % kTreeInfos], token0, p.window > 0 ? cur.span.cached + drafts - p.window : 0,
                                                   mask[0], mask[1], mask[2], mask[3], row0 + row, m == -INFINITY ? 0.f : m, half * HALF, again);
#pragma unroll
                        for (int e = 0; e < HALF; ++e) v[e] = __float_as_uint(again[e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < HALF; ++e) o[e] = fmaf(o[e], alpha, __uint_as_float(v[e]));
                return true;
            };
            for (int i = 0; i < steps; ++i) {
                const int b = (parity + i) & 1, w = shift ? i & 1 : 0, j = i >> shift, row = w * kTreeRows + r;
                const int token0 = (cur.span.first_tile + cur.tile + j) * kTreeTok;
                const unsigned s_at = tmem + unsigned(b) * 256u + unsigned(half * 64) + lanes;
                if (!(ok = wait(bar(bars.s_full[b]), s_phase[b]))) break;
                s_phase[b] ^= 1u;
                tc_fence_after();
                float next_alpha = 1.f;
                // the maximum of the step before, whose F is added below: this step's softmax moves that of its rows on
                const float before = WIDE && shift && w == 0 ? m1 : m0;
                if (__any_sync(0xffffffffu, row < rows)) {
                    const uint32_t *words = infos[(info + j) % kTreeInfos];
                    const bool masked = (words[0] & words[1] & words[2] & words[3]) != ~0u || tree_differs(p, token0, cur.span.cached);
                    uint32_t vis[2] = {~0u, ~0u};
                    if (masked) {
                        uint32_t mask[4];
                        const int drafts = load_mask(row < rows ? row : 0, mask), low = p.window > 0 ? cur.span.cached + drafts - p.window : 0;
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            vis[c] = drafts == 0 ? 0u : tree_visible(token0 + 64 * half + 32 * c, cur.span.cached, low, mask) & words[2 * half + c];
                    }
                    float top = -INFINITY;
                    uint32_t v[64];
                    tmem_load64(s_at, v);
                    tmem_load_wait();
                    // the largest scaled score is that of the largest score, or of the smallest one where the scale is negative
                    const bool up = p.scale_log2 >= 0.f;
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 64; ++e)             // what is not visible has the probability zero
                            if (!((vis[e >> 5] >> (e & 31)) & 1)) v[e] = up ? 0xff800000u : 0x7f800000u;
                    }
                    float tt[2] = {up ? -INFINITY : INFINITY, up ? -INFINITY : INFINITY};
                    if (up) {
#pragma unroll
                        for (int e = 0; e < 64; e += 4) {
                            tt[0] = fmaxf(tt[0], fmaxf(__uint_as_float(v[e]), __uint_as_float(v[e + 1])));
                            tt[1] = fmaxf(tt[1], fmaxf(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])));
                        }
                        top = fmaxf(tt[0], tt[1]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 64; ++e) tt[0] = fminf(tt[0], __uint_as_float(v[e]));
                        top = tt[0];
                    }
                    top = top == (up ? -INFINITY : INFINITY) ? -INFINITY : top * p.scale_log2;
                    tops[i & 1][half][r] = top;
                    if (!(ok = pair_wait())) break;
                    top = fmaxf(top, tops[i & 1][half ^ 1][r]);
                    const float m = w ? m1 : m0, now = fmaxf(m, top), base = now == -INFINITY ? 0.f : now;
                    next_alpha = m == now ? 1.f : ex2(m - now);
                    float sum[2] = {0.f, 0.f};
                    // 16 tokens: S -> P in two parts, in the place of S
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t out[16];
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            float x[2];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                x[h] = ex2(fmaf(__uint_as_float(v[16 * c + e + h]), p.scale_log2, -base));
                                if (AttentionBias<T>::factor != 1.f) x[h] *= AttentionBias<T>::factor;
                            }
                            sum[0] += x[0];
                            sum[1] += x[1];
                            const uint32_t hi = pack2(x[0], x[1], T());
                            float a, c2;
                            unpack_word(hi, a, c2, T());
                            out[e / 2] = hi;
                            out[8 + e / 2] = pack2(x[0] - a, x[1] - c2, T());
                        }
                        tmem_store16u(s_at + 16u * c, out);
                    }
                    tmem_store_wait();
                    const float l = (w ? l1 : l0) * next_alpha + (sum[0] + sum[1]);
                    if (w) { m1 = now; l1 = l; } else { m0 = now; l0 = l; }
                }
                tc_fence_before();
                mbar_arrive(bar(bars.p_full[b]));
                if (i > 0) {
                    if constexpr (WIDE) ok = (shift && w == 0) ? add(o1, i - 1, before) : add(o0, i - 1, before);
                    else ok = add(o0, i - 1, before);
                    if (!ok) break;
                }
                alpha = next_alpha;
            }
            if (!ok) break;
            if constexpr (WIDE) ok = shift ? add(o1, steps - 1, m1) : add(o0, steps - 1, m0);
            else ok = add(o0, steps - 1, m0);
            if (!ok) break;
            parity = (parity + steps) & 1;
            const bool whole = cur.tile == 0 && cnt == cur.span.tiles;
            // the two warps' sums
            auto finish = [&](float (&o)[HALF], float m, float l, int w) -> bool {
                tops[0][half][r] = l;
                if (!pair_wait()) return false;
                l += tops[0][half ^ 1][r];
                if (!pair_wait()) return false;                  // read by both before either writes again
                const int row = w * kTreeRows + r;
                if (row >= rows) return true;
                int32_t draft;
                const int head = attention_row<true>(p, cur.key_head, row0 + row, draft);
                if (w ? empty1 : empty0) { m = -INFINITY; l = 0.f; }
                if (!whole) {
                    float *part = tp.partial + ((2 * int64_t(blockIdx.x) + (cur.tile == 0 ? 1 : 0)) * 2 + w) * Shape::PART;
#pragma unroll
                    for (int d = 0; d < HALF; ++d) part[(half * HALF + d) * kTreeRows + r] = o[d];
                    if (half == 0) {
                        part[DP * kTreeRows + r] = m;
                        part[DP * kTreeRows + kTreeRows + r] = l;
                    }
                    return true;
                }
                const bool nothing = l == 0.f;
                const float inv = 1.f / l;
                T *dst = static_cast<T *>(p.o) + cur.seq * p.o_n + draft * p.o_t + int64_t(head) * p.o_h;
                tree_write<T, HALF>(dst, half * HALF, p.dim_v, p.o_d, tp.vec_o, o, nothing ? 0.f : inv, nothing);
                if (p.lse && half == 0)
                    p.lse[(int64_t(cur.seq) * p.drafts + draft) * p.heads + head] = nothing ? -INFINITY
                        : (m + (log2f(l) - AttentionBias<T>::value)) * 0.6931471805599453f;
                return true;
            };
            if (!(ok = finish(o0, m0, l0, 0))) break;
            if constexpr (WIDE)
                if (shift && !(ok = finish(o1, m1, l1, 1))) break;
            if (!whole) parts[cur.tile == 0 ? 1 : 0] = cur.seq * head_blocks + cur.hb;
            info = (info + cnt) % kTreeInfos;
            left -= cnt;
            cur.next(p);
        }
        if (tid == 0) {
            tp.partial_item[2 * blockIdx.x] = parts[0];
            tp.partial_item[2 * blockIdx.x + 1] = parts[1];
        }
    }

    // sequences with nothing to see
    for (int s = blockIdx.x; s < p.sequences; s += gridDim.x) {
        TreeSpan span;
        span.set(p, p.lengths[s]);
        if (rare(span.tiles == 0)) {
            for (int e = tid; e < p.heads * p.dim_v; e += kTreeThreads) {
                const int h = e / p.dim_v, d = e - h * p.dim_v;
                for (int t = 0; t < p.drafts; ++t)
                    static_cast<T *>(p.o)[s * p.o_n + t * p.o_t + int64_t(h) * p.o_h + d * p.o_d] = from_f32<T>(0.f);
            }
            if (p.lse)
                for (int h = tid; h < p.heads * p.drafts; h += kTreeThreads) p.lse[int64_t(s) * p.heads * p.drafts + h] = -INFINITY;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (rare(*abort_flag)) {
        if (warp < 8) tree_spoil<T>(tp, start, share);
        // copies that nobody waited for have to land before the CTA gives up its shared memory: the last ones into each place
        if (warp == 8 && lane < 10 && filled[lane] != 0) {
            const unsigned b = lane < 8 ? bar(bars.full[lane]) : bar(bars.q_full[lane - 8]);
            for (unsigned n = 0; n < (1u << 16) && !mbar_try_wait(b, filled[lane] - 1); ++n) { }
        }
    }
    if (warp == 11) {
        if (*abort_flag) {
            if (elect_one()) umma_commit(bar(bars.drain));
            __syncwarp();
            for (unsigned n = 0; n < (1u << 16) && !mbar_try_wait(bar(bars.drain), 0u); ++n) { }
            if (p.flags && lane == 0) atomicOr(p.flags, int(BTC_FLAG_TIMEOUT));
        }
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Items that span CTAs, as in the one-token kernels: block (c, y) joins 16 rows of the item that begins in CTA c's range and ends in a
// later one's; a thread has DP / 16 elements of a row.  The parts' maxima, and eight parts' elements, are loaded side by side.
constexpr int kTreeJoinThreads = 256, kTreeJoinRows = 16;
template <typename T, int DP>
__global__ void __launch_bounds__(kTreeJoinThreads) tree_join_kernel(const __grid_constant__ TreeParams tp, int ctas)
{
    constexpr int GROUPS = kTreeJoinThreads / kTreeJoinRows, EACH = DP / GROUPS, AHEAD = 4;
    const AttentionParams &p = tp.a;
    __shared__ int32_t parts, lost_at;
    __shared__ float all_tops[GROUPS][kTreeJoinRows], all_sums[GROUPS][kTreeJoinRows];
    const int c = blockIdx.x, tid = threadIdx.x, group = tid / kTreeJoinRows;
    early_begin();
    const int32_t item = load_now(tp.partial_item + 2 * c + 1);
    if (item < 0) return;
    const int left = ctas - c;
    const int32_t other = tid + 1 < left ? load_now(tp.partial_item + 2 * (c + tid + 1)) : -1;
    if (tid == 0) { parts = left; lost_at = INT32_MAX; }
    __syncthreads();
    auto ends = [&](int i, int32_t here) {                      // does the item end before CTA c + i?
        if (here == item) return;
        atomicMin(&parts, i);
        if (here == kTreeLost) atomicMin(&lost_at, i);
    };
    if (tid + 1 < left) ends(tid + 1, other);
    for (int i = tid + 1 + kTreeJoinThreads; i < left; i += kTreeJoinThreads) ends(i, tp.partial_item[2 * (c + i)]);
    __syncthreads();
    const int n = parts;
    const bool lost = lost_at == n;                             // by a CTA in which a wait gave up, and which may have held a part
    const int head_blocks = p.key_heads * p.blocks;
    const int seq = item / head_blocks, hb = item - seq * head_blocks, kh = hb / p.blocks, block = hb - kh * p.blocks;
    const int row = blockIdx.y * kTreeJoinRows + tid % kTreeJoinRows, group_row = block * 2 * kTreeRows + row;
    const bool mine = row < min(2 * kTreeRows, p.group - block * 2 * kTreeRows);
    const float *first = tp.partial + (4 * int64_t(c) + (row >> 7)) * TreeShape<DP>::PART + (row & 127);
    auto part = [&](int i) { return first + (i == 0 ? 2 : 4 * int64_t(i)) * TreeShape<DP>::PART; };
    // every 16th part's maximum and sum to a group
    float top = -INFINITY, l = 0.f;
    for (int i = group; mine && i < n; i += GROUPS) {
        const float m = part(i)[DP * kTreeRows], x = part(i)[DP * kTreeRows + kTreeRows], now = fmaxf(top, m);
        l = l * join_weight(top, now) + x * join_weight(m, now);
        top = now;
    }
    all_tops[group][tid % kTreeJoinRows] = top;
    all_sums[group][tid % kTreeJoinRows] = l;
    __syncthreads();
    if (!mine) return;
    top = -INFINITY;
    for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, all_tops[i][tid % kTreeJoinRows]);
    l = 0.f;
    for (int i = 0; i < GROUPS; ++i) l = fmaf(all_sums[i][tid % kTreeJoinRows], join_weight(all_tops[i][tid % kTreeJoinRows], top), l);
    if (rare(lost)) l = NAN;
    float o[EACH];
#pragma unroll
    for (int d = 0; d < EACH; ++d) o[d] = 0.f;
    for (int i = 0; i < n; i += AHEAD) {
        float x[AHEAD][EACH], m[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            m[a] = -INFINITY;
            if (i + a < n) m[a] = part(i + a)[DP * kTreeRows];
#pragma unroll
            for (int d = 0; d < EACH; ++d) x[a][d] = i + a < n ? part(i + a)[(group * EACH + d) * kTreeRows] : 0.f;
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (i + a >= n) continue;
            const float share = join_weight(m[a], top);
#pragma unroll
            for (int d = 0; d < EACH; ++d) o[d] = fmaf(x[a][d], share, o[d]);
        }
    }
    int32_t draft;
    const int head = attention_row<true>(p, kh, group_row, draft);
    const bool nothing = l == 0.f;
    T *dst = static_cast<T *>(p.o) + seq * p.o_n + draft * p.o_t + int64_t(head) * p.o_h;
    if constexpr (EACH == 8) {
        tree_write<T, 8>(dst, group * 8, p.dim_v, p.o_d, tp.vec_o, o, 1.f / l, nothing);
    } else {
#pragma unroll
        for (int d = 0; d < EACH; ++d)
            if (group * EACH + d < p.dim_v) dst[(group * EACH + d) * p.o_d] = from_f32<T>(nothing ? 0.f : o[d] * (1.f / l));
    }
    if (group == 0 && p.lse)
        p.lse[(int64_t(seq) * p.drafts + draft) * p.heads + head] = nothing ? -INFINITY : (top + (log2f(l) - AttentionBias<T>::value)) * 0.6931471805599453f;
}

}  // namespace btc
