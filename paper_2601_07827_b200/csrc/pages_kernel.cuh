// Bookkeeping and copies of a paged key-value cache.
//
// State (the caller's device memory): table [sequences][columns] of page numbers (-1: none), lengths, and one
// reference count per page (0: free).  Integer work on a few hundred KB: bound by latency, so each operation is one
// launch (plus one that moves page contents, where there are any).  extend and compact need a prefix sum over the
// whole pool; a cluster of 8 CTAs holds it in one launch: every CTA scans an eighth of the pool, the totals are
// exchanged through distributed shared memory, and cluster barriers separate reading the old state from
// writing the new one.  Free pages are handed out lowest number first and compaction keeps the order, so
// results do not depend on scheduling (the only atomics are integer additions).
// Page contents move with 16-byte accesses where sizes, strides and addresses allow, 16 KB per CTA and step: bound by
// HBM (each byte is read once and written once).
// Measured (replayed graphs): 8 sequences freed, 8 forked and 64 extended by a token 14.6 us, the same over 1000 sequences and
// 200000 pages 21.5 us; a compaction that moves 235 MB of pages 87 us, of which the copy is 70 (6.7 TB/s).
#pragma once

#include "../../include/btc.h"
#include "decoder_common.cuh"

namespace btc {

constexpr int kPagesCluster = 8, kPagesThreads = 1024;
constexpr int kPagesMaxDims = 8, kPagesMaxLayouts = 4, kPagesMaxTensors = 128;
constexpr int kPagesCopyThreads = 256, kPagesCopyUnits = 4;   // units per thread and step

struct PagesParams {
    int32_t *table, *lengths, *refs, *flags;
    int64_t table_n, table_j;
    int32_t sequences, columns, pages;
    FastDiv page;                        // tokens per page
    int32_t page_tokens;
    int32_t room;                        // tokens a table row can hold
    const int32_t *fresh;                // extend: new tokens per sequence
    int32_t *slots;                      // extend: [sequences][most]
    int32_t most;
    // workspace
    int32_t *count;                      // [0]: pairs in the list, [1]: compact: live pages
    int32_t *pairs;                      // (source, destination) ...
    int32_t *holes;                      // extend: free pages; compact: free pages below the live count
    int32_t *movers;                     // compact: live pages beyond it
    int32_t *map;                        // compact: new number of a page
    int64_t *begin;                      // extend: pages taken by the CTA's earlier sequences
    int32_t *rank;                       // extend: copies among the CTA's earlier sequences * 2 + (this one copies); -1: takes no part
};

struct PagesLayout {
    int64_t page_stride;                 // in units
    int64_t dim_stride[kPagesMaxDims];   // in units, smallest first
    FastDiv dim[kPagesMaxDims];
    int32_t dims;
    uint32_t units, chunks;              // units of one page; steps of a CTA for them
};
struct PagesCopyParams {
    PagesLayout layout[kPagesMaxLayouts];
    void *tensor[kPagesMaxTensors];
    int32_t layouts, tensors;            // tensor t has layout t % layouts
    uint32_t chunks;                     // of all layouts
    const int32_t *pairs;
    const int32_t *count;                // device count of pairs, or NULL: `most` pairs
    int64_t most;
    int32_t pages;
    int32_t *flags;
    // compact: renumber the table in the same launch
    int32_t *table;
    const int32_t *map;
    const int32_t *live;
    int64_t table_n, table_j;
    int32_t sequences, columns;
};

__device__ __forceinline__ void pages_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int64_t pages_peer_value(const int64_t *mine, unsigned rank)
{
    unsigned addr;
    int64_t v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(static_cast<unsigned>(__cvta_generic_to_shared(mine))), "r"(rank));
    asm volatile("ld.shared::cluster.s64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void pages_flag(int32_t *flags, int what)
{
    if (flags) atomicOr(flags, what);
}

// exclusive prefix sum of one value per thread over the CTA; `total` gets the sum.  scratch: 33 entries
__device__ __forceinline__ int64_t block_exclusive(int64_t v, int64_t *scratch, int64_t &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t x = v;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, k);
        if (lane >= k) x += y;
    }
    __syncthreads();                                     // scratch may still be read from the call before
    if (lane == 31) scratch[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int64_t w = scratch[lane];
        const int64_t own = w;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, w, k);
            if (lane >= k) w += y;
        }
        scratch[lane] = w - own;
        if (lane == 31) scratch[32] = w;
    }
    __syncthreads();
    total = scratch[32];
    return scratch[warp] + x - v;
}

// the CTA's share of the pool: a multiple of 4 pages
__device__ __forceinline__ void pool_share(int32_t pages, unsigned rank, int32_t &lo, int32_t &hi)
{
    const int64_t each = ((int64_t(pages) + kPagesCluster - 1) / kPagesCluster + 3) / 4 * 4;
    lo = int32_t(min(int64_t(pages), each * rank));
    hi = int32_t(min(int64_t(pages), each * (rank + 1)));
}
// four consecutive reference counts (pages beyond hi read as -1)
__device__ __forceinline__ int4 four_refs(const int32_t *refs, int32_t at, int32_t hi, bool vec)
{
    if (vec && at + 4 <= hi) return __ldcg(reinterpret_cast<const int4 *>(refs + at));
    int4 r = make_int4(-1, -1, -1, -1);
    if (at < hi) r.x = __ldcg(refs + at);
    if (at + 1 < hi) r.y = __ldcg(refs + at + 1);
    if (at + 2 < hi) r.z = __ldcg(refs + at + 2);
    if (at + 3 < hi) r.w = __ldcg(refs + at + 3);
    return r;
}

// extend: every sequence takes its new tokens; pages are allocated lowest number first, in the order of the sequences.
// A last page that is shared and partly filled is replaced by a copy.  A sequence takes part when its counts are in
// order; of those, the first whose pages do not fit and all after it get nothing.
static __global__ void __cluster_dims__(kPagesCluster, 1, 1) __launch_bounds__(kPagesThreads)
pages_extend_kernel(const __grid_constant__ PagesParams p)
{
    __shared__ int64_t scratch[33], totals[3];           // totals: free pages, pages wanted, copies of this CTA
    const unsigned rank = blockIdx.x;
    const int tid = threadIdx.x;
    const bool vec = (reinterpret_cast<uintptr_t>(p.refs) & 15) == 0;
    early_begin();

    // free pages of this CTA's share; the first four of a thread stay in registers (`head`: all, in pools of up to 32768)
    int32_t lo, hi;
    pool_share(p.pages, rank, lo, hi);
    const int4 head = four_refs(p.refs, lo + 4 * tid, hi, vec);
    const int head_free = (head.x == 0) + (head.y == 0) + (head.z == 0) + (head.w == 0);
    int64_t mine = head_free;
#pragma unroll 4
    for (int32_t at = lo + 4 * tid + 4 * kPagesThreads; at < hi; at += 4 * kPagesThreads) {
        const int4 r = four_refs(p.refs, at, hi, vec);
        mine += (r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0);
    }
    int64_t total;
    const int64_t head_before = block_exclusive(mine, scratch, total);     // (of use where the head is all)
    if (tid == 0) totals[0] = total;

    // what this CTA's sequences want
    const int32_t seq_each = (p.sequences + kPagesCluster - 1) / kPagesCluster;
    const int32_t s_lo = int32_t(min(int64_t(p.sequences), int64_t(seq_each) * rank)), s_hi = int32_t(min(int64_t(p.sequences), int64_t(s_lo) + seq_each));
    int64_t wanted = 0, copies = 0;
    for (int32_t base = s_lo; base < s_hi; base += kPagesThreads) {
        const int32_t s = base + tid;
        int64_t need = 0;
        int copy = 0;
        bool part = false;
        if (s < s_hi) {
            const int32_t add = p.fresh[s], length = p.lengths[s];
            if (add < 0 || length < 0 || length > p.room || add > p.most || (add > 0 && int64_t(length) + add > p.room)) {
                pages_flag(p.flags, BTC_FLAG_BAD_LENGTH);
            } else if (add > 0) {
                const int32_t full = int32_t(p.page.div(uint32_t(length))), after = int32_t(p.page.div(uint32_t(length + add - 1))) + 1;
                part = true;
                need = after - full;
                if (length != full * p.page_tokens) {
                    const int32_t last = p.table[s * p.table_n + full * p.table_j];
                    if (last < 0 || last >= p.pages) {
                        pages_flag(p.flags, BTC_FLAG_BAD_PAGE);
                        part = false;
                        need = 0;
                    } else {
                        copy = p.refs[last] > 1;
                        need += copy - 1;
                    }
                }
            }
        }
        // both prefix sums in one: a round has at most 1024 copies
        int64_t sum;
        const int64_t before = block_exclusive(need * 2048 + copy, scratch, sum);
        if (s < s_hi) {
            p.begin[s] = wanted + before / 2048;
            p.rank[s] = part ? int32_t((copies + before % 2048) * 2 + copy) : -1;
        }
        wanted += sum / 2048;
        copies += sum % 2048;
    }
    if (tid == 0) {
        totals[1] = wanted;
        totals[2] = copies;
        if (rank == 0) p.count[0] = 0;
    }
    pages_cluster_sync();
    int64_t free_before = 0, free_all = 0, want_before = 0, want_all = 0, copies_before = 0;
#pragma unroll
    for (unsigned r = 0; r < kPagesCluster; ++r) {
        const int64_t f = pages_peer_value(&totals[0], r), w = pages_peer_value(&totals[1], r), c = pages_peer_value(&totals[2], r);
        if (r < rank) { free_before += f; want_before += w; copies_before += c; }
        free_all += f;
        want_all += w;
    }
    // the list of free pages, as far as it is wanted
    int64_t at_rank = free_before;
    for (int32_t base = lo; base < hi && at_rank < want_all; base += 4 * kPagesThreads) {
        const int32_t at = base + 4 * tid;
        const int4 r = base == lo ? head : four_refs(p.refs, at, hi, vec);
        const int32_t v[4] = {r.x, r.y, r.z, r.w};
        int64_t sum = 0;
        int64_t k = at_rank + (hi - lo <= 4 * kPagesThreads ? head_before : block_exclusive((r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0), scratch, sum));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (v[j] == 0) {
                if (k < want_all) p.holes[k] = at + j;
                ++k;
            }
        at_rank += sum;
    }
    pages_cluster_sync();                                // the old state has been read, the list is complete

    // A warp per sequence, or, where calls bring a few tokens a sequence, a thread: a step is a chain of dependent
    // accesses, and 8 CTAs of warps would go through 1000 sequences in four rounds of it.  1000 sequences, threads / warps:
    // 21.6 / 24.5 us for 1 token each, 25.5 / 25.9 for 16, 31.0 / 25.9 for 32, 62 / 32 for 128
    const int wide = p.most <= 16 ? 1 : 32, part_lane = tid & (wide - 1);
    for (int32_t s = s_lo + tid / wide; s < s_hi; s += kPagesThreads / wide) {
        const int32_t info = p.rank[s], add = p.fresh[s], length = p.lengths[s];
        const int64_t begin = p.begin[s];
        bool granted = info >= 0;
        int64_t first = 0;
        int32_t full = 0, after = 0, old = -1;
        bool copy = false, kept = false;                  // kept: the last page is partly filled (and stays or is copied)
        if (granted) {
            full = int32_t(p.page.div(uint32_t(length)));
            after = int32_t(p.page.div(uint32_t(length + add - 1))) + 1;
            kept = length != full * p.page_tokens;
            copy = info & 1;
            first = want_before + begin;
            const int64_t need = after - full + (copy ? 1 : 0) - (kept ? 1 : 0);
            granted = first + need <= free_all;
            if (!granted && part_lane == 0) pages_flag(p.flags, BTC_FLAG_POOL_EXHAUSTED);
            if (kept) old = p.table[s * p.table_n + full * p.table_j];
        }
        if (wide == 32) __syncwarp();                     // every lane has the old page before lane 0 replaces it
        if (granted) {
            const int32_t last = copy ? __ldcg(p.holes + first) : old;
            if (part_lane == 0) {
                if (copy) {
                    p.table[s * p.table_n + full * p.table_j] = last;
                    p.refs[last] = 1;
                    atomicSub(p.refs + old, 1);
                    const int64_t k = copies_before + (info >> 1);
                    p.pairs[2 * k] = old;
                    p.pairs[2 * k + 1] = last;
                    atomicMax(p.count, int32_t(k + 1));
                }
                p.lengths[s] = length + add;
            }
            const int32_t from = full + (kept ? 1 : 0);
            const int64_t list = first + (copy ? 1 : 0) - from;      // page of column j: holes[list + j]
            for (int32_t j = from + part_lane; j < after; j += wide) {
                const int32_t page = __ldcg(p.holes + list + j);
                p.table[s * p.table_n + j * p.table_j] = page;
                p.refs[page] = 1;
            }
            for (int32_t i = part_lane; i < p.most; i += wide) {
                int32_t slot = -1;
                if (i < add) {
                    const int32_t t = length + i, j = int32_t(p.page.div(uint32_t(t)));
                    const int32_t page = j < from ? last : __ldcg(p.holes + list + j);
                    slot = page * p.page_tokens + (t - j * p.page_tokens);
                }
                p.slots[int64_t(s) * p.most + i] = slot;
            }
        } else {
            for (int32_t i = part_lane; i < p.most; i += wide) p.slots[int64_t(s) * p.most + i] = -1;
        }
    }
}

// fork: row dst[i] becomes a copy of row src[i], whose pages gain a reference.  A CTA per pair.
static __global__ void __launch_bounds__(128) pages_fork_kernel(const __grid_constant__ PagesParams p, const int32_t *src, const int32_t *dst)
{
    early_begin();
    const int32_t a = src[blockIdx.x], b = dst[blockIdx.x];
    if (a < 0 || a >= p.sequences || b < 0 || b >= p.sequences || a == b || p.lengths[b] != 0) {
        if (threadIdx.x == 0) pages_flag(p.flags, BTC_FLAG_BAD_SEQUENCE);
        return;
    }
    const int32_t length = p.lengths[a];
    for (int32_t j = threadIdx.x; j < p.columns; j += blockDim.x) {
        int32_t page = p.table[a * p.table_n + j * p.table_j];
        if (page >= p.pages) {
            pages_flag(p.flags, BTC_FLAG_BAD_PAGE);
            page = -1;
        }
        p.table[b * p.table_n + j * p.table_j] = page;
        if (page >= 0) atomicAdd(p.refs + page, 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) p.lengths[b] = length;
}

// free: the rows of the listed sequences are emptied, their pages lose a reference.  A CTA per sequence; a sequence
// that is listed twice is freed once.
static __global__ void __launch_bounds__(128) pages_free_kernel(const __grid_constant__ PagesParams p, const int32_t *list)
{
    early_begin();
    const int32_t s = list[blockIdx.x];
    if (s < 0 || s >= p.sequences) {
        if (threadIdx.x == 0) pages_flag(p.flags, BTC_FLAG_BAD_SEQUENCE);
        return;
    }
    for (int32_t j = threadIdx.x; j < p.columns; j += blockDim.x) {
        const int32_t page = atomicExch(p.table + s * p.table_n + j * p.table_j, -1);
        if (page < 0) continue;
        if (page >= p.pages) {
            pages_flag(p.flags, BTC_FLAG_BAD_PAGE);
        } else if (atomicSub(p.refs + page, 1) <= 0) {     // was free already: the state was inconsistent
            atomicAdd(p.refs + page, 1);
            pages_flag(p.flags, BTC_FLAG_BAD_PAGE);
        }
    }
    if (threadIdx.x == 0) p.lengths[s] = 0;
}

// compact: with L live pages, the live pages numbered L and higher move to the free pages below L, in order.  This
// kernel makes the list of moves, the new numbers and the new counts.
static __global__ void __cluster_dims__(kPagesCluster, 1, 1) __launch_bounds__(kPagesThreads)
pages_compact_kernel(const __grid_constant__ PagesParams p)
{
    __shared__ int64_t scratch[33], totals[1];            // totals: live pages of this CTA
    const unsigned rank = blockIdx.x;
    const int tid = threadIdx.x;
    const bool vec = (reinterpret_cast<uintptr_t>(p.refs) & 15) == 0;
    early_begin();
    int32_t lo, hi;
    pool_share(p.pages, rank, lo, hi);
    const bool one_round = hi - lo <= 4 * kPagesThreads;   // pools of up to 32768: every thread has its pages in `head`
    const int4 head = four_refs(p.refs, lo + 4 * tid, hi, vec);
    int64_t mine = (head.x > 0) + (head.y > 0) + (head.z > 0) + (head.w > 0), total;
#pragma unroll 4
    for (int32_t at = lo + 4 * tid + 4 * kPagesThreads; at < hi; at += 4 * kPagesThreads) {
        const int4 r = four_refs(p.refs, at, hi, vec);
        mine += (r.x > 0) + (r.y > 0) + (r.z > 0) + (r.w > 0);
    }
    const int64_t head_before = block_exclusive(mine, scratch, total);
    if (tid == 0) totals[0] = total;
    pages_cluster_sync();
    int64_t live_before = 0, live = 0;
#pragma unroll
    for (unsigned r = 0; r < kPagesCluster; ++r) {
        const int64_t v = pages_peer_value(&totals[0], r);
        if (r < rank) live_before += v;
        live += v;
    }
    // page x: live pages before it are n(x); a hole is number x - n(x) of the holes, a mover number n(x) - n(L)
    int64_t n = live_before;
    for (int32_t base = lo; base < hi; base += 4 * kPagesThreads) {
        const int32_t at = base + 4 * tid;
        const int4 r = base == lo ? head : four_refs(p.refs, at, hi, vec);
        const int32_t v[4] = {r.x, r.y, r.z, r.w};
        int64_t sum = 0;
        int64_t k = n + (one_round ? head_before : block_exclusive((r.x > 0) + (r.y > 0) + (r.z > 0) + (r.w > 0), scratch, sum));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t x = at + j;
            if (x >= hi) break;
            if (x == live) p.count[0] = int32_t(live - k);            // n(L) pages stay: as many moves as holes below L
            if (x < live) {
                if (v[j] <= 0) p.holes[x - k] = x;
            } else {
                // movers are listed from the last live page on, so that n(L) need not be known yet
                if (v[j] > 0) p.movers[live - 1 - k] = x;
                p.map[x] = x;
            }
            k += v[j] > 0;
        }
        n += sum;
    }
    if (rank == 0 && tid == 0) {
        if (live == p.pages) p.count[0] = 0;               // a full pool: there is no page number L
        p.count[1] = int32_t(live);
    }
    pages_cluster_sync();
    const int64_t moves = __ldcg(p.count);
    for (int64_t k = int64_t(rank) * kPagesThreads + tid; k < moves; k += kPagesCluster * kPagesThreads) {
        const int32_t src = __ldcg(p.movers + (moves - 1 - k)), dst = __ldcg(p.holes + k);
        p.pairs[2 * k] = src;
        p.pairs[2 * k + 1] = dst;
        p.map[src] = dst;
        p.refs[dst] = __ldcg(p.refs + src);
        p.refs[src] = 0;
    }
}

// moves page contents and, after a compaction, renumbers the table
template <typename U>
static __global__ void __launch_bounds__(kPagesCopyThreads) pages_copy_kernel(const __grid_constant__ PagesCopyParams p)
{
    early_begin();
    if (p.table) {
        const int64_t all = int64_t(p.sequences) * p.columns;
        const int32_t live = *p.live;
        for (int64_t e = int64_t(blockIdx.x) * kPagesCopyThreads + threadIdx.x; e < all; e += int64_t(gridDim.x) * kPagesCopyThreads) {
            const int64_t s = e / p.columns, j = e - s * p.columns;
            int32_t *entry = p.table + s * p.table_n + j * p.table_j;
            const int32_t page = *entry;
            if (page >= live && page < p.pages) *entry = p.map[page];
        }
    }
    const int64_t pairs = p.count ? int64_t(*p.count) : p.most;
    const uint32_t sets = uint32_t(p.tensors / p.layouts), per_pair = sets * p.chunks;
    const int64_t steps = pairs * per_pair;
    for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
        int64_t pair;
        uint32_t rest;
        if (steps < (int64_t(1) << 31)) {
            pair = uint32_t(step) / per_pair;
            rest = uint32_t(step) - uint32_t(pair) * per_pair;
        } else {
            pair = step / per_pair;
            rest = uint32_t(step - pair * per_pair);
        }
        const int32_t src = p.pairs[2 * pair], dst = p.pairs[2 * pair + 1];
        if (src < 0 || dst < 0 || src >= p.pages || dst >= p.pages) {
            if ((src >= p.pages || dst >= p.pages) && threadIdx.x == 0) pages_flag(p.flags, BTC_FLAG_BAD_PAGE);
            continue;
        }
        const uint32_t set = rest / p.chunks;
        uint32_t chunk = rest - set * p.chunks;
        int which = 0;
        while (which + 1 < p.layouts && chunk >= p.layout[which].chunks) chunk -= p.layout[which++].chunks;
        const PagesLayout &l = p.layout[which];
        U *base = static_cast<U *>(p.tensor[set * uint32_t(p.layouts) + which]);
        const U *from = base + src * l.page_stride;
        U *to = base + dst * l.page_stride;
        const uint32_t first = chunk * (kPagesCopyThreads * kPagesCopyUnits) + threadIdx.x;
        U v[kPagesCopyUnits];
        int64_t at[kPagesCopyUnits];
#pragma unroll
        for (int i = 0; i < kPagesCopyUnits; ++i) {
            uint32_t u = first + i * kPagesCopyThreads;
            at[i] = 0;
            if (u < l.units) {
                if (l.dims <= 1) {
                    at[i] = int64_t(u) * l.dim_stride[0];
                } else {
                    int64_t off = 0;
                    for (int d = 0; d + 1 < l.dims; ++d) {
                        const uint32_t q = l.dim[d].div(u);
                        off += int64_t(u - q * l.dim[d].d) * l.dim_stride[d];
                        u = q;
                    }
                    at[i] = off + int64_t(u) * l.dim_stride[l.dims - 1];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kPagesCopyUnits; ++i)
            if (first + i * kPagesCopyThreads < l.units) v[i] = from[at[i]];
#pragma unroll
        for (int i = 0; i < kPagesCopyUnits; ++i)
            if (first + i * kPagesCopyThreads < l.units) to[at[i]] = v[i];
    }
}

}  // namespace btc
