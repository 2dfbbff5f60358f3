// Products of a few tokens with 4-bit weights and group scales, optionally as the gated half of a feed-forward block.
//
//   z[t, n] = sum_g s[n, g] sum_{k in g} x[t, k] (c[n, k] - zero[n, g]),   y = z  or  y[t, n] = act(z[t, n]) z[t, N + n]
//
// Every code is read once: 2 T multiply-adds per half byte, bound by HBM for a few tokens.  The codes become f16 or
// bf16 numbers (whole numbers of at most 15: exact), the tensor core adds up at most 64 products in fp32, and each
// such sum is multiplied by its group's scale in fp32, so that no weight is rounded.  64 products with 15 fit fp32 as long as x is at
// most 2^117.
//
// Layout ("packed"): stretches of 16 weight rows x 256 k, one after the other along k.  A stretch is its groups' scales
// [group][8][2] (rows g and g + 8), its zeros likewise in bytes, and four blocks of 64 k, 512 bytes each: 16 bytes for each
// lane of a warp, which are its part of the M-side operand of four m16n8k16 products.  Lane (g, q) = (lane / 4, lane % 4) holds rows
// g and g + 8, k = 8 q .. 8 q + 7 and 32 + 8 q .. 32 + 8 q + 7 (the products' k may be taken in any order, as long as x
// follows it: step s takes k = 32 (s / 2) + 8 q + 4 (s % 2) .. + 3 from lane q, so that a lane's x for two steps are 16 bytes in a
// row).  Word s has the step's eight codes; the pair for operand register p at bits 4 p and 16 + 4 p.  For the gated form
// rows 0..7 of a block are gates and rows 8..15 the same columns' other factors.
//
// A warp takes 16 rows and copies stretches into a ring of its own with 16-byte cp.async (with loads into registers ahead of their
// use a thread needs 160 of them, which leaves one CTA to an SM: 20 us instead of 8 for 6144 x 4096); x lies in shared memory in the
// order in which the lanes take it.
//
// Measured (replayed graphs, weights from HBM): one token 6144 x 4096 in f16 6.8 us (13 MB), gated 28672 x 4096 for 8 tokens in bf16 24.9 us (64 MB: 2.6 TB/s),
// gated 57344 x 8192 for 32 tokens 178 us in bf16 and 198 us in e4m3 (floor 37), for 1024 tokens 4.6 ms (the products alone 0.57 at the matrix rate): the
// weights are made into numbers again for every 32 tokens.  8 tokens in fp32, gated 28672 x 4096: 39.5 us.
#pragma once

#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include "../../include/btc.h"
#include "decoder_common.cuh"

namespace btc {

constexpr int kL4Rows = 16, kL4K = 64, kL4Block = 512, kL4Warps = 8;
constexpr int kL4Stretch = 4, kL4Stages = 2;    // k blocks of a stretch, stretches in a warp's ring

struct Linear4Params {
    const unsigned char *packed;
    const void *x;
    const float *xs;
    void *y;
    int64_t x_t, x_k, xs_t, xs_g, y_t, y_n;
    int32_t tokens, k, n;                    // n: columns of y
    int32_t row_blocks, k_blocks;
    int32_t stretch_bytes, head_bytes, zeros_at;           // of a stretch; its scales and zeros; where its zeros are (0: none)
    int32_t group_log2;                      // k per scale, at most a stretch (longer groups repeat theirs)
    int32_t xgroup_log2;                     // e4m3 x: k per scale; 31: one scale per token
    int32_t x_type, y_type, scale_type, activation;        // btc_dtype_t; 0 none, 1 silu, 2 gelu (tanh form)
    int32_t vec_x;                           // 16-byte (e4m3: 8-byte) loads of x
    int32_t wk, chunk;                       // warps that share a row block's k; stretches staged at a time (a multiple of wk)
    int32_t slice;                           // stretches of a CTA: the cluster's CTAs split k
    int32_t staged_bytes;
};

struct Linear4PackParams {
    const unsigned char *codes, *zeros;
    const void *scales;
    unsigned char *out;
    int64_t row_bytes;
    int32_t k, n, row_blocks, stretches, groups, group_log2, row_group_log2;      // row_group_log2: 31 where one scale serves the row
    int32_t scale_bytes, stretch_bytes, head_bytes, zeros_at, gated;
};

// the weight row that row `i` of a block is, or -1 behind the last
__host__ __device__ __forceinline__ int64_t linear4_row(int64_t rb, int i, int32_t n, bool gated)
{
    if (!gated) {
        const int64_t row = rb * kL4Rows + i;
        return row < n ? row : -1;
    }
    const int64_t col = rb * 8 + (i & 7);
    return col < n ? col + (i < 8 ? 0 : int64_t(n)) : -1;
}

// one thread to a lane's 16 bytes of a block, and to a row's scale and zero of a group
static __global__ void linear4_pack_kernel(const __grid_constant__ Linear4PackParams p)
{
    const int per_stretch = kL4Stretch * kL4K >> p.group_log2, threads = kL4Stretch * 32 + per_stretch * kL4Rows;
    const int64_t all = int64_t(p.row_blocks) * p.stretches * threads;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < all; i += int64_t(gridDim.x) * blockDim.x) {
        const int64_t stretch = i / threads, rb = stretch / p.stretches;
        const int at = int(i - stretch * threads), first_k = int(stretch - rb * p.stretches) * (kL4Stretch * kL4K);
        unsigned char *out = p.out + stretch * p.stretch_bytes;
        if (at < kL4Stretch * 32) {
            const int lane = at & 31, g = lane >> 2, q = lane & 3, k0 = first_k + (at >> 5) * kL4K + q * 8;
            const int64_t row[2] = {linear4_row(rb, g, p.n, p.gated), linear4_row(rb, g + 8, p.n, p.gated)};
            uint32_t w[4];
            for (int s = 0; s < 4; ++s) {
                w[s] = 0;
                for (int pair = 0; pair < 4; ++pair)
                    for (int half = 0; half < 2; ++half) {
                        const int k = k0 + (s >> 1) * 32 + (s & 1) * 4 + (pair >> 1) * 2 + half;
                        const int64_t r = row[pair & 1];
                        uint32_t code = 8;
                        if (r >= 0 && k < p.k) code = (p.codes[r * p.row_bytes + (k >> 1)] >> (4 * (k & 1))) & 15u;
                        w[s] |= code << (16 * half + 4 * pair);
                    }
            }
            reinterpret_cast<uint4 *>(out + p.head_bytes)[at] = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            const int j = at - kL4Stretch * 32, r = j & 15, k = first_k + ((j >> 4) << p.group_log2);
            const int64_t row = linear4_row(rb, (r >> 1) + 8 * (r & 1), p.n, p.gated);
            const bool there = row >= 0 && k < p.k;
            const int64_t from = there ? row * p.groups + (k >> p.row_group_log2) : 0;
            if (p.scale_bytes == 4) reinterpret_cast<float *>(out)[j] = there ? static_cast<const float *>(p.scales)[from] : 0.f;
            else reinterpret_cast<unsigned short *>(out)[j] = there ? static_cast<const unsigned short *>(p.scales)[from] : 0;
            if (p.zeros) out[p.zeros_at + j] = there ? (p.zeros[from] & 15) : 8;
        }
    }
}

// The two numbers of each operand register from a word of eight codes, less the rows' zeros (whole numbers: exact).
// f16: 1024 + c and 1024 + 16 c are bit patterns; bf16: 128 + c.
// The mask and the pattern's constant part stay in registers, so that both are one instruction (a constant may stand in it once).
__device__ __forceinline__ uint32_t l4_pick(uint32_t w, uint32_t mask, uint32_t pattern)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "r"(mask), "r"(pattern));      // (w & mask) | pattern
    return r;
}
struct F16Codes {
    typedef __half T;
    uint32_t pattern;
    __device__ __forceinline__ F16Codes() { asm volatile("mov.b32 %0, 0x64006400;" : "=r"(pattern)); }
    __half2 low[2], high[2];                 // 1024 + zero of rows g and g + 8; -(64 + zero)
    __device__ __forceinline__ void zeros(int za, int zb)
    {
        const int z[2] = {za, zb};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lo = uint32_t(z[i]) * 0x10001u | 0x64006400u, hi = uint32_t(z[i]) * 0x100010u | 0xd400d400u;
            low[i] = *reinterpret_cast<const __half2 *>(&lo);
            high[i] = *reinterpret_cast<const __half2 *>(&hi);
        }
    }
    __device__ __forceinline__ void get(uint32_t w, uint32_t (&a)[4]) const
    {
        const __half2 sixteenth = __float2half2_rn(0.0625f);
        const uint32_t v = w >> 8;
        const uint32_t x[4] = {l4_pick(w, 0x000f000fu, pattern), l4_pick(w, 0x00f000f0u, pattern), l4_pick(v, 0x000f000fu, pattern),
                               l4_pick(v, 0x00f000f0u, pattern)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = *reinterpret_cast<const __half2 *>(&x[i]);
            const __half2 y = (i & 1) ? __hfma2(h, sixteenth, high[i & 1]) : __hsub2(h, low[i & 1]);
            a[i] = *reinterpret_cast<const uint32_t *>(&y);
        }
    }
};
struct BF16Codes {
    typedef __nv_bfloat16 T;
    __nv_bfloat162 low[2];
    uint32_t pattern;
    __device__ __forceinline__ BF16Codes() { asm volatile("mov.b32 %0, 0x43004300;" : "=r"(pattern)); }
    __device__ __forceinline__ void zeros(int za, int zb)
    {
        const uint32_t a = uint32_t(za) * 0x10001u | 0x43004300u, b = uint32_t(zb) * 0x10001u | 0x43004300u;
        low[0] = *reinterpret_cast<const __nv_bfloat162 *>(&a);
        low[1] = *reinterpret_cast<const __nv_bfloat162 *>(&b);
    }
    __device__ __forceinline__ void get(uint32_t w, uint32_t (&a)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = l4_pick(w >> (4 * i), 0x000f000fu, pattern);
            const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), low[i & 1]);
            a[i] = *reinterpret_cast<const uint32_t *>(&y);
        }
    }
};

// c = a b (FIRST) or c += a b
#define BTC_L4_MMA(TYPE, T)                                                                                                          \
    template <bool FIRST> __device__ __forceinline__ void l4_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, T)  \
    {                                                                                                                                \
        if constexpr (FIRST)                                                                                                         \
            asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "          \
                "{%10, %10, %10, %10};"                                                                                              \
                : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])                                                                     \
                : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));                                           \
        else                                                                                                                         \
            asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "          \
                "{%0, %1, %2, %3};"                                                                                                  \
                : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])                                                                     \
                : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));                                                     \
    }
BTC_L4_MMA("f16", __half)
BTC_L4_MMA("bf16", __nv_bfloat16)
#undef BTC_L4_MMA

// Eight x values of a token, k to k + 7, as they lie in memory (zeros behind the end)
template <int PARTS> struct Linear4X {
    uint4 raw[PARTS == 3 ? 2 : 1];
    __device__ __forceinline__ void load(const Linear4Params &p, int token, int k)
    {
        const int64_t at = int64_t(token) * p.x_t + int64_t(k) * p.x_k;
        const int left = p.k - k;
        uint32_t w[PARTS == 3 ? 8 : 4];
#pragma unroll
        for (int j = 0; j < (PARTS == 3 ? 8 : 4); ++j) w[j] = 0;
        if constexpr (PARTS == 3) {
            const float *x = static_cast<const float *>(p.x) + at;
            if (p.vec_x && left >= 8) {
                raw[0] = reinterpret_cast<const uint4 *>(x)[0];
                raw[1] = reinterpret_cast<const uint4 *>(x)[1];
                return;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) w[j] = __float_as_uint(x[j * p.x_k]);
            raw[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else if (p.x_type == BTC_E4M3) {
            const unsigned char *x = static_cast<const unsigned char *>(p.x) + at;
            if (p.vec_x && left >= 8) {
                const uint2 v = *reinterpret_cast<const uint2 *>(x);
                raw[0] = make_uint4(v.x, v.y, 0, 0);
                return;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) w[j >> 2] |= uint32_t(x[j * p.x_k]) << (8 * (j & 3));
        } else {
            const unsigned short *x = static_cast<const unsigned short *>(p.x) + at;
            if (p.vec_x && left >= 8) {
                raw[0] = *reinterpret_cast<const uint4 *>(x);
                return;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) w[j >> 1] |= uint32_t(x[j * p.x_k]) << (16 * (j & 1));
        }
        raw[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    // as operand words; fp32: three bf16 parts whose sum is the value (each is the leading 8 bits of what the parts before
    // leave: exact)
    __device__ __forceinline__ void convert(bool e4m3, uint4 (&out)[PARTS]) const
    {
        if constexpr (PARTS == 3) {
            const uint32_t v[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
            uint32_t w[3][4];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float rest = __uint_as_float(v[j]);
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const uint32_t lead = __float_as_uint(rest) & 0xffff0000u;
                    if (j & 1) w[i][j >> 1] |= lead; else w[i][j >> 1] = lead >> 16;
                    rest -= __uint_as_float(lead);
                }
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) out[i] = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        } else if (e4m3) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t((j < 2 ? raw[0].x : raw[0].y) >> (16 * (j & 1))), __NV_E4M3);
                w[j] = uint32_t(h.x) | uint32_t(h.y) << 16;
            }
            out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            out[0] = raw[0];
        }
    }
};

// x of `tokens` tokens from token0 on and `count` stretches of k, in the order in which the lanes take it: [k block][8 tokens]
// [part][half][lane], zeros behind the end of k.  Places of tokens that are not there stay as they are: they reach only columns of
// the product that nobody reads.
// A warp takes a token's stretch at a time, a lane 8 values of it.
template <int PARTS, int NT> __device__ __forceinline__ void l4_stage(const Linear4Params &p, uint4 *staged, int token0, int tokens, int stretch, int count)
{
    const int lane = threadIdx.x & 31;
    // lane 8 kb + 4 half + q of a stretch has k = 64 kb + 32 half + 8 q
    const int in_stretch = ((lane >> 3) * NT * PARTS * 2 + ((lane >> 2) & 1)) * 32 + (lane & 3);
    int token = 0, at = threadIdx.x >> 5;
    auto settle = [&]() {
        while (at >= count && token < tokens) { at -= count; ++token; }
    };
    settle();
    if (PARTS == 1 && p.x_type != BTC_E4M3 && p.vec_x) {
        const unsigned base = unsigned(__cvta_generic_to_shared(staged));
        while (token < tokens) {
            const int k = (stretch + at) * (kL4Stretch * kL4K) + lane * 8, bytes = max(0, min(16, (p.k - k) * 2));
            const unsigned short *x = static_cast<const unsigned short *>(p.x) + (bytes ? int64_t(token0 + token) * p.x_t + k : 0);
            const int to = (at * kL4Stretch * NT + (token >> 3)) * (PARTS * 64) + (token & 7) * 4 + in_stretch;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(base + unsigned(to) * 16u), "l"(x), "r"(bytes) : "memory");
            at += kL4Warps;
            settle();
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    constexpr int BATCH = 4;
    while (token < tokens) {
        Linear4X<PARTS> v[BATCH];
        int to[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            to[j] = -1;
            if (token < tokens) {
                to[j] = (at * kL4Stretch * NT + (token >> 3)) * (PARTS * 64) + (token & 7) * 4 + in_stretch;
                v[j].load(p, token0 + token, (stretch + at) * (kL4Stretch * kL4K) + lane * 8);
                at += kL4Warps;
                settle();
            }
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            if (to[j] < 0) continue;
            uint4 out[PARTS];
            v[j].convert(p.x_type == BTC_E4M3, out);
#pragma unroll
            for (int part = 0; part < PARTS; ++part) staged[to[j] + part * 64] = out[part];
        }
    }
}

__device__ __forceinline__ float l4_activation(float x, int kind)
{
    if (kind == 1) return x / (1.f + expf(-x));
    // 0.5 x (1 + tanh(u)) = x / (1 + exp(-2 u))
    const float u = 0.7978845608028654f * (x + 0.044715f * x * x * x);
    return x / (1.f + expf(-2.f * u));
}

__device__ __forceinline__ void l4_store(const Linear4Params &p, int token, int32_t col, float v)
{
    const int64_t at = int64_t(token) * p.y_t + int64_t(col) * p.y_n;
    if (p.y_type == BTC_F32) static_cast<float *>(p.y)[at] = v;
    else if (p.y_type == BTC_F16) static_cast<__half *>(p.y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(v);
}

// CODES: how codes become numbers; PARTS: parts of an x value; NT: blocks of 8 tokens; SHORT: scales of 32 k, of weights or x.
// A CTA: 8 warps = (8 / wk) row blocks x wk shares of the k of each chunk of x; a cluster's CTAs take consecutive slices of k
// for the same rows and are joined through distributed shared memory, in a fixed order.
// ZEROS: zeros are given; XG: x has scales of its own along k.  (As run-time choices inside the loop these, like the scales' type,
// cut it into pieces that the compiler cannot interleave.)
template <typename CODES, int PARTS, int NT, bool SHORT, bool ZEROS, bool XG>
__global__ void __launch_bounds__(kL4Warps * 32, NT == 1 && PARTS == 1 ? 3 : 2) linear4_kernel(const __grid_constant__ Linear4Params p)
{
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) unsigned char smem[];
    uint4 *staged = reinterpret_cast<uint4 *>(smem);           // [k block][8 tokens][part][half][lane]
    const cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = int(cluster.block_rank()), ranks = int(cluster.num_blocks());
    const int wk = p.wk, wr = kL4Warps / wk, my_k = warp % wk, my_r = warp / wk;
    const int rb = (int(blockIdx.x) / ranks) * wr + my_r;
    const int token0 = int(blockIdx.y) * (8 * NT);
    const int stretches = (p.k_blocks + kL4Stretch - 1) / kL4Stretch;
    const int first = rank * p.slice, count = max(0, min(p.slice, stretches - first));
    const int chunks = (count + p.chunk - 1) / p.chunk, share = p.chunk / wk;         // a warp's stretches of a chunk: share
    unsigned char *ring = smem + p.staged_bytes + warp * (kL4Stages * p.stretch_bytes);
    const unsigned ring_at = unsigned(__cvta_generic_to_shared(ring));
    const unsigned char *from = p.packed + (int64_t(rb < p.row_blocks ? rb : 0) * stretches + first) * p.stretch_bytes;

    early_begin();

    // stretch i of this warp: chunk i / share, there my_k * share + i % share
    int issue_chunk = 0, issue_in = 0, into = 0;
    auto issue = [&]() {
        const int at = issue_chunk * p.chunk + my_k * share + issue_in;
        if (rb < p.row_blocks && issue_chunk < chunks && at < count) {
            const unsigned char *src = from + int64_t(at) * p.stretch_bytes + lane * 16;
            const unsigned dst = ring_at + unsigned(into * p.stretch_bytes + lane * 16);
            static_assert(kL4Stretch * kL4Block == 4 * 512, "");
#pragma unroll
            for (int o = 0; o < 2048; o += 512) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + o), "l"(src + o) : "memory");
#pragma unroll
            for (int o = 2048; o < 2048 + 1024; o += 512)              // a head of at most 640 bytes more
                if (lane * 16 + o < p.stretch_bytes) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + o), "l"(src + o) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++into == kL4Stages) into = 0;
        if (++issue_in == share) { issue_in = 0; ++issue_chunk; }
    };
#pragma unroll
    for (int i = 0; i < kL4Stages - 1; ++i) issue();

    float total[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) total[i][j] = 0.f;
    CODES numbers;
    numbers.zeros(8, 8);
    int slot = 0;
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int chunk_first = first + chunk * p.chunk;        // its first stretch
        if (chunk > 0) __syncthreads();                         // the chunk before is done with
        l4_stage<PARTS, NT>(p, staged, token0, min(8 * NT, p.tokens - token0), chunk_first, min(p.chunk, count - chunk * p.chunk));
        __syncthreads();
        for (int i = 0; i < share; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kL4Stages - 2) : "memory");
            __syncwarp();                                       // every lane's copies have landed, the oldest place is free
            issue();
            const unsigned char *here = ring + slot * p.stretch_bytes;
            if (++slot == kL4Stages) slot = 0;
            const int at = my_k * share + i;                    // in the chunk
            if (rb >= p.row_blocks || chunk * p.chunk + at >= count) continue;
            const uint4 *x = staged + at * (kL4Stretch * NT * PARTS * 64) + lane;
            const uint4 *codes = reinterpret_cast<const uint4 *>(here + p.head_bytes) + lane;
            constexpr int PER = SHORT ? 8 : 4;                  // scales of the stretch, one for each 32 or 64 k
            float2 scale[PER];
            auto at_scale = [&](int j) { return (j * (kL4Stretch * kL4K / PER) >> p.group_log2) * 8 + (lane >> 2); };
            if (p.scale_type == BTC_F32) {
#pragma unroll
                for (int j = 0; j < PER; ++j) scale[j] = reinterpret_cast<const float2 *>(here)[at_scale(j)];
            } else if (p.scale_type == BTC_F16) {
#pragma unroll
                for (int j = 0; j < PER; ++j) unpack_word(reinterpret_cast<const uint32_t *>(here)[at_scale(j)], scale[j].x, scale[j].y, __half());
            } else {
#pragma unroll
                for (int j = 0; j < PER; ++j) unpack_word(reinterpret_cast<const uint32_t *>(here)[at_scale(j)], scale[j].x, scale[j].y, __nv_bfloat16());
            }
#pragma unroll
            for (int kb = 0; kb < kL4Stretch; ++kb) {
                const uint4 c = codes[kb * 32];
                const uint32_t words[4] = {c.x, c.y, c.z, c.w};
                float part[NT][4];
#pragma unroll
                for (int half = 0; half < 2; ++half) {          // two steps to a 16-byte piece of x: 32 k
                    if (ZEROS && (SHORT || half == 0)) {
                        const int g = (kb * kL4K + (SHORT ? 32 * half : 0)) >> p.group_log2;
                        const uint32_t z = reinterpret_cast<const unsigned short *>(here + p.zeros_at)[g * 8 + (lane >> 2)];
                        numbers.zeros(int(z & 15u), int(z >> 8));
                    }
                    uint32_t a[2][4];
                    numbers.get(words[2 * half], a[0]);
                    numbers.get(words[2 * half + 1], a[1]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int q = PARTS - 1; q >= 0; --q) {
                            const uint4 b = x[(kb * NT * PARTS + nt * PARTS + q) * 64 + half * 32];
                            if ((SHORT || half == 0) && q == PARTS - 1) l4_mma<true>(part[nt], a[0], b.x, b.y, typename CODES::T());
                            else l4_mma<false>(part[nt], a[0], b.x, b.y, typename CODES::T());
                            l4_mma<false>(part[nt], a[1], b.z, b.w, typename CODES::T());
                        }
                    if (!SHORT && half == 0) continue;
                    const float2 s = scale[SHORT ? 2 * kb + half : kb];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (XG) {
                            const int k = ((chunk_first + at) * kL4Stretch + kb) * kL4K + (SHORT ? 32 * half : 0), t = token0 + nt * 8 + 2 * (lane & 3);
                            const int64_t xg = int64_t(k >> p.xgroup_log2) * p.xs_g;
                            const float xa = k < p.k && t < p.tokens ? p.xs[t * p.xs_t + xg] : 1.f;
                            const float xb = k < p.k && t + 1 < p.tokens ? p.xs[(t + 1) * p.xs_t + xg] : 1.f;
                            part[nt][0] *= xa; part[nt][1] *= xb; part[nt][2] *= xa; part[nt][3] *= xb;
                        }
                        total[nt][0] = fmaf(part[nt][0], s.x, total[nt][0]);
                        total[nt][1] = fmaf(part[nt][1], s.x, total[nt][1]);
                        total[nt][2] = fmaf(part[nt][2], s.y, total[nt][2]);
                        total[nt][3] = fmaf(part[nt][3], s.y, total[nt][3]);
                    }
                }
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");

    // join: [warp][token][row] of this CTA, then the warps of a row block and the cluster's CTAs
    constexpr int TT = 8 * NT;
    float *sums = reinterpret_cast<float *>(smem);
    __syncthreads();                                            // x is done with
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            sums[(warp * TT + nt * 8 + 2 * (lane & 3) + (j & 1)) * kL4Rows + (lane >> 2) + 8 * (j >> 1)] = total[nt][j];
    if (ranks > 1) cluster.sync(); else __syncthreads();
    const bool gated = p.activation != 0;
    const int per = gated ? 8 : 16, columns = wr * per, outputs = columns * min(TT, p.tokens - token0);
    for (int i = rank * kL4Warps * 32 + tid; i < outputs; i += ranks * kL4Warps * 32) {
        const int t = i / columns, c = i - t * columns, r = c / per, row = c - r * per;
        const int64_t col = (int64_t(int(blockIdx.x) / ranks) * wr + r) * per + row;
        if (col >= p.n) continue;
        float a = 0.f, b = 0.f;
        for (int from = 0; from < ranks; ++from) {
            const float *there_sums = ranks > 1 ? cluster.map_shared_rank(sums, from) : sums;
            for (int w = 0; w < wk; ++w) {
                const float *at = there_sums + ((r * wk + w) * TT + t) * kL4Rows + row;
                a += at[0];
                if (gated) b += at[8];
            }
        }
        if (p.xs && p.xgroup_log2 == 31) {
            const float s = p.xs[int64_t(token0 + t) * p.xs_t];
            a *= s;
            b *= s;
        }
        l4_store(p, token0 + t, int32_t(col), gated ? l4_activation(a, p.activation) * b : a);
    }
    if (ranks > 1) cluster.sync();                              // the others still read this CTA's sums
}

}  // namespace btc
