// The residual's addition and the root-mean-square norm after it, forward and backward.
//
//   h = x + r,   n = h / sqrt(mean(h^2) + eps),   y = n w          (y in x's type, or in 8 bits with scales)
//   dh' = dh + rms^-1 (g - n mean(g n)) with g = dy w;   dx = dr = dh',   dw = sum over the rows of dy n
//
// Bound by HBM: a row is read once into registers, its sum of squares goes through the warp and shared memory, and
// everything that depends on it is written from those registers.  A thread holds `C` chunks of `CH` neighbouring
// elements (16 bytes of x), chunk q = thread + j * threads, so that every access of a warp is contiguous.
// Measured in replayed graphs: 8192 rows of 8192 with the stream in fp32 and an 8-bit result 119 us (740 MB: 6.2 TB/s), 16384 rows of 4096 in
// bf16 forward and backward 175 us (1074 MB: 6.1 TB/s; floor 164), 8192 rows of 4096 with the stream in fp32 173 us (floor 143), 16 rows of 4096
// 2.1 us.  A row has at most 1024 threads and so 64 registers in each: the backward pass of rows over 8192 spills 500 to 730 bytes a thread in 16 bits
// with vectors (2048 rows of 16384 in bf16 with the forward pass 158 us, floor 82) and in fp32 (326 us, floor 164), of long rows of single elements
// 820 to 1010 bytes, rows with the stream in fp32 90.
#pragma once

#include <cuda_fp8.h>

#include "decoder_common.cuh"

namespace btc {

constexpr int kNormMaxDim = 16384;
constexpr int kNormWarpRows = 4;             // rows of a CTA where a warp takes a row

struct AddNormParams {
    const void *x, *r, *w;                   // backward: x is the kept sum
    const void *dy, *dh;
    void *h, *y;                             // backward: h is dr, y is dx
    float *s, *partial;
    int64_t x_t, x_d, r_t, r_d, h_t, h_d, y_t, y_d, s_t, s_g, dy_t, dy_d, dh_t, dh_d;
    int64_t rows;
    int32_t dim, chunks, group;              // group: elements per scale, 0: the row
    float inv_dim, eps;
};

// CH elements as they lie in memory.  CH > 1: contiguous and aligned to the chunk or 16 bytes; CH == 1: any stride
template <typename T, int CH> struct NormChunk {
    static constexpr int WORDS = CH * int(sizeof(T)) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T *row, int64_t, int q)
    {
        const unsigned char *at = reinterpret_cast<const unsigned char *>(row) + size_t(q) * (CH * sizeof(T));
        if constexpr (WORDS >= 4) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const uint4 v = reinterpret_cast<const uint4 *>(at)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else {
            static_assert(WORDS == 2, "");
            const uint2 v = *reinterpret_cast<const uint2 *>(at);
            w[0] = v.x; w[1] = v.y;
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void get(float (&v)[CH]) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) unpack_word(w[i], v[2 * i], v[2 * i + 1], T());
        }
    }
    __device__ __forceinline__ static void store(T *row, int64_t, int q, const float (&v)[CH])
    {
        unsigned char *at = reinterpret_cast<unsigned char *>(row) + size_t(q) * (CH * sizeof(T));
        uint32_t o[WORDS];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < CH; ++i) o[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) o[i] = pack2(v[2 * i], v[2 * i + 1], T());
        }
        if constexpr (WORDS >= 4) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) reinterpret_cast<uint4 *>(at)[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        } else {
            *reinterpret_cast<uint2 *>(at) = make_uint2(o[0], o[1]);
        }
    }
};
template <typename T> struct NormChunk<T, 1> {
    T v0;
    __device__ __forceinline__ void load(const T *row, int64_t stride, int q) { v0 = row[q * stride]; }
    __device__ __forceinline__ void zero() { v0 = from_f32<T>(0.f); }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f32(v0); }
    __device__ __forceinline__ static void store(T *row, int64_t stride, int q, const float (&v)[1]) { row[q * stride] = from_f32<T>(v[0]); }
};

template <int CH> __device__ __forceinline__ void store_e4m3(unsigned char *row, int64_t stride, int q, const float (&v)[CH])
{
    if constexpr (CH == 1) {
        row[q * stride] = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else {
        uint32_t o[CH / 4];
#pragma unroll
        for (int i = 0; i < CH / 4; ++i)
            o[i] = uint32_t(__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3)) |
                   uint32_t(__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3)) << 16;
        if constexpr (CH == 8) *reinterpret_cast<uint2 *>(row + q * 8) = make_uint2(o[0], o[1]);
        else *reinterpret_cast<uint32_t *>(row + q * 4) = o[0];
    }
}

// The scale of a group whose largest modulus has these bits, and its reciprocal.  The scale is a normal number, so that the
// reciprocal is finite; a group that holds an infinity or NaN has the scale NaN and codes of zero.  Both are products with rounded
// reciprocals (1 / 448 and 1 / scale): a unit of fp32 more than divisions would give, 2^-20 of a code's step.
__device__ __forceinline__ void e4m3_scale(uint32_t top, float &scale, float &inv)
{
    const bool finite = top < 0x7f800000u;
    scale = finite ? fmaxf(__uint_as_float(top) * (1.f / 448.f), 1.17549435e-38f) : __uint_as_float(0x7fc00000u);
    inv = finite ? 1.f / scale : 0.f;
}

// Sums (a, b) over the row's threads: a warp, or the CTA through `room` (two rows of one entry per warp that alternate, so that one
// barrier per row is enough: a warp writes to a row again only after the next barrier, which all readers have passed)
template <bool WARP> __device__ __forceinline__ float2 row_sum(float2 v, float2 (*room)[32], int turn)
{
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, k);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, k);
    }
    if constexpr (!WARP) {
        const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0) room[turn][threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < warps ? room[turn][lane] : make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            v.x += __shfl_xor_sync(0xffffffffu, v.x, k);
            v.y += __shfl_xor_sync(0xffffffffu, v.y, k);
        }
    }
    return v;
}

// WARP: a warp to a row, kNormWarpRows rows to a CTA; otherwise a CTA to a row
template <typename TX, typename TR, bool E4M3, int CH, int C, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kNormWarpRows : 1024) add_norm_forward_kernel(const __grid_constant__ AddNormParams p)
{
    __shared__ float2 room[2][32];
    __shared__ uint32_t tops[E4M3 && CH == 1 ? (WARP ? kNormWarpRows : 1) * (C * (WARP ? 32 : 1024) / 32) : 1];
    early_begin();
    const int thread = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x;
    const int64_t row = WARP ? int64_t(blockIdx.x) * kNormWarpRows + (threadIdx.x >> 5) : int64_t(blockIdx.x);
    if (WARP && row >= p.rows) return;
    const TX *x = static_cast<const TX *>(p.x) + row * p.x_t;
    const TR *r = static_cast<const TR *>(p.r) + row * p.r_t;
    NormChunk<TX, CH> raw[C], weight[C];
    NormChunk<TR, CH> rest[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int q = thread + j * threads;
        raw[j].zero();
        rest[j].zero();
        if (q < p.chunks) {
            raw[j].load(x, p.x_d, q);
            if (p.r) rest[j].load(r, p.r_d, q);
        }
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int q = thread + j * threads;
        if (p.w && q < p.chunks) weight[j].load(static_cast<const TX *>(p.w), 1, q);
        else weight[j].zero();
    }
    float v[C][CH];
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int q = thread + j * threads;
        float a[CH];
        raw[j].get(v[j]);
        rest[j].get(a);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (p.r) v[j][i] += a[i];
            sum.x = fmaf(v[j][i], v[j][i], sum.x);
        }
        if (p.h && q < p.chunks) NormChunk<TR, CH>::store(static_cast<TR *>(p.h) + row * p.h_t, p.h_d, q, v[j]);
    }
    sum = row_sum<WARP>(sum, room, 0);
    const float inv = rsqrtf(fmaf(sum.x, p.inv_dim, p.eps));
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        float a[CH];
        weight[j].get(a);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            v[j][i] *= inv;
            if (p.w) v[j][i] *= a[i];
        }
    }
    if constexpr (!E4M3) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int q = thread + j * threads;
            if (q < p.chunks) NormChunk<TX, CH>::store(static_cast<TX *>(p.y) + row * p.y_t, p.y_d, q, v[j]);
        }
    } else {
        unsigned char *y = static_cast<unsigned char *>(p.y) + row * p.y_t;
        float *s = p.s + row * p.s_t;
        uint32_t tj[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            tj[j] = 0;
#pragma unroll
            for (int i = 0; i < CH; ++i) tj[j] = max(tj[j], __float_as_uint(v[j][i]) & 0x7fffffffu);
            if (thread + j * threads >= p.chunks) tj[j] = 0;       // not of the row (0 * inf is NaN)
            top = max(top, tj[j]);
        }
        if (p.group == 0) {
            // one scale per row
            top = __reduce_max_sync(0xffffffffu, top);
            if constexpr (!WARP) {
                uint32_t *out = reinterpret_cast<uint32_t *>(room[1]);
                const int lane = threadIdx.x & 31;
                if (lane == 0) out[threadIdx.x >> 5] = top;
                __syncthreads();
                top = __reduce_max_sync(0xffffffffu, lane < int(blockDim.x >> 5) ? out[lane] : 0u);
            }
            float scale, back;
            e4m3_scale(top, scale, back);
            if (thread == 0) s[0] = scale;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int q = thread + j * threads;
#pragma unroll
                for (int i = 0; i < CH; ++i) v[j][i] = back == 0.f ? 0.f : v[j][i] * back;
                if (q < p.chunks) store_e4m3<CH>(y, p.y_d, q, v[j]);
            }
        } else if constexpr (CH > 1) {
            // a group is group / CH neighbouring lanes (a power of two, at most a warp)
            const int lanes = p.group / CH;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int q = thread + j * threads;
                uint32_t t = tj[j];
                for (int k = 1; k < lanes; k <<= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, k));
                float scale, back;
                e4m3_scale(t, scale, back);
#pragma unroll
                for (int i = 0; i < CH; ++i) v[j][i] = back == 0.f ? 0.f : v[j][i] * back;
                if (q < p.chunks) {
                    store_e4m3<CH>(y, p.y_d, q, v[j]);
                    if ((thread & (lanes - 1)) == 0) s[int64_t(q / lanes) * p.s_g] = scale;
                }
            }
        } else {
            // single elements: maxima of the groups in shared memory (integers: any order gives the same)
            uint32_t *mine = tops + (WARP ? (threadIdx.x >> 5) * C : 0);
            const int groups = (p.dim + p.group - 1) / p.group;
            for (int g = thread; g < groups; g += threads) mine[g] = 0;
            if (WARP) __syncwarp(); else __syncthreads();
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int q = thread + j * threads;
                if (q < p.chunks) atomicMax(mine + q / p.group, tj[j]);
            }
            if (WARP) __syncwarp(); else __syncthreads();
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int q = thread + j * threads;
                if (q >= p.chunks) continue;
                float scale, back;
                e4m3_scale(mine[q / p.group], scale, back);
                v[j][0] = back == 0.f ? 0.f : v[j][0] * back;
                store_e4m3<CH>(y, p.y_d, q, v[j]);
                if (q % p.group == 0) s[int64_t(q / p.group) * p.s_g] = scale;
            }
        }
    }
}

// CTAs that each take every gridDim-th row (WARP: every gridDim-th four): a thread keeps its columns and so its part of dw in
// registers; at the end a CTA writes one row of `partial`.
template <typename TX, typename TR, int CH, int C, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kNormWarpRows : 1024) add_norm_backward_kernel(const __grid_constant__ AddNormParams p)
{
    __shared__ float2 room[2][32];
    __shared__ float joined[WARP ? kNormWarpRows * 32 * C * CH : 1];
    early_begin();
    const int thread = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x;
    const int64_t step = int64_t(gridDim.x) * (WARP ? kNormWarpRows : 1);
    const int64_t begin = WARP ? int64_t(blockIdx.x) * kNormWarpRows + (threadIdx.x >> 5) : int64_t(blockIdx.x);
    NormChunk<TX, CH> weight[C];
    float dw[C][CH];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int q = thread + j * threads;
        weight[j].zero();
        if (p.w && q < p.chunks) weight[j].load(static_cast<const TX *>(p.w), 1, q);
#pragma unroll
        for (int i = 0; i < CH; ++i) dw[j][i] = 0.f;
    }
    NormChunk<TR, CH> kept[C], grad[C];
    NormChunk<TX, CH> dy[C];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int q = thread + j * threads;
            kept[j].zero(); grad[j].zero(); dy[j].zero();
            if (row < p.rows && q < p.chunks) {
                kept[j].load(static_cast<const TR *>(p.x) + row * p.x_t, p.x_d, q);
                dy[j].load(static_cast<const TX *>(p.dy) + row * p.dy_t, p.dy_d, q);
                if (p.dh) grad[j].load(static_cast<const TR *>(p.dh) + row * p.dh_t, p.dh_d, q);
            }
        }
    };
    fetch(begin);
    int turn = 0;
    for (int64_t row = begin; row < p.rows; row += step, turn ^= 1) {
        float h[C][CH], g[C][CH];
        float2 sum = make_float2(0.f, 0.f);
        NormChunk<TR, CH> rest[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float a[CH];
            kept[j].get(h[j]);
            dy[j].get(g[j]);
            weight[j].get(a);
            rest[j] = grad[j];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                sum.x = fmaf(h[j][i], h[j][i], sum.x);
                sum.y = fmaf(p.w ? g[j][i] * a[i] : g[j][i], h[j][i], sum.y);
            }
        }
        fetch(row + step);
        sum = row_sum<WARP>(sum, room, turn);
        const float inv = rsqrtf(fmaf(sum.x, p.inv_dim, p.eps));
        // rms^-1 (g - n mean(g n)), the difference first: rms^-1 squared may be beyond fp32 where the result is not
        const float mean = sum.y * inv * p.inv_dim;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int q = thread + j * threads;
            float a[CH], b[CH], o[CH];
            weight[j].get(a);
            rest[j].get(b);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const float n = h[j][i] * inv;
                dw[j][i] = fmaf(g[j][i], n, dw[j][i]);
                o[i] = fmaf(n, -mean, p.w ? g[j][i] * a[i] : g[j][i]) * inv;
                if (p.dh) o[i] += b[i];
            }
            if (q < p.chunks) {
                if (p.y) NormChunk<TX, CH>::store(static_cast<TX *>(p.y) + row * p.y_t, p.y_d, q, o);
                if (p.h) NormChunk<TR, CH>::store(static_cast<TR *>(p.h) + row * p.h_t, p.h_d, q, o);
            }
        }
    }
    if (!p.partial) return;
    float *out = p.partial + int64_t(blockIdx.x) * p.dim;
    if constexpr (WARP) {
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int i = 0; i < CH; ++i) joined[(threadIdx.x >> 5) * (32 * C * CH) + (thread + j * 32) * CH + i] = dw[j][i];
        __syncthreads();
        for (int d = threadIdx.x; d < p.dim; d += 32 * kNormWarpRows) {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < kNormWarpRows; ++k) t += joined[k * (32 * C * CH) + d];
            out[d] = t;
        }
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int q = thread + j * threads;
            if (q < p.chunks)
#pragma unroll
                for (int i = 0; i < CH; ++i) out[q * CH + i] = dw[j][i];
        }
    }
}

// dw = sum of the CTAs' rows, in a fixed order: 32 columns per block, 32 warps to their rows
static __global__ void __launch_bounds__(1024) add_norm_weight_gradient_kernel(const float *partial, int rows, int dim, float *dw)
{
    __shared__ float tile[32][33];
    early_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float t = 0.f;
    if (col < dim)
#pragma unroll 8
        for (int r = warp; r < rows; r += 32) t += partial[int64_t(r) * dim + col];
    tile[warp][lane] = t;
    __syncthreads();
    t = tile[lane][warp];
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) t += __shfl_xor_sync(0xffffffffu, t, k);
    if (lane == 0 && blockIdx.x * 32 + warp < dim) dw[blockIdx.x * 32 + warp] = t;
}

}  // namespace btc
