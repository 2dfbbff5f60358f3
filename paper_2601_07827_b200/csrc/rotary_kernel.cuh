// Head norm and rotary positions, forward and backward, with the keys and values of the forward pass
// optionally written into cache pages.
//
// With x one head's D values, r = 1 / sqrt(mean(x^2) + eps), n = x r, m = n w, and for each rotated
// pair (a, b) the rotation (y_a, y_b) = mult (m_a cos - m_b sin, m_b cos + m_a sin):
//   backward: dm = the transposed rotation of dy (sin negated), dw = sum over tokens and heads of dm n,
//   g = dm w, dx = r (g - n mean(g n)).
// A pass moves each value once in each direction (forward: x in, y out; backward: x and dy in, dx out)
// and does a few operations per value: it is bound by memory, for a handful of tokens by latency.
//
// Layout.  A value's partner in the rotation and the head's sum of squares must meet, so a head is owned
// by a group of 2^k neighbouring lanes, a lane holding whole pairs: with 16-byte vectors lane c holds
// pairs [c V, (c + 1) V), V = 16 bytes / element, i.e. two vectors (at c V and c V + pairs in the half
// layout, neighbours in the interleaved one), so the rotation needs no exchange and the norm k shuffles.
// The angle's cosine and sine depend on the token and the pair only: a group keeps them in registers
// over the `heads_per_unit` heads that it takes of one token.
// Heads whose sizes, strides or addresses do not allow 16-byte vectors run the same code with one
// element per access, a warp per head, lane l holding pairs l, l + 32, l + 64, l + 96.
#pragma once

#include "../../include/btc.h"
#include "decoder_common.cuh"

namespace btc {

constexpr int kRotaryMaxDim = 256;
constexpr int kRotaryThreads = 256;

struct RotaryPart {
    const void *x;                 // input [T, heads, dim]
    void *y;                       // output, dense or pages; backward: dx (laid out like x)
    const void *dy;                // backward only (laid out like y)
    const void *w;                 // norm weight, or NULL
    int64_t x_t, x_h, x_d;         // element strides
    int64_t y_t, y_h, y_d, y_page; // y_t: per token, or per slot of a page
    int32_t heads, dim;
    int32_t pairs, rest_pairs;     // rotated pairs; pairs of values that are not rotated (the last may lack its second)
    int32_t copy;                  // 1: values pass through unchanged (bit for bit)
    int32_t paged;
    int32_t units;                 // groups of heads per token
};

struct RotaryParams {
    RotaryPart part[3];
    const int32_t *pos, *slots;
    const uint64_t *freq;          // turns per position in units of 2^-64 turn
    int32_t *flags;
    float *partial;                // backward: [CTA][kRotaryMaxDim] sums of dm n of the CTA's part
    int64_t tokens;
    uint32_t units_per_token, heads_per_unit;
    int32_t lanes_log2;            // lanes per head
    int32_t norm;
    float eps, mult;
    FastDiv page;                  // tokens per page
    int32_t slot_count;            // slots in the pool
    uint32_t ctas[2];              // backward: CTAs of the query part / key part
};

// cos and sin of position * frequency.  The product is taken in units of 2^-64 turn modulo one turn, which
// is exact whatever the position; its upper 32 bits are the angle to 2^-33 turn.
__device__ __forceinline__ void rotary_angle(int32_t pos, uint64_t freq, float mult, float &c, float &s)
{
    const int32_t half_turns = int32_t((uint64_t(int64_t(pos)) * freq) >> 32);   // in 2^-31 half turns, [-1, 1)
    sincospif(float(half_turns) * 4.656612873077393e-10f, &s, &c);
    c *= mult;
    s *= mult;
}

// The pairs of one lane: N slots, their element positions, and loads and stores that present slot j as (a[j], b[j]).
template <typename T, bool VECTOR, bool INTERLEAVED> struct RotaryLane {
    static constexpr int V = 16 / int(sizeof(T));
    static constexpr int N = VECTOR ? V : 4;
    struct Raw { uint4 a, b; };
    int ea, eb;                    // VECTOR: element offsets of the two vectors
    bool active, rotated;          // VECTOR: the lane has pairs; they are rotated
    int lane, pairs, rest, dim;

    __device__ __forceinline__ void set(const RotaryPart &p, int lane_in_head)
    {
        lane = lane_in_head;
        pairs = p.pairs; rest = p.rest_pairs; dim = p.dim;
        if (VECTOR) {
            const int first = lane * V;
            active = first < pairs + rest;
            rotated = first < pairs;
            if (INTERLEAVED || !rotated) { ea = 2 * first; eb = ea + V; }
            else { ea = first; eb = first + pairs; }
        }
    }
    __device__ __forceinline__ bool slot_rotated(int j) const { return VECTOR ? rotated : lane + 32 * j < pairs; }
    __device__ __forceinline__ int slot_pair(int j) const { return VECTOR ? lane * V + j : lane + 32 * j; }
    // scalar form: element positions of slot j (dim or more: absent)
    __device__ __forceinline__ void slot_elements(int j, int &a, int &b) const
    {
        const int p = lane + 32 * j;
        if (p < pairs) {
            a = INTERLEAVED ? 2 * p : p;
            b = INTERLEAVED ? a + 1 : p + pairs;
        } else {
            const int q = p - pairs;
            a = q < rest ? 2 * pairs + q : dim;
            b = q < rest ? 2 * pairs + rest + q : dim;
        }
    }
    __device__ __forceinline__ Raw load_raw(const T *row) const
    {
        Raw r;
        r.a = r.b = make_uint4(0, 0, 0, 0);
        if (active) {
            r.a = *reinterpret_cast<const uint4 *>(row + ea);
            r.b = *reinterpret_cast<const uint4 *>(row + eb);
        }
        return r;
    }
    __device__ __forceinline__ void unpack(const Raw &r, float (&a)[N], float (&b)[N]) const
    {
        if constexpr (VECTOR) {
            float u[V], v[V];
            unpack16(r.a, u, T());
            unpack16(r.b, v, T());
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    a[j] = u[2 * j]; b[j] = u[2 * j + 1];
                    a[V / 2 + j] = v[2 * j]; b[V / 2 + j] = v[2 * j + 1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) { a[j] = u[j]; b[j] = v[j]; }
            }
        }
    }
    __device__ __forceinline__ void load(const T *row, int64_t stride, float (&a)[N], float (&b)[N]) const
    {
        if constexpr (VECTOR) {
            unpack(load_raw(row), a, b);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int e, f;
                slot_elements(j, e, f);
                a[j] = e < dim ? to_f32(row[e * stride]) : 0.f;
                b[j] = f < dim ? to_f32(row[f * stride]) : 0.f;
            }
        }
    }
    __device__ __forceinline__ void store(T *row, int64_t stride, const float (&a)[N], const float (&b)[N]) const
    {
        if constexpr (VECTOR) {
            float u[V], v[V];
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    u[2 * j] = a[j]; u[2 * j + 1] = b[j];
                    v[2 * j] = a[V / 2 + j]; v[2 * j + 1] = b[V / 2 + j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) { u[j] = a[j]; v[j] = b[j]; }
            }
            if (active) {
                *reinterpret_cast<uint4 *>(row + ea) = pack16(u, T());
                *reinterpret_cast<uint4 *>(row + eb) = pack16(v, T());
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int e, f;
                slot_elements(j, e, f);
                if (e < dim) row[e * stride] = from_f32<T>(a[j]);
                if (f < dim) row[f * stride] = from_f32<T>(b[j]);
            }
        }
    }
    __device__ __forceinline__ void copy(const T *src, int64_t ss, T *dst, int64_t ds) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            int e, f;
            slot_elements(j, e, f);
            if (e < dim) dst[e * ds] = src[e * ss];
            if (f < dim) dst[f * ds] = src[f * ss];
        }
    }
};

__device__ __forceinline__ float group_sum(float v, int lanes_log2)
{
    for (int k = 0; k < lanes_log2; ++k) v += __shfl_xor_sync(0xffffffffu, v, 1 << k);
    return v;
}

// A group of lanes takes one unit: `heads_per_unit` heads of one part of one token.
template <typename T, bool VECTOR, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryThreads) rotary_forward_kernel(const __grid_constant__ RotaryParams p)
{
    typedef RotaryLane<T, VECTOR, INTERLEAVED> Lane;
    constexpr int N = Lane::N;
    constexpr int FLIGHT = VECTOR ? 4 : 1;      // heads whose loads are issued together
    const int lanes = 1 << p.lanes_log2;
    const int64_t unit = int64_t(blockIdx.x) * (kRotaryThreads >> p.lanes_log2) + (threadIdx.x >> p.lanes_log2);
    int64_t token;
    uint32_t u;
    if (p.tokens * p.units_per_token < (int64_t(1) << 31)) {
        token = uint32_t(unit) / p.units_per_token;
        u = uint32_t(unit) - uint32_t(token) * p.units_per_token;
    } else {
        token = unit / p.units_per_token;
        u = uint32_t(unit - token * p.units_per_token);
    }
    bool valid = token < p.tokens;               // the lanes of a warp stay together for the shuffles
    if (!valid) { token = 0; u = 0; }
    int which = 0;
    while (which < 2 && u >= uint32_t(p.part[which].units)) u -= uint32_t(p.part[which++].units);
    const RotaryPart &part = p.part[which];
    Lane lane;
    lane.set(part, threadIdx.x & (lanes - 1));

    const int first = int(u * p.heads_per_unit);
    const int count = valid ? min(int(p.heads_per_unit), part.heads - first) : 0;
    const T *x = static_cast<const T *>(part.x) + token * part.x_t + first * part.x_h;
    T *y = static_cast<T *>(part.y) + first * part.y_h;
    bool write = valid;
    if (part.paged) {
        const int32_t slot = p.slots[token];
        write = valid && slot >= 0 && slot < p.slot_count;
        if (valid && slot >= p.slot_count && p.flags) atomicOr(p.flags, int(BTC_FLAG_BAD_SLOT));
        const uint32_t at = write ? uint32_t(slot) : 0u, page = p.page.div(at);
        y += int64_t(page) * part.y_page + int64_t(at - page * p.page.d) * part.y_t;
    } else {
        y += token * part.y_t;
    }

    float c[N], s[N], wa[N], wb[N];
    const bool norm = p.norm && !part.copy;
    if (part.pairs > 0) {
        const int32_t pos = p.pos[token];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            c[j] = 1.f;
            s[j] = 0.f;
            if (lane.slot_rotated(j)) rotary_angle(pos, p.freq[lane.slot_pair(j)], p.mult, c[j], s[j]);
        }
    }
    if (norm && part.w) {
        lane.load(static_cast<const T *>(part.w), 1, wa, wb);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) wa[j] = wb[j] = 1.f;
    }

    const uint32_t steps = p.heads_per_unit;     // the same for every lane of the warp
    for (uint32_t h0 = 0; h0 < steps; h0 += FLIGHT) {
        typename Lane::Raw raw[FLIGHT];
        if constexpr (VECTOR) {
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i) {
                raw[i].a = raw[i].b = make_uint4(0, 0, 0, 0);
                if (int(h0) + i < count) raw[i] = lane.load_raw(x + (int64_t(h0) + i) * part.x_h);
            }
        }
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            const int h = int(h0) + i;
            const bool here = h < count;
            T *row = y + int64_t(h) * part.y_h;
            if (part.copy) {
                if (here && write) {
                    if constexpr (VECTOR) {
                        if (lane.active) {
                            *reinterpret_cast<uint4 *>(row + lane.ea) = raw[i].a;
                            *reinterpret_cast<uint4 *>(row + lane.eb) = raw[i].b;
                        }
                    } else {
                        lane.copy(x + int64_t(h) * part.x_h, part.x_d, row, part.y_d);
                    }
                }
            }
            float a[N], b[N];
            if constexpr (VECTOR) {
                lane.unpack(raw[i], a, b);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) a[j] = b[j] = 0.f;
                if (here && !part.copy) lane.load(x + int64_t(h) * part.x_h, part.x_d, a, b);
            }
            if (p.norm) {                         // all lanes: a warp may hold heads of several parts
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < N; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
                ss = group_sum(ss, p.lanes_log2);
                const float r = rsqrtf(ss / float(part.dim) + p.eps);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    a[j] = a[j] * r * wa[j];
                    b[j] = b[j] * r * wb[j];
                }
            }
            if (part.copy || !here || !write) continue;
            if (part.pairs > 0) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (lane.slot_rotated(j)) {
                        const float t = a[j] * c[j] - b[j] * s[j];
                        b[j] = b[j] * c[j] + a[j] * s[j];
                        a[j] = t;
                    }
            }
            lane.store(row, part.y_d, a, b);
        }
    }
}

// Persistent CTAs, each for one part: a thread keeps its pairs (the lane's place in the head never changes) and
// so its share of dw in registers over all units it takes; at the end the CTA's groups are added in shared memory
// in a fixed order and the CTA writes one row of `partial`.
template <typename T, bool VECTOR, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryThreads, 2) rotary_backward_kernel(const __grid_constant__ RotaryParams p)
{
    typedef RotaryLane<T, VECTOR, INTERLEAVED> Lane;
    constexpr int N = Lane::N;
    __shared__ float sums[kRotaryThreads / 32][kRotaryMaxDim];
    const int lanes = 1 << p.lanes_log2;
    const int which = blockIdx.x < p.ctas[0] ? 0 : 1;
    const RotaryPart &part = p.part[which];
    const uint32_t cta = which ? blockIdx.x - p.ctas[0] : blockIdx.x;
    const int groups = kRotaryThreads >> p.lanes_log2;
    Lane lane;
    lane.set(part, threadIdx.x & (lanes - 1));
    float wa[N], wb[N], da[N], db[N];
    if (p.norm && part.w) {
        lane.load(static_cast<const T *>(part.w), 1, wa, wb);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) wa[j] = wb[j] = 1.f;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) da[j] = db[j] = 0.f;

    const int64_t units = p.tokens * part.units;
    const int64_t stride = int64_t(p.ctas[which]) * groups;
    const int64_t begin = int64_t(cta) * groups;         // the CTA's first unit; its warps take the same number of steps
    for (int64_t base = begin; base < units; base += stride) {
        int64_t unit = base + (threadIdx.x >> p.lanes_log2);
        const bool valid = unit < units;
        if (!valid) unit = 0;
        int64_t token;
        if (units < (int64_t(1) << 32)) token = uint32_t(unit) / uint32_t(part.units);
        else token = unit / part.units;
        const int first = int(unit - token * part.units) * int(p.heads_per_unit);
        const int count = valid ? min(int(p.heads_per_unit), part.heads - first) : 0;
        const T *x = static_cast<const T *>(part.x) + token * part.x_t + first * part.x_h;
        T *dx = static_cast<T *>(part.y) + token * part.x_t + first * part.x_h;
        const T *dy = static_cast<const T *>(part.dy) + token * part.y_t + first * part.y_h;
        float c[N], s[N];
        if (part.pairs > 0) {
            const int32_t pos = p.pos[token];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                c[j] = 1.f;
                s[j] = 0.f;
                if (lane.slot_rotated(j)) rotary_angle(pos, p.freq[lane.slot_pair(j)], p.mult, c[j], s[j]);
            }
        }
        for (uint32_t h0 = 0; h0 < p.heads_per_unit; h0 += 2) {
            constexpr int FLIGHT = VECTOR ? 2 : 1;
            typename Lane::Raw rx[FLIGHT], rg[FLIGHT];
            if constexpr (VECTOR) {
#pragma unroll
                for (int i = 0; i < FLIGHT; ++i) {
                    rx[i].a = rx[i].b = rg[i].a = rg[i].b = make_uint4(0, 0, 0, 0);
                    if (int(h0) + i < count) {
                        rg[i] = lane.load_raw(dy + (int64_t(h0) + i) * part.y_h);
                        if (p.norm) rx[i] = lane.load_raw(x + (int64_t(h0) + i) * part.x_h);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int h = int(h0) + i;
                const bool here = h < count;
                float ga[N], gb[N], a[N], b[N];
                if constexpr (VECTOR) {
                    lane.unpack(rg[i], ga, gb);
                    if (p.norm) lane.unpack(rx[i], a, b);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) a[j] = b[j] = ga[j] = gb[j] = 0.f;
                    if (here) {
                        lane.load(dy + int64_t(h) * part.y_h, part.y_d, ga, gb);
                        if (p.norm) lane.load(x + int64_t(h) * part.x_h, part.x_d, a, b);
                    }
                }
                if (part.pairs > 0) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (lane.slot_rotated(j)) {
                            const float t = ga[j] * c[j] + gb[j] * s[j];
                            gb[j] = gb[j] * c[j] - ga[j] * s[j];
                            ga[j] = t;
                        }
                }
                if (p.norm) {
                    float ss = 0.f, dot = 0.f;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
                        dot = fmaf(ga[j] * wa[j], a[j], fmaf(gb[j] * wb[j], b[j], dot));
                    }
                    ss = group_sum(ss, p.lanes_log2);
                    dot = group_sum(dot, p.lanes_log2);
                    const float r = rsqrtf(ss / float(part.dim) + p.eps);
                    const float mean = dot * r / float(part.dim);    // mean(g n)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float na = a[j] * r, nb = b[j] * r;
                        if (here) {
                            da[j] = fmaf(ga[j], na, da[j]);
                            db[j] = fmaf(gb[j], nb, db[j]);
                        }
                        ga[j] = r * (ga[j] * wa[j] - na * mean);
                        gb[j] = r * (gb[j] * wb[j] - nb * mean);
                    }
                }
                if (here) lane.store(dx + int64_t(h) * part.x_h, part.x_d, ga, gb);
            }
        }
    }
    if (!p.norm || !p.partial) return;
    // the warp's groups hold the same pairs: add them, then the warps
    for (int k = p.lanes_log2; k < 5; ++k) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            da[j] += __shfl_xor_sync(0xffffffffu, da[j], 1 << k);
            db[j] += __shfl_xor_sync(0xffffffffu, db[j], 1 << k);
        }
    }
    const int warp = threadIdx.x >> 5, l = threadIdx.x & 31;
    if (l < lanes) {
        if constexpr (VECTOR) {
            if (lane.active) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int ia = !INTERLEAVED ? lane.ea + j : (j < N / 2 ? lane.ea + 2 * j : lane.eb + 2 * (j - N / 2));
                    const int ib = !INTERLEAVED ? lane.eb + j : ia + 1;
                    sums[warp][ia] = da[j];
                    sums[warp][ib] = db[j];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int e, f;
                lane.slot_elements(j, e, f);
                if (e < part.dim) sums[warp][e] = da[j];
                if (f < part.dim) sums[warp][f] = db[j];
            }
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < part.dim; d += kRotaryThreads) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < kRotaryThreads / 32; ++i) t += sums[i][d];
        p.partial[int64_t(blockIdx.x) * kRotaryMaxDim + d] = t;
    }
}

// dw = sum of the CTAs' rows, in a fixed order: 32 columns per block, 32 lanes of rows each
__global__ void __launch_bounds__(1024) rotary_weight_gradient_kernel(const float *partial, int rows_q, int rows_k, int dim,
                                                                      float *dwq, float *dwk)
{
    __shared__ float tile[32][33];
    const int which = blockIdx.y;
    float *dw = which ? dwk : dwq;
    if (!dw) return;
    const int rows = which ? rows_k : rows_q, first = which ? rows_q : 0;
    const int col = blockIdx.x * 32 + (threadIdx.x & 31);
    float t = 0.f;
    if (col < dim)
        for (int r = threadIdx.x >> 5; r < rows; r += 32) t += partial[int64_t(first + r) * kRotaryMaxDim + col];
    tile[threadIdx.x >> 5][threadIdx.x & 31] = t;
    __syncthreads();
    t = tile[threadIdx.x & 31][threadIdx.x >> 5];
    for (int k = 1; k < 32; k <<= 1) t += __shfl_xor_sync(0xffffffffu, t, k);
    const int out = blockIdx.x * 32 + (threadIdx.x >> 5);
    if ((threadIdx.x & 31) == 0 && out < dim) dw[out] = t;
}

}  // namespace btc
