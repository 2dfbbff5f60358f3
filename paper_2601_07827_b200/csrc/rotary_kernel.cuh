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
// by a group of 2^k neighbouring lanes, a lane holding whole pairs: with vectors of V elements lane c holds
// pairs [c V, (c + 1) V), i.e. two vectors (at c V and c V + pairs in the half layout, neighbours in the
// interleaved one), so the rotation needs no exchange and the norm k shuffles.  Vectors are 16 bytes where
// sizes, strides and addresses allow, else 8; what allows neither runs the same code with one element per
// access, a warp per head, lane l holding pairs l, l + 32, l + 64, l + 96.
// The angles depend on token and pair only: a CTA takes a few tokens with all their heads and computes each
// angle once, into shared memory (computed by every group for itself they were a quarter of all instructions).
// Measured (replayed graphs): 16384 tokens x 80 heads of 128 appended to pages (f16, 671 MB) 110 us = 6.1 TB/s; 16384 x 40 heads
// with norm, bf16: forward 65 us (336 MB), backward 110 us (503 MB), both held up by their instructions (67 % and 63 % of
// the issue slots); 128 x 48 heads appended 3.2 us.
#pragma once

#include "../../include/btc.h"
#include "decoder_common.cuh"

namespace btc {

constexpr int kRotaryMaxDim = 256;
constexpr int kRotaryThreads = 256;
constexpr int kRotaryMaxTokens = 32;     // tokens a CTA takes at a time

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
    float inv_dim;
    uint32_t ctas;                 // CTAs of the part, tokens a CTA takes at a time
    int32_t cta_tokens;
    FastDiv head;                  // heads
};

struct RotaryParams {
    RotaryPart part[3];
    const int32_t *pos, *slots;
    const uint64_t *freq;          // turns per position in units of 2^-64 turn
    int32_t *flags;
    float *partial;                // backward: [CTA][kRotaryMaxDim] sums of dm n of the CTA's part
    int64_t tokens;
    int32_t pairs;                 // of queries and keys
    int32_t lanes_log2;            // lanes per head
    int32_t norm;
    float eps, mult;
    FastDiv page;                  // tokens per page
    int32_t slot_count;            // slots in the pool
    FastDiv pair;                  // pairs
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

// Where a CTA keeps the angles of its tokens: with vectors in the order in which the lanes' 16-byte (or 8-byte) reads
// are neighbours.  V = 1: one element per access.
template <int V> __device__ __forceinline__ int angle_place(int pair)
{
    constexpr int Q = V >= 4 ? 4 : V;
    if (V <= 4) return pair;
    const int chunk = pair / V, j = pair % V;
    return (j / Q) * (kRotaryMaxDim / 2 / V * Q) + chunk * Q + j % Q;
}
template <int V>
__device__ __forceinline__ void angles_to_shared(const RotaryParams &p, int64_t first, int tokens, float *c, float *s)
{
    for (int e = threadIdx.x; e < tokens * p.pairs; e += kRotaryThreads) {
        const int t = int(p.pair.div(uint32_t(e))), i = e - t * p.pairs;
        float x, y;
        rotary_angle(p.pos[first + t], p.freq[i], p.mult, x, y);
        const int at = t * (kRotaryMaxDim / 2) + angle_place<V>(i);
        c[at] = x;
        s[at] = y;
    }
}

// The pairs of one lane: N slots, their element positions, and loads and stores that present slot j as (a[j], b[j]).
// V: elements per access (1: the scalar form).
template <typename T, int V, bool INTERLEAVED> struct RotaryLane {
    static constexpr bool VECTOR = V > 1;
    static constexpr int N = VECTOR ? V : 4;
    typedef typename VectorOf<VECTOR ? V * int(sizeof(T)) : 16>::type Vec;
    struct Raw { Vec a, b; };
    __device__ __forceinline__ static Raw no_raw()     // zeros
    {
        Raw r;
        r.a = r.b = Vec{};
        return r;
    }
    int ea, eb;                    // VECTOR: element offsets of the two vectors
    uint32_t oa, ob;               // the same in bytes
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
            if (!active) ea = eb = 0;      // reads what is there, counts for nothing
            oa = uint32_t(ea) * uint32_t(sizeof(T));
            ob = uint32_t(eb) * uint32_t(sizeof(T));
        }
    }
    __device__ __forceinline__ bool slot_rotated(int j) const { return VECTOR ? rotated : lane + 32 * j < pairs; }
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
    // `base` is the same in the whole CTA and the offset of the head (bytes) has 32 bits, so that an access needs one add
    __device__ __forceinline__ Raw load_raw(const void *base, uint32_t off = 0) const
    {
        Raw r;
        r.a = *reinterpret_cast<const Vec *>(static_cast<const char *>(base) + (off + oa));
        r.b = *reinterpret_cast<const Vec *>(static_cast<const char *>(base) + (off + ob));
        return r;
    }
    // a lane's share of a sum over the head
    __device__ __forceinline__ float share(float2 v) const { return !VECTOR || active ? v.x + v.y : 0.f; }
    __device__ __forceinline__ void store_raw(void *base, uint32_t off, const Raw &r) const
    {
        if (active) {
            *reinterpret_cast<Vec *>(static_cast<char *>(base) + (off + oa)) = r.a;
            *reinterpret_cast<Vec *>(static_cast<char *>(base) + (off + ob)) = r.b;
        }
    }
    // slots 2i and 2i + 1 are the halves of a[i] and b[i]
    static constexpr int N2 = N / 2;
    __device__ __forceinline__ void unpack(const Raw &r, float2 (&a)[N2], float2 (&b)[N2]) const
    {
        if constexpr (VECTOR) {
            float u[V], v[V];
            unpack_vector<T, V>(r.a, u);
            unpack_vector<T, V>(r.b, v);
            auto from = [&](int e) { return e < V ? u[e] : v[e - V]; };
#pragma unroll
            for (int i = 0; i < N2; ++i) {
                if (INTERLEAVED) {
                    a[i] = make_float2(from(4 * i), from(4 * i + 2));
                    b[i] = make_float2(from(4 * i + 1), from(4 * i + 3));
                } else {
                    a[i] = make_float2(u[2 * i], u[2 * i + 1]);
                    b[i] = make_float2(v[2 * i], v[2 * i + 1]);
                }
            }
        }
    }
    __device__ __forceinline__ void load(const T *row, int64_t stride, float2 (&a)[N2], float2 (&b)[N2]) const
    {
        if constexpr (VECTOR) {
            unpack(load_raw(row), a, b);
        } else {
            float x[N], y[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int e, f;
                slot_elements(j, e, f);
                x[j] = e < dim ? to_f32(row[e * stride]) : 0.f;
                y[j] = f < dim ? to_f32(row[f * stride]) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < N2; ++i) {
                a[i] = make_float2(x[2 * i], x[2 * i + 1]);
                b[i] = make_float2(y[2 * i], y[2 * i + 1]);
            }
        }
    }
    template <typename Off>
    __device__ __forceinline__ void store(T *base, Off off, int64_t stride, const float2 (&a)[N2], const float2 (&b)[N2]) const
    {
        if constexpr (VECTOR) {
            float u[V], v[V];
            auto into = [&](int e) -> float & { return e < V ? u[e] : v[e - V]; };
#pragma unroll
            for (int i = 0; i < N2; ++i) {
                if (INTERLEAVED) {
                    into(4 * i) = a[i].x; into(4 * i + 2) = a[i].y;
                    into(4 * i + 1) = b[i].x; into(4 * i + 3) = b[i].y;
                } else {
                    u[2 * i] = a[i].x; u[2 * i + 1] = a[i].y;
                    v[2 * i] = b[i].x; v[2 * i + 1] = b[i].y;
                }
            }
            Raw r;
            r.a = pack_vector<T, V>(u);
            r.b = pack_vector<T, V>(v);
            store_raw(base, off, r);
        } else {
            T *row = base + off;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int e, f;
                slot_elements(j, e, f);
                if (e < dim) row[e * stride] = from_f32<T>(j & 1 ? a[j / 2].y : a[j / 2].x);
                if (f < dim) row[f * stride] = from_f32<T>(j & 1 ? b[j / 2].y : b[j / 2].x);
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
    // (a, b) <- (a c - b s, b c + a s) with a token's angles on the rotated slots; BACK: the transposed rotation
    // (FULL: every slot of every head is rotated, nothing is asked)
    template <bool BACK, bool FULL>
    __device__ __forceinline__ void rotate(const float *cosines, const float *sines, float2 (&a)[N2], float2 (&b)[N2]) const
    {
        float2 c[N2], s[N2];
        if constexpr (VECTOR) {
            constexpr int Q = V >= 4 ? 4 : V;
            typedef typename VectorOf<Q * 4>::type Angles;
            if (!FULL && !rotated) return;
#pragma unroll
            for (int i = 0; i < V / Q; ++i) {
                const int at = i * (kRotaryMaxDim / 2 / V * Q) + lane * Q;
                float x[Q], y[Q];
                unpack_vector<float, Q>(*reinterpret_cast<const Angles *>(cosines + at), x);
                unpack_vector<float, Q>(*reinterpret_cast<const Angles *>(sines + at), y);
#pragma unroll
                for (int j = 0; j < Q / 2; ++j) {
                    c[i * Q / 2 + j] = make_float2(x[2 * j], x[2 * j + 1]);
                    s[i * Q / 2 + j] = make_float2(y[2 * j], y[2 * j + 1]);
                }
            }
        } else {
            // slots that are not rotated: the identity would still mix an infinite partner in (0 * inf), so they are put back
#pragma unroll
            for (int i = 0; i < N2; ++i) {
                const int p0 = slot_rotated(2 * i) ? lane + 64 * i : 0, p1 = slot_rotated(2 * i + 1) ? lane + 64 * i + 32 : 0;
                c[i] = make_float2(cosines[p0], cosines[p1]);
                s[i] = make_float2(sines[p0], sines[p1]);
            }
        }
#pragma unroll
        for (int i = 0; i < N2; ++i) {
            const float2 minus = make_float2(-s[i].x, -s[i].y);
            const float2 x = fma2(b[i], BACK ? s[i] : minus, mul2(a[i], c[i])), y = fma2(a[i], BACK ? minus : s[i], mul2(b[i], c[i]));
            if constexpr (VECTOR) {
                a[i] = x;
                b[i] = y;
            } else {
                if (slot_rotated(2 * i)) { a[i].x = x.x; b[i].x = y.x; }
                if (slot_rotated(2 * i + 1)) { a[i].y = x.y; b[i].y = y.y; }
            }
        }
    }
};

// sum over the lanes of a head; the same number of steps in the whole launch
__device__ __forceinline__ float group_sum(float v, int lanes_log2)
{
    if (lanes_log2 >= 4) {
        if (lanes_log2 == 5) v += __shfl_xor_sync(0xffffffffu, v, 16);
        v += __shfl_xor_sync(0xffffffffu, v, 8);
    }
    if (lanes_log2 >= 3) v += __shfl_xor_sync(0xffffffffu, v, 4);
    if (lanes_log2 >= 2) v += __shfl_xor_sync(0xffffffffu, v, 2);
    if (lanes_log2 >= 1) v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v;
}

// Offsets inside what a CTA takes at a time: the vector forms have them in bytes and 32 bits (the host checks that
// strides are not negative and that they fit), the scalar form in elements and 64 bits
template <typename T, int V> struct RotaryOffset {
    typedef uint32_t type;
    static constexpr int SCALE = int(sizeof(T));
};
template <typename T> struct RotaryOffset<T, 1> {
    typedef int64_t type;
    static constexpr int SCALE = 1;
};

// A CTA takes `cta_tokens` tokens of one part (queries, keys or values); its groups of lanes take the (token, head)
// pairs in turn, the next one's loads issued before the present one is computed.
template <typename T, int V, bool INTERLEAVED, bool FULL>
__global__ void __launch_bounds__(kRotaryThreads, 3) rotary_forward_kernel(const __grid_constant__ RotaryParams p)
{
    typedef RotaryLane<T, V, INTERLEAVED> Lane;
    constexpr int N2 = Lane::N2;
    early_begin();
    __shared__ __align__(16) float cosines[kRotaryMaxTokens * kRotaryMaxDim / 2], sines[kRotaryMaxTokens * kRotaryMaxDim / 2];
    const int lanes = 1 << p.lanes_log2, groups = kRotaryThreads >> p.lanes_log2, group = threadIdx.x >> p.lanes_log2;
    uint32_t cta = blockIdx.x;
    int which = 0;
    while (which < 2 && cta >= p.part[which].ctas) cta -= p.part[which++].ctas;
    const RotaryPart &part = p.part[which];
    const int64_t first = int64_t(cta) * part.cta_tokens;
    const int tokens = int(min(int64_t(part.cta_tokens), p.tokens - first)), heads = part.heads, items = tokens * heads;
    const bool norm = p.norm && !part.copy, turning = part.pairs > 0;
    typedef typename RotaryOffset<T, V>::type Off;
    constexpr int SCALE = RotaryOffset<T, V>::SCALE;
    const Off x_t = Off(part.x_t * SCALE), x_h = Off(part.x_h * SCALE), y_t = Off(part.y_t * SCALE), y_h = Off(part.y_h * SCALE);
    const T *x0 = static_cast<const T *>(part.x) + first * part.x_t;
    T *y0 = static_cast<T *>(part.y) + (part.paged ? 0 : first * part.y_t);
    const FastDiv by_heads = part.head;
    const float inv_dim = part.inv_dim;
    const bool copy = part.copy, paged = part.paged;
    Lane lane;
    lane.set(part, threadIdx.x & (lanes - 1));
    float2 wa[N2], wb[N2];
    // the (token, head) pair number `item`; past the end: the last one again, which is not stored
    auto place = [&](int item, int &token, int &head) {
        item = min(item, items - 1);
        token = int(by_heads.div(uint32_t(item)));
        head = item - token * heads;
    };
    int token, head;
    place(group, token, head);
    typename Lane::Raw ahead;
    if constexpr (V > 1) ahead = lane.load_raw(x0, token * x_t + head * x_h);
    // while the first loads are under way
#pragma unroll
    for (int j = 0; j < N2; ++j) wa[j] = wb[j] = both(1.f);
    if (norm && part.w) lane.load(static_cast<const T *>(part.w), 1, wa, wb);
    if (turning) {
        angles_to_shared<V>(p, first, tokens, cosines, sines);
        __syncthreads();
    }
#pragma unroll 2
    for (int item = group; item < items + group; item += groups) {      // the same steps in every lane: shuffles follow
        const typename Lane::Raw raw = ahead;
        int next_token, next_head;
        place(item + groups, next_token, next_head);
        if constexpr (V > 1) ahead = lane.load_raw(x0, next_token * x_t + next_head * x_h);
        float2 a[N2], b[N2];
        if constexpr (V > 1) lane.unpack(raw, a, b);
        else lane.load(x0 + (token * x_t + head * x_h), part.x_d, a, b);
        if (norm) {
            float2 squares = both(0.f);
#pragma unroll
            for (int j = 0; j < N2; ++j) squares = fma2(a[j], a[j], fma2(b[j], b[j], squares));
            const float ss = group_sum(lane.share(squares), p.lanes_log2);
            const float2 r = both(rsqrtf(fmaf(ss, inv_dim, p.eps)));
#pragma unroll
            for (int j = 0; j < N2; ++j) {
                a[j] = mul2(mul2(a[j], r), wa[j]);
                b[j] = mul2(mul2(b[j], r), wb[j]);
            }
        }
        bool store = item < items;
        T *dst = y0;
        Off at_y = head * y_h;
        if (paged) {
            const int32_t slot = p.slots[first + token];
            if (slot >= p.slot_count && p.flags) atomicOr(p.flags, int(BTC_FLAG_BAD_SLOT));
            store = store && slot >= 0 && slot < p.slot_count;
            const uint32_t at = store ? uint32_t(slot) : 0u, page = p.page.div(at);
            dst += int64_t(page) * part.y_page + int64_t(at - page * p.page.d) * part.y_t;
        } else {
            at_y += token * y_t;
        }
        if (copy) {
            if (store) {
                if constexpr (V > 1) lane.store_raw(dst, at_y, raw);
                else lane.copy(x0 + (token * x_t + head * x_h), part.x_d, dst + at_y, part.y_d);
            }
        } else {
            if (turning) lane.template rotate<false, FULL>(cosines + token * (kRotaryMaxDim / 2), sines + token * (kRotaryMaxDim / 2), a, b);
            if (store) lane.store(dst, at_y, part.y_d, a, b);
        }
        token = next_token;
        head = next_head;
    }
}

// Persistent CTAs, each for one part, `cta_tokens` tokens at a time: a thread keeps its pairs (the lane's place in the
// head never changes) and so its share of dw in registers over everything it takes; at the end the CTA's groups are
// added in shared memory in a fixed order and the CTA writes one row of `partial`.
template <typename T, int V, bool INTERLEAVED, bool FULL>
__global__ void __launch_bounds__(kRotaryThreads, 2) rotary_backward_kernel(const __grid_constant__ RotaryParams p)
{
    typedef RotaryLane<T, V, INTERLEAVED> Lane;
    constexpr int N = Lane::N, N2 = Lane::N2;
    __shared__ __align__(16) float cosines[kRotaryMaxTokens * kRotaryMaxDim / 2], sines[kRotaryMaxTokens * kRotaryMaxDim / 2];
    __shared__ float sums[kRotaryThreads / 32][kRotaryMaxDim];
    early_begin();
    const int lanes = 1 << p.lanes_log2, groups = kRotaryThreads >> p.lanes_log2, group = threadIdx.x >> p.lanes_log2;
    const int which = blockIdx.x < p.part[0].ctas ? 0 : 1;
    const RotaryPart &part = p.part[which];
    const uint32_t cta = which ? blockIdx.x - p.part[0].ctas : blockIdx.x;
    typedef typename RotaryOffset<T, V>::type Off;
    constexpr int SCALE = RotaryOffset<T, V>::SCALE;
    const int heads = part.heads;
    const Off x_t = Off(part.x_t * SCALE), x_h = Off(part.x_h * SCALE), y_t = Off(part.y_t * SCALE), y_h = Off(part.y_h * SCALE);
    const FastDiv by_heads = part.head;
    const float inv_dim = part.inv_dim;
    const bool turning = p.pairs > 0, norm = p.norm;
    Lane lane;
    lane.set(part, threadIdx.x & (lanes - 1));
    float2 wa[N2], wb[N2], da2[N2], db2[N2];
#pragma unroll
    for (int j = 0; j < N2; ++j) {
        wa[j] = wb[j] = both(1.f);
        da2[j] = db2[j] = both(0.f);
    }
    if (p.norm && part.w) lane.load(static_cast<const T *>(part.w), 1, wa, wb);

    for (int64_t first = int64_t(cta) * part.cta_tokens; first < p.tokens; first += int64_t(part.ctas) * part.cta_tokens) {
        const int tokens = int(min(int64_t(part.cta_tokens), p.tokens - first)), items = tokens * heads;
        const T *x0 = static_cast<const T *>(part.x) + first * part.x_t, *g0 = static_cast<const T *>(part.dy) + first * part.y_t;
        T *d0 = static_cast<T *>(part.y) + first * part.x_t;
        // where the (token, head) pair number `item` lies.  Past the end: the last one again, whose dy is not read (dx may be
        // the same memory and written by now) and whose sums are left out, not multiplied by zero: an infinity would stay
        auto place = [&](int item, int &token, Off &at_x, Off &at_y) {
            item = min(item, items - 1);
            token = int(by_heads.div(uint32_t(item)));
            const int head = item - token * heads;
            at_x = token * x_t + head * x_h;
            at_y = token * y_t + head * y_h;
        };
        int token;
        Off at_x, at_y;
        place(group, token, at_x, at_y);
        typename Lane::Raw ahead_x, ahead_g;
        if constexpr (V > 1) {
            ahead_g = Lane::no_raw();
            if (group < items) ahead_g = lane.load_raw(g0, at_y);
            if (norm) ahead_x = lane.load_raw(x0, at_x);
        }
        if (turning) {
            __syncthreads();                                            // the tokens before are done with
            angles_to_shared<V>(p, first, tokens, cosines, sines);
            __syncthreads();
        }
#pragma unroll 2
        for (int item = group; item < items + group; item += groups) {
            const typename Lane::Raw rx = ahead_x, rg = ahead_g;
            int next_token;
            Off next_x, next_y;
            place(item + groups, next_token, next_x, next_y);
            if constexpr (V > 1) {
                if (item + groups < items) {                            // past the end both stay as they are
                    ahead_g = lane.load_raw(g0, next_y);
                    if (norm) ahead_x = lane.load_raw(x0, next_x);
                }
            }
            float2 ga[N2], gb[N2], a[N2], b[N2];
            if constexpr (V > 1) {
                lane.unpack(rg, ga, gb);
                if (norm) lane.unpack(rx, a, b);
            } else {
#pragma unroll
                for (int j = 0; j < N2; ++j) ga[j] = gb[j] = both(0.f);
                if (item < items) lane.load(g0 + at_y, part.y_d, ga, gb);
                if (norm) lane.load(x0 + at_x, part.x_d, a, b);
            }
            if (turning) lane.template rotate<true, FULL>(cosines + token * (kRotaryMaxDim / 2), sines + token * (kRotaryMaxDim / 2), ga, gb);
            if (norm) {
                // with g = dm w:  dx = r (g - x r^2 mean(g x)),  dw += dm x r
                float2 squares = both(0.f), dots = both(0.f), pa[N2], pb[N2];
#pragma unroll
                for (int j = 0; j < N2; ++j) {
                    squares = fma2(a[j], a[j], fma2(b[j], b[j], squares));
                    pa[j] = mul2(ga[j], wa[j]);
                    pb[j] = mul2(gb[j], wb[j]);
                    dots = fma2(pa[j], a[j], fma2(pb[j], b[j], dots));
                }
                const float ss = group_sum(lane.share(squares), p.lanes_log2), dot = group_sum(lane.share(dots), p.lanes_log2);
                const float r = rsqrtf(fmaf(ss, inv_dim, p.eps));
                const float2 r2 = both(r), pull = both(-(dot * r * inv_dim) * r * r);          // x pull = -n r mean(g n)
                const bool counts = item < items;
#pragma unroll
                for (int j = 0; j < N2; ++j) {
                    if (counts) {
                        da2[j] = fma2(ga[j], mul2(a[j], r2), da2[j]);
                        db2[j] = fma2(gb[j], mul2(b[j], r2), db2[j]);
                    }
                    ga[j] = fma2(pa[j], r2, mul2(a[j], pull));
                    gb[j] = fma2(pb[j], r2, mul2(b[j], pull));
                }
            }
            if (item < items) lane.store(d0, at_x, part.x_d, ga, gb);
            token = next_token;
            at_x = next_x;
            at_y = next_y;
        }
    }
    if (!p.norm || !p.partial) return;
    float da[N], db[N];
#pragma unroll
    for (int j = 0; j < N2; ++j) {
        da[2 * j] = da2[j].x; da[2 * j + 1] = da2[j].y;
        db[2 * j] = db2[j].x; db[2 * j + 1] = db2[j].y;
    }
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
        if constexpr (V > 1) {
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

// dw = sum of the CTAs' rows, in a fixed order: 8 columns per block, 128 threads to a column's rows
constexpr int kRotaryGradColumns = 8, kRotaryGradThreads = 1024;
static __global__ void __launch_bounds__(kRotaryGradThreads) rotary_weight_gradient_kernel(const float *partial, int rows_q, int rows_k, int dim,
                                                                                         float *dwq, float *dwk)
{
    __shared__ float tile[kRotaryGradThreads / 32][kRotaryGradColumns];
    early_begin();
    const int which = blockIdx.y;
    float *dw = which ? dwk : dwq;
    if (!dw) return;
    const int rows = which ? rows_k : rows_q, first = which ? rows_q : 0;
    const int col = blockIdx.x * kRotaryGradColumns + (threadIdx.x % kRotaryGradColumns);
    float t = 0.f;
    if (col < dim)
#pragma unroll 4
        for (int r = threadIdx.x / kRotaryGradColumns; r < rows; r += kRotaryGradThreads / kRotaryGradColumns)
            t += partial[int64_t(first + r) * kRotaryMaxDim + col];
    // the warp's 4 rows of threads, then the warps
    t += __shfl_xor_sync(0xffffffffu, t, 8);
    t += __shfl_xor_sync(0xffffffffu, t, 16);
    if ((threadIdx.x & 31) < kRotaryGradColumns) tile[threadIdx.x / 32][threadIdx.x & 31] = t;
    __syncthreads();
    const int warp = threadIdx.x / 32;
    if (warp >= kRotaryGradColumns) return;
    t = tile[threadIdx.x & 31][warp];
    for (int k = 1; k < 32; k <<= 1) t += __shfl_xor_sync(0xffffffffu, t, k);
    const int out = blockIdx.x * kRotaryGradColumns + warp;
    if ((threadIdx.x & 31) == 0 && out < dim) dw[out] = t;
}

}  // namespace btc
