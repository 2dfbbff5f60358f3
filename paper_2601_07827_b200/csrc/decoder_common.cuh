// Building blocks of the decoder operators: element types, 16-byte vectors, divisions by run-time constants.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace btc {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Vectors of 16 or 8 bytes as fp32 values and back (one rounding to nearest even per value).
template <int BYTES> struct VectorOf;
template <> struct VectorOf<16> { typedef uint4 type; };
template <> struct VectorOf<8> { typedef uint2 type; };

__device__ __forceinline__ void unpack_word(uint32_t w, float &lo, float &hi, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    lo = f.x;
    hi = f.y;
}
__device__ __forceinline__ void unpack_word(uint32_t w, float &lo, float &hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T, int V> __device__ __forceinline__ void unpack_vector(const typename VectorOf<V * int(sizeof(T))>::type &r, float (&v)[V])
{
    constexpr int WORDS = V * int(sizeof(T)) / 4;
    uint32_t w[WORDS];
    w[0] = r.x; w[1] = r.y;
    if constexpr (WORDS == 4) { w[2] = r.z; w[3] = r.w; }
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
        else unpack_word(w[i], v[2 * i], v[2 * i + 1], T());
    }
}
template <typename T, int V> __device__ __forceinline__ typename VectorOf<V * int(sizeof(T))>::type pack_vector(const float (&v)[V])
{
    constexpr int WORDS = V * int(sizeof(T)) / 4;
    uint32_t w[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
        else w[i] = pack2(v[2 * i], v[2 * i + 1], T());
    }
    if constexpr (WORDS == 4) return make_uint4(w[0], w[1], w[2], w[3]);
    else return make_uint2(w[0], w[1]);
}

// The decoder kernels may be launched while the one before it in the stream still runs (its set-up is then hidden): it
// touches nothing before that one has ended, and lets the next one do the same.
__device__ __forceinline__ void early_begin()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// Pairs of fp32 operations.  (As the packed two-in-one instructions they cost more moves between registers than
// they save: the rotary kernels took 3 to 10 % longer with them.)
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 without a divide: q = (n * mul) >> shift in 64 bits, with
// shift = 31 + ceil(log2 d) and mul = ceil(2^shift / d) <= 2^32 - 1 (exact because mul * d - 2^shift < d)
struct FastDiv {
    uint32_t mul = 1, shift = 0, d = 1;
    void set(int64_t divisor)
    {
        int s = 0;
        while ((int64_t(1) << s) < divisor) ++s;
        d = uint32_t(divisor);
        shift = uint32_t(31 + s);
        mul = uint32_t(((uint64_t(1) << shift) + uint64_t(divisor) - 1) / uint64_t(divisor));
    }
    __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const { return uint32_t((uint64_t(n) * mul) >> shift); }
};

}  // namespace btc
