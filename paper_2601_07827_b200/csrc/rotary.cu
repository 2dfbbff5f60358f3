// C entry points of the head norm and rotary position operator (rotary_kernel.cuh).
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstring>
#include <vector>

#include "decoder_host.h"
#include "rotary_kernel.cuh"

using namespace btc;

struct btc_rotary_s {
    btc_handle_s handle;
    btc_dtype_t dtype = BTC_F32;
    int32_t layout = BTC_ROTARY_HALF, pairs = 0, norm = 0;
    double multiplier = 1.0, eps = 0.0;
    bool has[3] = {false, false, false};
    TensorDesc x[3], y[3];
    bool paged[3] = {false, false, false}, x_aliases = false;
    int64_t tokens = 0, pages = 1, page_tokens = 1;
    uint64_t *d_freq = nullptr;
};

namespace {

constexpr int kBackwardCtasPerSm = 2;   // what the registers allow to run at once

size_t esize(btc_dtype_t t) { return t == BTC_F32 ? 4 : 2; }

// Do vectors of v elements fit: pairs and the unrotated rest in whole vectors per lane, at most 32 lanes to a head,
// heads contiguous, every other stride a multiple of the vector.  (Base addresses are looked at when a call is made.)
bool strides_allow_vectors(const btc_rotary_s &op, int64_t v)
{
    for (int i = 0; i < 3; ++i) {
        if (!op.has[i]) continue;
        const int64_t dim = op.x[i].extent[2], pairs = i < 2 ? op.pairs : 0;
        if (pairs % v != 0 || (dim - 2 * pairs) % (2 * v) != 0 || dim > 64 * v) return false;
        for (const TensorDesc *t : {&op.x[i], &op.y[i]}) {
            const size_t r = t->extent.size();
            if (t->stride[r - 1] != 1) return false;
            for (size_t k = 0; k + 1 < r; ++k)
                if (t->extent[k] > 1 && t->stride[k] % v != 0) return false;
            // byte offsets inside the tokens that a CTA takes at a time are formed in 32 bits, unsigned
            const int64_t token = t->stride[r - 3], head = t->stride[r - 2];
            if (token < 0 || head < 0 || (__int128(token) * kRotaryMaxTokens + __int128(head) * t->extent[r - 2] + 256) * 4 > INT32_MAX) return false;
        }
    }
    return true;
}

// bytes per access of a call whose addresses are multiples of `aligned`: 16, 8, or 0 for single elements
int vector_bytes(const btc_rotary_s &op, uintptr_t addresses)
{
    for (int bytes = 16; bytes >= 8; bytes /= 2)
        if (addresses % uintptr_t(bytes) == 0 && strides_allow_vectors(op, int64_t(bytes / int(esize(op.dtype))))) return bytes;
    return 0;
}

int lanes_log2_for(const btc_rotary_s &op, int bytes)
{
    if (bytes == 0) return 5;
    int64_t most = 1;
    const int64_t v = bytes / int64_t(esize(op.dtype));
    for (int i = 0; i < 3; ++i)
        if (op.has[i]) most = std::max(most, op.x[i].extent[2] / (2 * v));
    int k = 0;
    while ((int64_t(1) << k) < most) ++k;
    return k;
}

// Tokens a CTA takes at a time: so many that a group of lanes has `items` heads to do (the angles, the barrier and the
// address work are then spread over them) as long as that leaves `ctas` CTAs; few tokens go one to a CTA,
// because then only latency counts.  (16384 tokens, forward: 24 heads to a group and 4 CTAs per SM at least 110 us for 80 heads
// and 171 with the backward pass for 40; 8 and 6: 115 and 173; 5 and 6: 122 and 181.)
int tokens_per_cta(int64_t tokens, int64_t heads, int lanes_log2, int items, int64_t ctas)
{
    const int64_t groups = kRotaryThreads >> lanes_log2;
    int64_t n = std::min<int64_t>(kRotaryMaxTokens, std::max<int64_t>(1, items * groups / heads));
    while (n > 1 && (tokens + n - 1) / n < ctas) n = (n + 1) / 2;
    return int(n);
}

void fill_part(const btc_rotary_s &op, int i, RotaryPart &p)
{
    const TensorDesc &x = op.x[i], &y = op.y[i];
    p.x_t = x.stride[0]; p.x_h = x.stride[1]; p.x_d = x.stride[2];
    p.paged = op.paged[i];
    const size_t o = op.paged[i] ? 1 : 0;
    p.y_page = op.paged[i] ? y.stride[0] : 0;
    p.y_t = y.stride[o]; p.y_h = y.stride[o + 1]; p.y_d = y.stride[o + 2];
    p.heads = int32_t(x.extent[1]);
    p.dim = int32_t(x.extent[2]);
    p.pairs = i < 2 ? op.pairs : 0;
    p.rest_pairs = (p.dim - 2 * p.pairs + 1) / 2;
    p.copy = i == 2;
    p.inv_dim = 1.f / float(p.dim);
    p.head.set(p.heads);
}

template <typename T, int V>
btc_error_t launch_forward(const RotaryParams &p, bool interleaved, bool full, unsigned blocks, cudaStream_t st)
{
    constexpr bool F = V > 1;              // the scalar form asks for each slot in any case
    void (*kernel)(const RotaryParams) = interleaved ? (full ? rotary_forward_kernel<T, V, true, F> : rotary_forward_kernel<T, V, true, false>)
                                                     : (full ? rotary_forward_kernel<T, V, false, F> : rotary_forward_kernel<T, V, false, false>);
    return launch_early(kernel, blocks, kRotaryThreads, 0, st, p);
}
template <typename T, int V>
btc_error_t launch_backward(const RotaryParams &p, bool interleaved, bool full, unsigned blocks, cudaStream_t st)
{
    constexpr bool F = V > 1;              // the scalar form asks for each slot in any case
    void (*kernel)(const RotaryParams) = interleaved ? (full ? rotary_backward_kernel<T, V, true, F> : rotary_backward_kernel<T, V, true, false>)
                                                     : (full ? rotary_backward_kernel<T, V, false, F> : rotary_backward_kernel<T, V, false, false>);
    // Not set up early: persistent CTAs that arrive while the SMs still drain the kernel before cost large 16-bit passes
    // 3 to 5 %, and small ones gain next to nothing.  Forward and backward, 40 heads of 128 in bf16, set up early in
    // brackets: 8 tokens 6.7 us [6.5], 777 18.2 [18.1], 2048 34.3 [34.1], 4096 55.4 [58.2], 16384 170.6 [175.3]; 8 heads of 80
    // in fp32: 777 tokens 14.5 [14.5], 16384 85.5 [85.6]
    kernel<<<blocks, kRotaryThreads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? BTC_SUCCESS : BTC_ERR_CUDA;
}

#define BTC_ROTARY_DISPATCH(F, dtype, bytes, ...)                                                                        \
    ((dtype) == BTC_F32 ? ((bytes) == 16 ? F<float, 4>(__VA_ARGS__) : (bytes) == 8 ? F<float, 2>(__VA_ARGS__) : F<float, 1>(__VA_ARGS__))              \
     : (dtype) == BTC_F16 ? ((bytes) == 16 ? F<__half, 8>(__VA_ARGS__) : (bytes) == 8 ? F<__half, 4>(__VA_ARGS__) : F<__half, 1>(__VA_ARGS__))          \
     : ((bytes) == 16 ? F<__nv_bfloat16, 8>(__VA_ARGS__) : (bytes) == 8 ? F<__nv_bfloat16, 4>(__VA_ARGS__) : F<__nv_bfloat16, 1>(__VA_ARGS__)))

}  // namespace

extern "C" {

btc_error_t btc_create_rotary(btc_handle_t handle, int32_t layout, int32_t pairs, const double *frequencies,
                              double multiplier, int32_t norm, double eps, btc_tensor_info_t Xq, btc_tensor_info_t Yq,
                              btc_tensor_info_t Xk, btc_tensor_info_t Yk, btc_tensor_info_t Xv, btc_tensor_info_t Yv,
                              btc_rotary_t *out)
{
    if (!handle || !Xq || !Yq || !out) return BTC_ERR_INVALID_ARGUMENT;
    if ((Xk == nullptr) != (Yk == nullptr) || (Xv == nullptr) != (Yv == nullptr)) return BTC_ERR_INVALID_ARGUMENT;
    if (layout != BTC_ROTARY_HALF && layout != BTC_ROTARY_INTERLEAVED) return BTC_ERR_INVALID_ARGUMENT;
    if (pairs < 0 || (pairs > 0 && !frequencies) || !fits_f32(multiplier)) return BTC_ERR_INVALID_ARGUMENT;
    if (norm && !(eps == 0.0 || (eps >= double(FLT_MIN) && fits_f32(eps)))) return BTC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < pairs; ++i)
        if (!std::isfinite(frequencies[i])) return BTC_ERR_INVALID_ARGUMENT;
    return guarded([&]() -> btc_error_t {
        btc_tensor_info_t X[3] = {Xq, Xk, Xv}, Y[3] = {Yq, Yk, Yv};
        btc_rotary_s op;
        op.handle = *handle;
        op.dtype = Xq->desc.dtype;
        op.layout = layout; op.pairs = pairs; op.norm = norm != 0; op.multiplier = multiplier; op.eps = eps;
        if (!decoder_type(op.dtype)) return BTC_ERR_NOT_SUPPORTED;
        bool any_paged = false;
        for (int i = 0; i < 3; ++i) {
            op.has[i] = X[i] != nullptr;
            if (!op.has[i]) continue;
            const TensorDesc &x = X[i]->desc, &y = Y[i]->desc;
            if (x.dtype != op.dtype || y.dtype != op.dtype) return BTC_ERR_NOT_SUPPORTED;
            if (x.extent.size() != 3 || !(y.extent.size() == 3 || (i > 0 && y.extent.size() == 4))) return BTC_ERR_INVALID_ARGUMENT;
            op.x[i] = x;
            op.y[i] = y;
            op.paged[i] = y.extent.size() == 4;
            const size_t o = op.paged[i] ? 2 : 1;
            if (i == 0) op.tokens = x.extent[0];
            if (x.extent[0] != op.tokens || y.extent[o] != x.extent[1] || y.extent[o + 1] != x.extent[2]) return BTC_ERR_EXTENT_MISMATCH;
            if (i == 1 && x.extent[2] != Xq->desc.extent[2]) return BTC_ERR_EXTENT_MISMATCH;
            if (op.paged[i]) {
                if (any_paged && (y.extent[0] != op.pages || y.extent[1] != op.page_tokens)) return BTC_ERR_EXTENT_MISMATCH;
                any_paged = true;
                op.pages = y.extent[0];
                op.page_tokens = y.extent[1];
                if (op.pages > INT32_MAX || op.page_tokens > INT32_MAX || op.pages * op.page_tokens > INT32_MAX) return BTC_ERR_NOT_SUPPORTED;
            } else if (y.extent[0] != op.tokens) {
                return BTC_ERR_EXTENT_MISMATCH;
            }
            if (x.extent[2] > kRotaryMaxDim || x.extent[1] > INT32_MAX / 2 || op.tokens > (int64_t(1) << 40)) return BTC_ERR_NOT_SUPPORTED;
            if (!spans_fit(x) || !spans_fit(y)) return BTC_ERR_NOT_SUPPORTED;
            if (i < 2 && 2 * int64_t(pairs) > x.extent[2]) return BTC_ERR_INVALID_ARGUMENT;
            if (d_may_alias(y)) return BTC_ERR_D_ALIASING;
            op.x_aliases = op.x_aliases || d_may_alias(x);
        }
        if (pairs > 0 && op.handle.device >= 0) {
            // turns per position modulo one turn (positions are whole), in units of 2^-64 turn
            std::vector<uint64_t> f(size_t(pairs), 0);
            for (int32_t i = 0; i < pairs; ++i) {
                const long double turns = static_cast<long double>(frequencies[i]) / (2.0L * 3.14159265358979323846264338327950288L);
                const long double frac = turns - floorl(turns);                         // [0, 1]
                const long double scaled = floorl(frac * 18446744073709551616.0L + 0.5L);
                f[size_t(i)] = scaled >= 18446744073709551616.0L ? 0 : uint64_t(scaled);
            }
            if (cudaMalloc(&op.d_freq, f.size() * 8) != cudaSuccess) {
                cudaGetLastError();
                return BTC_ERR_OUT_OF_MEMORY;
            }
            // the copy of ordinary memory may still be under way when cudaMemcpy returns: wait, so that any stream may run the operation
            if (cudaMemcpy(op.d_freq, f.data(), f.size() * 8, cudaMemcpyHostToDevice) != cudaSuccess ||
                cudaStreamSynchronize(nullptr) != cudaSuccess) {
                cudaGetLastError();
                cudaFree(op.d_freq);
                return BTC_ERR_CUDA;
            }
        }
        btc_rotary_s *kept = new (std::nothrow) btc_rotary_s(std::move(op));
        if (!kept) {
            if (op.d_freq) cudaFree(op.d_freq);
            return BTC_ERR_OUT_OF_MEMORY;
        }
        *out = kept;
        return BTC_SUCCESS;
    });
}

btc_error_t btc_destroy_rotary(btc_rotary_t *op)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    if (*op) {
        if ((*op)->d_freq) cudaFree((*op)->d_freq);
        delete *op;
    }
    *op = nullptr;
    return BTC_SUCCESS;
}

btc_error_t btc_rotary_workspace_size(btc_rotary_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = op->norm ? size_t(op->handle.sm_count) * kBackwardCtasPerSm * kRotaryMaxDim * sizeof(float) : 0;
    return BTC_SUCCESS;
}

btc_error_t btc_rotary_execute(btc_rotary_t op, void *cuda_stream, const int32_t *positions, const int32_t *slots,
                               const void *Wq, const void *Wk, const void *Xq, void *Yq, const void *Xk, void *Yk,
                               const void *Xv, void *Yv, int32_t *flags)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    const void *X[3] = {Xq, Xk, Xv}, *W[3] = {Wq, Wk, nullptr};
    void *Y[3] = {Yq, Yk, Yv};
    bool any_paged = false;
    uintptr_t addresses = 0;
    const size_t es = esize(op->dtype);
    for (int i = 0; i < 3; ++i) {
        if (!op->has[i]) {
            if (X[i] || Y[i] || W[i]) return BTC_ERR_INVALID_ARGUMENT;
            continue;
        }
        any_paged = any_paged || op->paged[i];
        if (!X[i] || !Y[i] || (W[i] && !op->norm)) return BTC_ERR_INVALID_ARGUMENT;
        for (const void *q : {X[i], static_cast<const void *>(Y[i]), W[i]}) {
            if (!aligned_to(q, es)) return BTC_ERR_MISALIGNED;
            addresses |= reinterpret_cast<uintptr_t>(q);
        }
    }
    if ((op->pairs > 0 && !positions) || (any_paged && !slots)) return BTC_ERR_INVALID_ARGUMENT;
    if (!aligned_to(positions, 4) || !aligned_to(slots, 4) || !aligned_to(flags, 4)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;

    RotaryParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    const int bytes = vector_bytes(*op, addresses);
    p.lanes_log2 = lanes_log2_for(*op, bytes);
    int64_t blocks = 0;
    for (int i = 0; i < 3; ++i) {
        if (!op->has[i]) continue;
        RotaryPart &part = p.part[i];
        fill_part(*op, i, part);
        part.x = X[i]; part.y = Y[i]; part.w = W[i];
        if (part.heads > INT32_MAX / kRotaryMaxTokens / 2) return BTC_ERR_NOT_SUPPORTED;
        part.cta_tokens = tokens_per_cta(op->tokens, part.heads, p.lanes_log2, 24, int64_t(op->handle.sm_count) * 4);
        const int64_t ctas = (op->tokens + part.cta_tokens - 1) / part.cta_tokens;
        if (ctas > INT32_MAX / 4) return BTC_ERR_NOT_SUPPORTED;
        part.ctas = uint32_t(ctas);
        blocks += ctas;
    }
    p.pos = positions; p.slots = slots; p.freq = op->d_freq; p.flags = flags;
    p.tokens = op->tokens;
    p.pairs = op->pairs;
    p.pair.set(std::max(op->pairs, 1));
    p.norm = op->norm; p.eps = float(op->eps); p.mult = float(op->multiplier);
    p.page.set(op->page_tokens);
    p.slot_count = int32_t(op->pages * op->page_tokens);
    return BTC_ROTARY_DISPATCH(launch_forward, op->dtype, bytes, p, op->layout == BTC_ROTARY_INTERLEAVED,
                               2 * int64_t(op->pairs) == op->x[0].extent[2], unsigned(blocks), static_cast<cudaStream_t>(cuda_stream));
}

btc_error_t btc_rotary_backward(btc_rotary_t op, void *cuda_stream, const int32_t *positions, const void *Wq,
                                const void *Wk, const void *Xq, const void *dYq, void *dXq, const void *Xk,
                                const void *dYk, void *dXk, float *dWq, float *dWk, void *workspace,
                                size_t workspace_bytes)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    if (op->has[2] || op->paged[1]) return BTC_ERR_NOT_SUPPORTED;
    if (op->x_aliases) return BTC_ERR_D_ALIASING;
    const void *X[2] = {Xq, Xk}, *dY[2] = {dYq, dYk}, *W[2] = {Wq, Wk};
    void *dX[2] = {dXq, dXk};
    float *dW[2] = {dWq, dWk};
    uintptr_t addresses = 0;
    const size_t es = esize(op->dtype);
    for (int i = 0; i < 2; ++i) {
        if (!op->has[i]) {
            if (X[i] || dY[i] || dX[i] || W[i] || dW[i]) return BTC_ERR_INVALID_ARGUMENT;
            continue;
        }
        if (!dY[i] || !dX[i] || (op->norm && !X[i]) || ((W[i] || dW[i]) && !op->norm)) return BTC_ERR_INVALID_ARGUMENT;
        if (!aligned_to(dW[i], 4)) return BTC_ERR_MISALIGNED;
        for (const void *q : {op->norm ? X[i] : nullptr, dY[i], static_cast<const void *>(dX[i]), W[i]}) {
            if (!aligned_to(q, es)) return BTC_ERR_MISALIGNED;
            addresses |= reinterpret_cast<uintptr_t>(q);
        }
    }
    if (op->pairs > 0 && !positions) return BTC_ERR_INVALID_ARGUMENT;
    if (!aligned_to(positions, 4)) return BTC_ERR_MISALIGNED;
    const bool sums = dWq || dWk;
    size_t need = 0;
    btc_rotary_workspace_size(op, &need);
    if (sums && (!workspace || workspace_bytes < need)) return BTC_ERR_WORKSPACE_TOO_SMALL;
    if (sums && !aligned_to(workspace, 256)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;

    RotaryParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    const int bytes = vector_bytes(*op, addresses);
    p.lanes_log2 = lanes_log2_for(*op, bytes);
    const int64_t most = int64_t(op->handle.sm_count) * kBackwardCtasPerSm;
    int64_t all_heads = 0;
    for (int i = 0; i < 2; ++i)
        if (op->has[i]) all_heads += op->x[i].extent[1];
    if (all_heads > INT32_MAX / kRotaryMaxTokens / 2) return BTC_ERR_NOT_SUPPORTED;
    for (int i = 0; i < 2; ++i) {
        if (!op->has[i]) continue;
        RotaryPart &part = p.part[i];
        fill_part(*op, i, part);
        part.x = X[i]; part.dy = dY[i]; part.y = dX[i]; part.w = W[i];
        // each part gets CTAs by its share of the heads, at least one, at most one per block of tokens
        const int64_t share = std::max<int64_t>(1, std::min(most - 1, ((most - 1) * part.heads + all_heads / 2) / all_heads));
        part.cta_tokens = tokens_per_cta(op->tokens, part.heads, p.lanes_log2, 16, share);
        part.ctas = uint32_t(std::min<int64_t>(share, (op->tokens + part.cta_tokens - 1) / part.cta_tokens));
    }
    p.pos = positions; p.freq = op->d_freq;
    p.partial = sums ? static_cast<float *>(workspace) : nullptr;
    p.tokens = op->tokens;
    p.pairs = op->pairs;
    p.pair.set(std::max(op->pairs, 1));
    p.norm = op->norm; p.eps = float(op->eps); p.mult = float(op->multiplier);
    p.page.set(1);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const btc_error_t rc = BTC_ROTARY_DISPATCH(launch_backward, op->dtype, bytes, p, op->layout == BTC_ROTARY_INTERLEAVED,
                                               2 * int64_t(op->pairs) == op->x[0].extent[2], unsigned(p.part[0].ctas + p.part[1].ctas), st);
    if (rc != BTC_SUCCESS || !sums) return rc;
    const int dim = int(op->x[0].extent[2]);
    return launch_early(rotary_weight_gradient_kernel, dim3(unsigned((dim + kRotaryGradColumns - 1) / kRotaryGradColumns), 2), kRotaryGradThreads,
                        0, st, static_cast<const float *>(p.partial), int(p.part[0].ctas), int(p.part[1].ctas), dim, dWq, dWk);
}

}  // extern "C"
