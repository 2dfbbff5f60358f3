// C entry points of the products with 4-bit weights (linear4_kernel.cuh).
#include <algorithm>
#include <atomic>
#include <climits>
#include <cstring>
#include <type_traits>

#include "decoder_host.h"
#include "linear4_kernel.cuh"

using namespace btc;

struct btc_linear4_s {
    btc_handle_s handle;
    TensorDesc x, xs, y;
    bool x_scaled = false, zeros = false;
    btc_dtype_t scale_type = BTC_F32;
    int32_t group = 0, x_group = 0, activation = 0;
    int64_t row_blocks = 0, k_blocks = 0, stretches = 0, groups = 1;
    int32_t stretch_bytes = 0, head_bytes = 0, zeros_at = 0;
    int32_t nt = 1, wk = 8, ranks = 1, chunk = 8, slice = 8;       // see plan()
    size_t staged = 0, shared = 0;
};

namespace {

constexpr int64_t kMaxExtent = int64_t(1) << 24;           // of k and n: indices and counts stay in 32 bits
constexpr int64_t kMaxTokens = int64_t(1) << 19;           // tiles of 16 or more tokens in a grid's second dimension
constexpr int64_t kStagedBytes = 64 * 1024;                // of x at a time: more leaves one CTA to an SM

size_t esize(btc_dtype_t t) { return t == BTC_F32 ? 4 : (t == BTC_E4M3 ? 1 : 2); }
int parts_of(const btc_linear4_s &op) { return op.x.dtype == BTC_F32 ? 3 : 1; }
int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int32_t log2_of(int32_t group) { return group == 0 ? 31 : 31 - __builtin_clz(unsigned(group)); }

// k per scale within a stretch, as a power of two
int32_t stretch_group_log2(const btc_linear4_s &op) { return std::min(log2_of(op.group), log2_of(kL4Stretch * kL4K)); }

// How rows and k are spread over CTAs (8 warps = 8 / wk row blocks x wk shares of k; `ranks` CTAs of a cluster split k once more).
// Measured with weights from HBM, bf16, (wk, ranks), row blocks x stretches; best in brackets:
//   1 token    384 x 16: (4, 1) 7.7 us [7.7], 256 x 56: (4, 2) 13.2 [12.4], 896 x 16: (1, 1) 20.2 [20.2], 1792 x 32: (1, 2) 62 [62], 128 x 8: (8, 1) 3.4 [3.4]
//   8 tokens   384 x 16: (1, 4) 9.1 [9.1], 256 x 56: (2, 4) 14.5 [14.5], 896 x 16: (1, 1) 22.9 [22.9], 1792 x 32: (1, 2) 71 [71], 128 x 8: (8, 1) 4.5 [4.5]
//   32 tokens  384 x 16: (1, 4) 19.8 [19.8], 256 x 56: (1, 8) 28.0 [28.0], 896 x 16: (1, 2) 56.7 [52.0], 1792 x 32: (1, 2) 176 [175], 64 x 4: (8, 2) 7.3 [7.2]
// The same rule for other types of x, over the same row blocks x stretches (384 x 16, 256 x 56, 896 x 16 gated, 1792 x 32 gated, 128 x 8):
//   e4m3   1 token   7.0 12.7 18.5 67.9 3.7 us [7.2 12.1 18.6 64.4 3.8]    8 tokens  10.2 15.4 22.9 82.2 5.1 [9.1 15.4 22.9 75.8 5.1]
//          32 tokens 21.0 31.2 61.9 198 10.5 [21.0 31.0 56.0 193 9.7]
//   fp32   1 token   10.6 17.8 32.8 103 5.1 [10.6 17.7 30.4 103 4.8]       8 tokens  12.3 23.6 38.4 123 5.5 [12.1 20.5 36.0 123 5.5]
//          32 tokens 32.1 59.8 109 369 9.2 [32.1 53.3 109 369 9.2]
// (up to 15 % from the best; the choice of all pairs of 1, 2, 4, 8 was timed).
void plan(btc_linear4_s &op)
{
    const int64_t tokens = op.x.extent[0], sms = op.handle.sm_count;
    // more than 8 tokens, and more than 16, take wider products, so that a code becomes a number once for them (fp32 with its
    // three parts up to 16)
    op.nt = tokens <= 8 ? 1 : (tokens <= 16 || op.x.dtype == BTC_F32 ? 2 : 4);
    const int64_t block = int64_t(op.nt) * parts_of(op) * 1024 * kL4Stretch;      // x of a stretch in shared memory
    // splits of k: until there is a CTA for each SM (with short k for most of them)
    const int64_t enough = op.stretches <= 16 ? sms * 7 / 10 : sms;
    int64_t splits = 1;
    while (op.row_blocks * splits / kL4Warps < enough && splits < op.stretches && splits < 64) splits *= 2;
    // over a cluster's CTAs as far as that keeps the x that each of them brings small, the rest over warps
    const int64_t most = tokens > 16 ? 8 : 4, x_bytes = std::min<int64_t>(tokens, 8 * op.nt) * op.x.extent[1] * int64_t(esize(op.x.dtype) == 4 ? 4 : 2);
    op.ranks = 1;
    if (splits == 1) {
        if (op.stretches * block > kStagedBytes) op.ranks = 2;
    } else {
        while (op.ranks < most && op.ranks < splits && (x_bytes / op.ranks > 32 * 1024 || splits / op.ranks > kL4Warps)) op.ranks *= 2;
    }
    op.wk = int32_t(std::min<int64_t>(kL4Warps, std::max<int64_t>(1, splits / op.ranks)));
    while (op.wk * block > kStagedBytes && op.wk > 1) op.wk /= 2;
    op.slice = int32_t((op.stretches + op.ranks - 1) / op.ranks);
    op.chunk = int32_t(std::min(round_up(op.slice, op.wk), std::max<int64_t>(op.wk, kStagedBytes / block / op.wk * op.wk)));
    op.staged = size_t(op.chunk * block);
    op.shared = std::max(op.staged + size_t(kL4Warps) * kL4Stages * size_t(op.stretch_bytes), size_t(kL4Warps) * 8 * size_t(op.nt) * kL4Rows * 4);
}

template <typename CODES, int PARTS, int NT, bool SHORT, bool ZEROS, bool XG>
btc_error_t launch(const btc_linear4_s &op, const Linear4Params &p, dim3 blocks, cudaStream_t st)
{
    static std::atomic<bool> configured[64] = {};
    const int slot = op.handle.device & 63;
    if (!configured[slot].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(linear4_kernel<CODES, PARTS, NT, SHORT, ZEROS, XG>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024) != cudaSuccess) {
            cudaGetLastError();
            return BTC_ERR_CUDA;
        }
        configured[slot].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3(kL4Warps * 32);
    cfg.dynamicSmemBytes = op.shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(op.ranks);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = op.ranks > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, linear4_kernel<CODES, PARTS, NT, SHORT, ZEROS, XG>, p) != cudaSuccess) {
        cudaGetLastError();
        return BTC_ERR_CUDA;
    }
    return BTC_SUCCESS;
}
template <typename CODES, int PARTS, int NT, bool SHORT> btc_error_t launch_scaled(const btc_linear4_s &op, const Linear4Params &p, dim3 blocks, cudaStream_t st)
{
    if constexpr (std::is_same<CODES, F16Codes>::value)
        if (op.x_group != 0) return op.zeros ? launch<CODES, PARTS, NT, SHORT, true, true>(op, p, blocks, st) : launch<CODES, PARTS, NT, SHORT, false, true>(op, p, blocks, st);
    return op.zeros ? launch<CODES, PARTS, NT, SHORT, true, false>(op, p, blocks, st) : launch<CODES, PARTS, NT, SHORT, false, false>(op, p, blocks, st);
}
template <typename CODES, int PARTS> btc_error_t launch_typed(const btc_linear4_s &op, const Linear4Params &p, dim3 blocks, cudaStream_t st)
{
    const bool narrow = op.group == 32 || op.x_group == 32;
    if constexpr (PARTS == 1)
        if (op.nt == 4) return narrow ? launch_scaled<CODES, PARTS, 4, true>(op, p, blocks, st) : launch_scaled<CODES, PARTS, 4, false>(op, p, blocks, st);
    if (narrow) return op.nt == 1 ? launch_scaled<CODES, PARTS, 1, true>(op, p, blocks, st) : launch_scaled<CODES, PARTS, 2, true>(op, p, blocks, st);
    return op.nt == 1 ? launch_scaled<CODES, PARTS, 1, false>(op, p, blocks, st) : launch_scaled<CODES, PARTS, 2, false>(op, p, blocks, st);
}

bool group_ok(int32_t g) { return g == 0 || g == 32 || g == 64 || g == 128 || g == 256; }

}  // namespace

extern "C" {

btc_error_t btc_create_linear4(btc_handle_t handle, btc_tensor_info_t X, btc_tensor_info_t XS, btc_tensor_info_t Y, int32_t x_group,
                               btc_dtype_t scale_type, int32_t group, int32_t zeros, int32_t activation, btc_linear4_t *out)
{
    if (!handle || !X || !Y || !out) return BTC_ERR_INVALID_ARGUMENT;
    if (!group_ok(group) || !group_ok(x_group) || activation < BTC_ACTIVATION_NONE || activation > BTC_ACTIVATION_GELU) return BTC_ERR_INVALID_ARGUMENT;
    return guarded([&]() -> btc_error_t {
        btc_linear4_s op;
        op.handle = *handle;
        op.x = X->desc; op.y = Y->desc;
        op.x_scaled = XS != nullptr;
        if (XS) op.xs = XS->desc;
        op.scale_type = scale_type;
        op.group = group; op.x_group = x_group; op.zeros = zeros != 0; op.activation = activation;
        if (op.x.extent.size() != 2 || op.y.extent.size() != 2 || (XS && op.xs.extent.size() != 2)) return BTC_ERR_INVALID_ARGUMENT;
        if ((op.x.dtype == BTC_E4M3) != op.x_scaled || (x_group != 0 && !op.x_scaled)) return BTC_ERR_INVALID_ARGUMENT;
        if (!(decoder_type(op.x.dtype) || op.x.dtype == BTC_E4M3) || !decoder_type(op.y.dtype) || !decoder_type(scale_type)) return BTC_ERR_NOT_SUPPORTED;
        if (XS && op.xs.dtype != BTC_F32) return BTC_ERR_NOT_SUPPORTED;
        const int64_t tokens = op.x.extent[0], k = op.x.extent[1], n = op.y.extent[1];
        if (op.y.extent[0] != tokens) return BTC_ERR_EXTENT_MISMATCH;
        if (XS && (op.xs.extent[0] != tokens || op.xs.extent[1] != (x_group ? (k + x_group - 1) / x_group : 1))) return BTC_ERR_EXTENT_MISMATCH;
        if (tokens > kMaxTokens || k > kMaxExtent || n > kMaxExtent) return BTC_ERR_NOT_SUPPORTED;
        for (const TensorDesc *t : {&op.x, &op.y, XS ? &op.xs : nullptr})
            if (t && !spans_fit(*t)) return BTC_ERR_NOT_SUPPORTED;
        if (d_may_alias(op.y)) return BTC_ERR_D_ALIASING;
        op.row_blocks = activation ? (n + 7) / 8 : (n + kL4Rows - 1) / kL4Rows;
        op.k_blocks = (k + kL4K - 1) / kL4K;
        op.stretches = (op.k_blocks + kL4Stretch - 1) / kL4Stretch;
        op.groups = group ? (k + group - 1) / group : 1;
        const int32_t per = (kL4Stretch * kL4K) >> stretch_group_log2(op);
        op.zeros_at = op.zeros ? per * kL4Rows * int32_t(esize(scale_type)) : 0;
        op.head_bytes = per * kL4Rows * int32_t(esize(scale_type)) + (op.zeros ? per * kL4Rows : 0);
        op.stretch_bytes = op.head_bytes + kL4Stretch * kL4Block;
        plan(op);
        btc_linear4_s *kept = new (std::nothrow) btc_linear4_s(std::move(op));
        if (!kept) return BTC_ERR_OUT_OF_MEMORY;
        *out = kept;
        return BTC_SUCCESS;
    });
}

btc_error_t btc_destroy_linear4(btc_linear4_t *op)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    delete *op;
    *op = nullptr;
    return BTC_SUCCESS;
}

btc_error_t btc_linear4_workspace_size(btc_linear4_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = 0;
    return BTC_SUCCESS;
}

btc_error_t btc_linear4_packed_size(btc_linear4_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = size_t(op->row_blocks * op->stretches * op->stretch_bytes);
    return BTC_SUCCESS;
}

btc_error_t btc_linear4_pack(btc_linear4_t op, void *cuda_stream, const uint8_t *codes, const void *scales, const uint8_t *zeros, void *packed)
{
    if (!op || !codes || !scales || !packed || (zeros != nullptr) != op->zeros) return BTC_ERR_INVALID_ARGUMENT;
    if (!aligned_to(scales, esize(op->scale_type)) || !aligned_to(packed, 256)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;
    Linear4PackParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.codes = codes; p.zeros = zeros; p.scales = scales;
    p.out = static_cast<unsigned char *>(packed);
    p.k = int32_t(op->x.extent[1]);
    p.row_bytes = (int64_t(p.k) + 1) / 2;
    p.n = int32_t(op->y.extent[1]);
    p.row_blocks = int32_t(op->row_blocks);
    p.stretches = int32_t(op->stretches);
    p.groups = int32_t(op->groups);
    p.group_log2 = stretch_group_log2(*op);
    p.row_group_log2 = log2_of(op->group);
    p.scale_bytes = int32_t(esize(op->scale_type));
    p.stretch_bytes = op->stretch_bytes; p.head_bytes = op->head_bytes; p.zeros_at = op->zeros_at;
    p.gated = op->activation != 0;
    const int64_t work = op->row_blocks * op->stretches * (kL4Stretch * 32 + ((kL4Stretch * kL4K) >> p.group_log2) * kL4Rows);
    linear4_pack_kernel<<<unsigned(std::min<int64_t>((work + 255) / 256, int64_t(op->handle.sm_count) * 16)), 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p);
    return cudaGetLastError() == cudaSuccess ? BTC_SUCCESS : BTC_ERR_CUDA;
}

btc_error_t btc_linear4_execute(btc_linear4_t op, void *cuda_stream, const void *packed, const void *X, const float *XS, void *Y,
                                void *workspace, size_t workspace_bytes)
{
    (void)workspace;
    (void)workspace_bytes;
    if (!op || !packed || !X || !Y || (XS != nullptr) != op->x_scaled) return BTC_ERR_INVALID_ARGUMENT;
    const int64_t es = int64_t(esize(op->x.dtype));
    if (!aligned_to(packed, 256) || !aligned_to(X, size_t(es)) || !aligned_to(Y, esize(op->y.dtype)) || !aligned_to(XS, 4)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;
    Linear4Params p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.packed = static_cast<const unsigned char *>(packed);
    p.x = X; p.xs = XS; p.y = Y;
    p.x_t = op->x.stride[0]; p.x_k = op->x.stride[1];
    if (op->x_scaled) { p.xs_t = op->xs.stride[0]; p.xs_g = op->xs.stride[1]; }
    p.y_t = op->y.stride[0]; p.y_n = op->y.stride[1];
    p.tokens = int32_t(op->x.extent[0]);
    p.k = int32_t(op->x.extent[1]);
    p.n = int32_t(op->y.extent[1]);
    p.row_blocks = int32_t(op->row_blocks);
    p.k_blocks = int32_t(op->k_blocks);
    p.stretch_bytes = op->stretch_bytes; p.head_bytes = op->head_bytes; p.zeros_at = op->zeros_at;
    p.group_log2 = stretch_group_log2(*op);
    p.xgroup_log2 = log2_of(op->x_group);
    p.x_type = op->x.dtype; p.y_type = op->y.dtype; p.scale_type = op->scale_type; p.activation = op->activation;
    const int64_t access = es == 1 ? 8 : 16;
    p.vec_x = (p.x_k == 1 || p.k == 1) && (p.tokens == 1 || p.x_t * es % access == 0) && aligned_to(X, size_t(access));
    p.wk = op->wk;
    p.chunk = op->chunk;
    p.slice = op->slice;
    p.staged_bytes = int32_t(op->staged);
    const int64_t wr = kL4Warps / op->wk, groups = (op->row_blocks + wr - 1) / wr, tiles = (p.tokens + 8 * op->nt - 1) / (8 * op->nt);
    const dim3 blocks(unsigned(groups * op->ranks), unsigned(tiles));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (op->x.dtype) {
    case BTC_F32: return launch_typed<BF16Codes, 3>(*op, p, blocks, st);
    case BTC_BF16: return launch_typed<BF16Codes, 1>(*op, p, blocks, st);
    default: return launch_typed<F16Codes, 1>(*op, p, blocks, st);
    }
}

}  // extern "C"
