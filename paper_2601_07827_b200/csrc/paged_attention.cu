// C entry points of the paged attention operator (paged_attention_kernel.cuh).
#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstring>

#include "decoder_host.h"
#include "paged_attention_kernel.cuh"

using namespace btc;

struct btc_paged_attention_s {
    btc_handle_s handle;
    TensorDesc q, k, v, table, o;
    double scale = 1.0;
    int32_t window = 0;
    int32_t dp = 64, nt = 1;       // padded head size, blocks of 8 query heads per item
    int64_t blocks = 1;            // items per key head
};

namespace {

constexpr double kLog2E = 1.4426950408889634;

size_t esize(btc_dtype_t t) { return t == BTC_F32 ? 4 : 2; }

// CTAs of the first kernel: one per SM (shared memory admits no second)
int ctas_of(const btc_paged_attention_s &op) { return op.handle.sm_count; }

int64_t slot_floats(const btc_paged_attention_s &op) { return int64_t(8 * op.nt) * op.dp + 16 * op.nt; }

size_t workspace_bytes_of(const btc_paged_attention_s &op)
{
    const size_t ctas = size_t(ctas_of(op));
    return ctas * 2 * size_t(slot_floats(op)) * sizeof(float) + ctas * 2 * sizeof(int32_t);
}

bool rows_allow_vectors(const TensorDesc &t, int64_t elements)
{
    const size_t r = t.extent.size();
    if (t.stride[r - 1] != 1) return false;
    for (size_t i = 0; i + 1 < r; ++i)
        if (t.stride[i] % elements != 0) return false;
    return true;
}

template <typename T, int DP, int NT>
btc_error_t launch(const AttentionParams &p, int device, int ctas, cudaStream_t st)
{
    typedef AttentionShape<T, DP, NT> Shape;
    static std::atomic<bool> configured[64] = {};
    const int slot = device & 63;
    if (!configured[slot].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(paged_attention_kernel<T, DP, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::SMEM) != cudaSuccess) {
            cudaGetLastError();
            return BTC_ERR_CUDA;
        }
        configured[slot].store(true, std::memory_order_relaxed);
    }
    const btc_error_t rc = launch_early(paged_attention_kernel<T, DP, NT>, dim3(unsigned(ctas)), Shape::WARPS * 32, Shape::SMEM, st, p);
    if (rc != BTC_SUCCESS) return rc;
    return launch_early(paged_attention_join_kernel<T, DP, NT>, dim3(unsigned(ctas), kJoinSlices), kJoinThreads, 0, st, p, ctas);
}

template <typename T> btc_error_t launch_typed(const btc_paged_attention_s &op, const AttentionParams &p, cudaStream_t st)
{
    const int dev = op.handle.device, ctas = ctas_of(op);
    if (op.dp == 64) return op.nt == 1 ? launch<T, 64, 1>(p, dev, ctas, st) : launch<T, 64, 2>(p, dev, ctas, st);
    if constexpr (sizeof(T) == 4)
        if (op.dp == 96) return op.nt == 1 ? launch<T, 96, 1>(p, dev, ctas, st) : launch<T, 96, 2>(p, dev, ctas, st);
    if (op.dp == 128) return op.nt == 1 ? launch<T, 128, 1>(p, dev, ctas, st) : launch<T, 128, 2>(p, dev, ctas, st);
    return launch<T, 256, 1>(p, dev, ctas, st);
}

}  // namespace

extern "C" {

btc_error_t btc_create_paged_attention(btc_handle_t handle, btc_tensor_info_t Q, btc_tensor_info_t K,
                                       btc_tensor_info_t V, btc_tensor_info_t table, btc_tensor_info_t O, double scale,
                                       int32_t window, btc_paged_attention_t *out)
{
    if (!handle || !Q || !K || !V || !table || !O || !out) return BTC_ERR_INVALID_ARGUMENT;
    if (window < 0 || !fits_f32(scale * kLog2E)) return BTC_ERR_INVALID_ARGUMENT;
    return guarded([&]() -> btc_error_t {
        const TensorDesc &q = Q->desc, &k = K->desc, &v = V->desc, &t = table->desc, &o = O->desc;
        if (q.extent.size() != 3 || k.extent.size() != 4 || v.extent.size() != 4 || t.extent.size() != 2 || o.extent.size() != 3)
            return BTC_ERR_INVALID_ARGUMENT;
        if (!decoder_type(q.dtype) || k.dtype != q.dtype || v.dtype != q.dtype || o.dtype != q.dtype || t.dtype != BTC_I32)
            return BTC_ERR_NOT_SUPPORTED;
        if (k.extent[3] != q.extent[2] || o.extent[2] != v.extent[3] || o.extent[0] != q.extent[0] || o.extent[1] != q.extent[1] ||
            t.extent[0] != q.extent[0] || v.extent[0] != k.extent[0] || v.extent[1] != k.extent[1] || v.extent[2] != k.extent[2] ||
            q.extent[1] % k.extent[2] != 0)
            return BTC_ERR_EXTENT_MISMATCH;
        if (q.extent[2] > kAttnMaxDim || v.extent[3] > kAttnMaxDim) return BTC_ERR_NOT_SUPPORTED;
        if (k.extent[0] > INT32_MAX || k.extent[1] > INT32_MAX || t.extent[1] > INT32_MAX || q.extent[0] > kAttnMaxSequences ||
            q.extent[1] > INT32_MAX / 2 || q.extent[1] * o.extent[2] > INT32_MAX / 2)
            return BTC_ERR_NOT_SUPPORTED;
        for (const TensorDesc *d : {&q, &k, &v, &t, &o})
            if (!spans_fit(*d)) return BTC_ERR_NOT_SUPPORTED;
        if (d_may_alias(o)) return BTC_ERR_D_ALIASING;
        btc_paged_attention_s op;
        op.handle = *handle;
        op.q = q; op.k = k; op.v = v; op.table = t; op.o = o;
        op.scale = scale;
        op.window = window;
        const int64_t dim = std::max(q.extent[2], v.extent[3]), group = q.extent[1] / k.extent[2];
        // fp32 heads of 65 to 96 elements have a size of their own because products and shared memory bound them (padded to
        // 128 in brackets): 24 windows of 1000 tokens, heads of 80: 17.4 us [19.6]; 64 ragged requests, heads of 80: 112
        // [154], of 96: 117 [154], 16 heads to a key head: 186 [282]; 8 requests 25 [31]; 2 x 128 Ki tokens 240 [339]; one
        // request 12.6 [12.8]
        op.dp = dim <= 64 ? 64 : (dim <= 96 && q.dtype == BTC_F32 ? 96 : (dim <= 128 ? 128 : 256));
        // Groups of more than 8 heads take 16 at a time, so that the cache is read once per 16 heads (8 at a time in
        // brackets: 64 ragged requests, groups of 9: 108 us [133], of 12: 114 [133], of 16: 114 [134], of 24: 194 [197], of 16 with heads
        // of 64: 72 [95], of 16 in fp32: 282 [301]; 2 x 128 Ki tokens, groups of 16: 183 [241]).  A lone short request loses (1500
        // tokens, groups of 16: 15.5 [12.3]), but lengths are not known here.  Heads of more than 128 elements 8 at a time
        // (the output of 16 would not fit the registers)
        op.nt = group > 8 && op.dp <= 128 ? 2 : 1;
        op.blocks = (group + 8 * op.nt - 1) / (8 * op.nt);
        if (__int128(q.extent[0]) * k.extent[2] * op.blocks > INT32_MAX) return BTC_ERR_NOT_SUPPORTED;
        // tiles of all sequences: 38 bits of the kernel's prefix sum
        if (__int128(q.extent[0]) * (std::min<int64_t>(t.extent[1] * k.extent[1], INT32_MAX) / kAttnTok + 1) >= (__int128(1) << 38)) return BTC_ERR_NOT_SUPPORTED;
        btc_paged_attention_s *kept = new (std::nothrow) btc_paged_attention_s(std::move(op));
        if (!kept) return BTC_ERR_OUT_OF_MEMORY;
        *out = kept;
        return BTC_SUCCESS;
    });
}

btc_error_t btc_destroy_paged_attention(btc_paged_attention_t *op)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    delete *op;
    *op = nullptr;
    return BTC_SUCCESS;
}

btc_error_t btc_paged_attention_workspace_size(btc_paged_attention_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = workspace_bytes_of(*op);
    return BTC_SUCCESS;
}

btc_error_t btc_paged_attention_execute(btc_paged_attention_t op, void *cuda_stream, const void *Q, const void *K,
                                        const void *V, const int32_t *table, const int32_t *lengths, void *O, float *lse,
                                        void *workspace, size_t workspace_bytes, int32_t *flags)
{
    if (!op || !Q || !K || !V || !table || !lengths || !O) return BTC_ERR_INVALID_ARGUMENT;
    const size_t es = esize(op->q.dtype);
    for (const void *x : {Q, K, V, static_cast<const void *>(O)})
        if (!aligned_to(x, es)) return BTC_ERR_MISALIGNED;
    if (!aligned_to(table, 4) || !aligned_to(lengths, 4) || !aligned_to(lse, 4) || !aligned_to(flags, 4)) return BTC_ERR_MISALIGNED;
    if (!workspace || workspace_bytes < workspace_bytes_of(*op)) return BTC_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned_to(workspace, 256)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;

    AttentionParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.q = Q; p.k = K; p.v = V; p.o = O;
    p.table = table; p.lengths = lengths; p.lse = lse; p.flags = flags;
    const int64_t ctas = ctas_of(*op);
    p.partial = static_cast<float *>(workspace);
    p.partial_item = reinterpret_cast<int32_t *>(p.partial + ctas * 2 * slot_floats(*op));
    p.q_n = op->q.stride[0]; p.q_h = op->q.stride[1]; p.q_d = op->q.stride[2];
    p.o_n = op->o.stride[0]; p.o_h = op->o.stride[1]; p.o_d = op->o.stride[2];
    p.k_page = op->k.stride[0]; p.k_slot = op->k.stride[1]; p.k_head = op->k.stride[2]; p.k_d = op->k.stride[3];
    p.v_page = op->v.stride[0]; p.v_slot = op->v.stride[1]; p.v_head = op->v.stride[2]; p.v_d = op->v.stride[3];
    p.table_n = op->table.stride[0]; p.table_j = op->table.stride[1];
    p.sequences = int32_t(op->q.extent[0]);
    p.heads = int32_t(op->q.extent[1]);
    p.key_heads = int32_t(op->k.extent[2]);
    p.group = p.heads / p.key_heads;
    p.blocks = int32_t(op->blocks);
    p.dim_k = int32_t(op->k.extent[3]);
    p.dim_v = int32_t(op->v.extent[3]);
    p.pages = int32_t(op->k.extent[0]);
    p.columns = int32_t(op->table.extent[1]);
    p.window = op->window;
    p.page.set(op->k.extent[1]);
    p.room = int32_t(std::min<int64_t>(op->table.extent[1] * op->k.extent[1], 0x7ffffff0));
    const int64_t vec = int64_t(16 / es);
    p.vec_k = rows_allow_vectors(op->k, vec) && aligned_to(K, 16);
    p.vec_v = rows_allow_vectors(op->v, vec) && aligned_to(V, 16);
    p.whole_tiles = !(p.vec_k && p.vec_v) ? 0 : (op->k.extent[1] % kAttnTok == 0 ? kAttnTok : (op->k.extent[1] % 8 == 0 ? 8 : 0));
    p.vec_q = es == 2 && p.dim_k % 2 == 0 && rows_allow_vectors(op->q, 2) && aligned_to(Q, 4);
    p.scale_log2 = float(op->scale * kLog2E);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (op->q.dtype) {
    case BTC_F32: return launch_typed<float>(*op, p, st);
    case BTC_F16: return launch_typed<__half>(*op, p, st);
    default: return launch_typed<__nv_bfloat16>(*op, p, st);
    }
}

}  // extern "C"
