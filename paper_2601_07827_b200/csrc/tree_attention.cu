// C entry points of the attention of drafted tokens (the kernels of paged_attention_kernel.cuh in their tree form).
#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstring>

#include "decoder_host.h"
#include "paged_attention_kernel.cuh"
#include "tree_umma_kernel.cuh"

using namespace btc;

struct btc_tree_attention_s {
    btc_handle_s handle;
    TensorDesc q, k, v, table, masks, o;
    double scale = 1.0;
    int32_t window = 0;
    int32_t dp = 64, nt = 1;       // padded head size, blocks of 8 rows per item
    int64_t blocks = 1;            // items per key head
    uint32_t poll_limit = kWaitPollLimit;
};

namespace {

constexpr double kLog2E = 1.4426950408889634;
constexpr int64_t kMaxDrafts = 128;
// Tokens of a table row that count: the kernels form a length and the drafts behind it, and the end of a tile, in 32 bits.
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 256;
static_assert(kMaxTokens % kTreeTok == 0 && kMaxTokens + kMaxDrafts <= INT32_MAX, "");

size_t esize(btc_dtype_t t) { return t == BTC_F32 ? 4 : 2; }

// CTAs of the first kernel: one per SM (shared memory admits no second)
int ctas_of(const btc_tree_attention_s &op) { return op.handle.sm_count; }

int64_t slot_floats(const btc_tree_attention_s &op) { return int64_t(8 * op.nt) * op.dp + 16 * op.nt; }

bool rows_allow_vectors(const TensorDesc &t, int64_t elements)
{
    const size_t r = t.extent.size();
    if (t.stride[r - 1] != 1) return false;
    for (size_t i = 0; i + 1 < r; ++i)
        if (t.stride[i] % elements != 0) return false;
    return true;
}

// May the tcgen05 kernel run, as far as the descriptors say?  It counts places in the cache in 16 bytes and 32 bits: up to 64 GB
// between the first and the last token of a head.
bool umma_fits(const btc_tree_attention_s &op)
{
    if (op.q.dtype == BTC_F32 || op.dp > 128) return false;
    // Up to 16 rows to a key head the warp kernels read the cache once and are quicker, or nearly (tcgen05 in brackets), 8 / 16 / 24 rows:
    //   32 requests of 64 to 8192 tokens   heads of 128, bf16 53 / 93 / 146 us [82 / 82 / 82], f16 53 / 93 / 146 [92 / 92 / 92];
    //                                      heads of 64, bf16 42 / 65 / 100 [68 / 69 / 68], f16 42 / 65 / 99 [74 / 76 / 75]; of 32, bf16 42 / 63 / 97 [67 / 67 / 67]
    //   one of 1500                        heads of 128 13 / 18 / 20 [21 / 21 / 21]; of 64 12 / 16 / 17 [16 / 16 / 16]
    //   4 x 64 Ki tokens                   heads of 128, bf16 178 / 264 / 516 [231 / 231 / 228], f16 179 / 271 / 509 [254 / 245 / 244];
    //                                      heads of 64, bf16 138 / 183 / 351 [197 / 197 / 197]; of 32, f16 127 / 174 / 339 [206 / 207 / 207]
    // (Heads of 96 take what heads of 128 take.  Between 9 and 16 rows of large heads the sides are 15 % apart, in either direction.)
    if (op.q.extent[1] * (op.q.extent[2] / op.k.extent[2]) <= 16) return false;
    if (float(op.scale * kLog2E) == 0.f) return false;      // -inf for what is not visible would not survive the product
    for (const TensorDesc *t : {&op.k, &op.v}) {
        if (!rows_allow_vectors(*t, 8) || t->stride[0] < 0 || t->stride[1] < 0) return false;
        if (__int128(t->stride[0] / 8) * (t->extent[0] - 1) + __int128(t->stride[1] / 8) * (t->extent[1] - 1) >= int64_t(UINT32_MAX)) return false;
        if (t->stride[0] / 8 > UINT32_MAX || t->stride[1] / 8 > UINT32_MAX) return false;
    }
    return true;
}

int64_t umma_part_floats(const btc_tree_attention_s &op) { return op.dp == 64 ? TreeShape<64>::PART : TreeShape<128>::PART; }

size_t workspace_bytes_of(const btc_tree_attention_s &op)
{
    const size_t ctas = size_t(ctas_of(op));
    if (umma_fits(op))                     // room for either kernel: which one runs depends on the addresses of a call
        return std::max(ctas * 4 * size_t(umma_part_floats(op)) * sizeof(float), ctas * 2 * size_t(slot_floats(op)) * sizeof(float)) + ctas * 2 * sizeof(int32_t);
    return ctas * 2 * size_t(slot_floats(op)) * sizeof(float) + ctas * 2 * sizeof(int32_t);
}

template <typename T, int DP, int NT>
btc_error_t launch(const AttentionParams &p, int device, int ctas, cudaStream_t st)
{
    typedef AttentionShape<T, DP, NT> Shape;
    static std::atomic<bool> configured[64] = {};
    const int slot = device & 63;
    if (!configured[slot].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(paged_attention_kernel<T, DP, NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::SMEM) != cudaSuccess) {
            cudaGetLastError();
            return BTC_ERR_CUDA;
        }
        configured[slot].store(true, std::memory_order_relaxed);
    }
    const btc_error_t rc = launch_early(paged_attention_kernel<T, DP, NT, true>, dim3(unsigned(ctas)), Shape::WARPS * 32, Shape::SMEM, st, p);
    if (rc != BTC_SUCCESS) return rc;
    return launch_early(paged_attention_join_kernel<T, DP, NT, true>, dim3(unsigned(ctas), kJoinSlices), kJoinThreads, 0, st, p, ctas);
}

template <typename T> btc_error_t launch_typed(const btc_tree_attention_s &op, const AttentionParams &p, cudaStream_t st)
{
    const int dev = op.handle.device, ctas = ctas_of(op);
    if (op.dp == 64) return op.nt == 1 ? launch<T, 64, 1>(p, dev, ctas, st) : launch<T, 64, 2>(p, dev, ctas, st);
    if constexpr (sizeof(T) == 4)
        if (op.dp == 96) return op.nt == 1 ? launch<T, 96, 1>(p, dev, ctas, st) : launch<T, 96, 2>(p, dev, ctas, st);
    if (op.dp == 128) return op.nt == 1 ? launch<T, 128, 1>(p, dev, ctas, st) : launch<T, 128, 2>(p, dev, ctas, st);
    return launch<T, 256, 1>(p, dev, ctas, st);
}

// A tensor map of 16-bit elements with boxes of 64 elements (128 bytes, swizzled) x box[1] x ..; false where the tensor has none
bool encode_map(btc_dtype_t dtype, int rank, const void *base, const int64_t *extent, const int64_t *stride, const int32_t *box, CUtensorMap *out)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Encode encode = [] {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            fn = nullptr;
        }
        return reinterpret_cast<Encode>(fn);
    }();
    if (!encode || !aligned_to(base, 16)) return false;
    cuuint64_t dim[5], bytes[4];
    cuuint32_t b[5], steps[5] = {1, 1, 1, 1, 1};
    for (int d = 0; d < rank; ++d) {
        if (extent[d] < 1 || extent[d] > INT32_MAX || box[d] < 1 || box[d] > 256) return false;
        dim[d] = cuuint64_t(extent[d]);
        b[d] = cuuint32_t(box[d]);
        if (d == 0) continue;
        // (where there is one entry its stride is never used)
        const int64_t s = extent[d] == 1 ? 8 : stride[d];
        if (s <= 0 || s % 8 != 0 || s >= int64_t(1) << 38) return false;
        bytes[d - 1] = cuuint64_t(s) * 2;
    }
    return encode(out, dtype == BTC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, cuuint32_t(rank), const_cast<void *>(base),
                  dim, bytes, b, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct TreeMaps {
    CUtensorMap q, k, v;
};

// What of a call's tensors bulk copies can fetch: keys and values where pages are whole boxes of 8 rows or more, queries where
// 128 rows are whole drafts.
void encode_maps(const btc_tree_attention_s &op, TreeParams &tp, TreeMaps &m)
{
    std::memset(static_cast<void *>(&m), 0, sizeof m);
    const AttentionParams &p = tp.a;
    int32_t rows = kTreeTok;
    while (rows >= 8 && int64_t(p.page.d) % rows != 0) rows /= 2;
    if (rows >= 8) {
        const int32_t box[4] = {64, rows, 1, 1};
        const int64_t ek[4] = {p.dim_k, op.k.extent[1], p.key_heads, p.pages}, sk[4] = {1, p.k_slot, p.k_head, p.k_page};
        const int64_t ev[4] = {p.dim_v, op.v.extent[1], p.key_heads, p.pages}, sv[4] = {1, p.v_slot, p.v_head, p.v_page};
        if (encode_map(op.q.dtype, 4, p.k, ek, sk, box, &m.k) && encode_map(op.q.dtype, 4, p.v, ev, sv, box, &m.v)) tp.box_kv = rows;
    }
    const int32_t sharing = int32_t(p.sharing.d);
    if (p.q_d == 1 && (p.group <= kTreeRows || (sharing <= kTreeRows && kTreeRows % sharing == 0))) {
        const int32_t drafts = p.group <= kTreeRows ? p.drafts : kTreeRows / sharing;
        const int32_t box[5] = {64, sharing, drafts, 1, 1};
        const int64_t e[5] = {p.dim_k, sharing, p.drafts, p.key_heads, p.sequences}, s[5] = {1, p.q_h, p.q_t, sharing * p.q_h, p.q_n};
        if (encode_map(op.q.dtype, 5, p.q, e, s, box, &m.q)) tp.box_q = drafts;
    }
}

template <typename T, int DP, bool WIDE> btc_error_t launch_umma_rows(const TreeParams &p, const TreeMaps &maps, int device, int ctas, cudaStream_t st)
{
    static std::atomic<bool> configured[64] = {};
    const int slot = device & 63;
    if (!configured[slot].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(tree_umma_kernel<T, DP, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, TreeShape<DP>::SMEM) != cudaSuccess) {
            cudaGetLastError();
            return BTC_ERR_CUDA;
        }
        configured[slot].store(true, std::memory_order_relaxed);
    }
    const btc_error_t rc = launch_early(tree_umma_kernel<T, DP, WIDE>, dim3(unsigned(ctas)), kTreeThreads, TreeShape<DP>::SMEM, st, p, maps.q, maps.k, maps.v);
    if (rc != BTC_SUCCESS) return rc;
    const int rows = std::min(p.a.group, 2 * kTreeRows);
    return launch_early(tree_join_kernel<T, DP>, dim3(unsigned(ctas), unsigned((rows + kTreeJoinRows - 1) / kTreeJoinRows)), kTreeJoinThreads, 0, st, p, ctas);
}

template <typename T, int DP> btc_error_t launch_umma(const TreeParams &p, const TreeMaps &maps, int device, int ctas, cudaStream_t st)
{
    return p.a.group > kTreeRows ? launch_umma_rows<T, DP, true>(p, maps, device, ctas, st) : launch_umma_rows<T, DP, false>(p, maps, device, ctas, st);
}

}  // namespace

extern "C" {

btc_error_t btc_create_tree_attention(btc_handle_t handle, btc_tensor_info_t Q, btc_tensor_info_t K, btc_tensor_info_t V,
                                      btc_tensor_info_t table, btc_tensor_info_t masks, btc_tensor_info_t O, double scale,
                                      int32_t window, btc_tree_attention_t *out)
{
    if (!handle || !Q || !K || !V || !table || !masks || !O || !out) return BTC_ERR_INVALID_ARGUMENT;
    if (window < 0 || !fits_f32(scale * kLog2E)) return BTC_ERR_INVALID_ARGUMENT;
    return guarded([&]() -> btc_error_t {
        const TensorDesc &q = Q->desc, &k = K->desc, &v = V->desc, &t = table->desc, &m = masks->desc, &o = O->desc;
        if (q.extent.size() != 4 || k.extent.size() != 4 || v.extent.size() != 4 || t.extent.size() != 2 || m.extent.size() != 3 ||
            o.extent.size() != 4)
            return BTC_ERR_INVALID_ARGUMENT;
        if (!decoder_type(q.dtype) || k.dtype != q.dtype || v.dtype != q.dtype || o.dtype != q.dtype || t.dtype != BTC_I32 || m.dtype != BTC_I32)
            return BTC_ERR_NOT_SUPPORTED;
        const int64_t n = q.extent[0], drafts = q.extent[1], heads = q.extent[2], key_heads = k.extent[2];
        if (k.extent[3] != q.extent[3] || o.extent[3] != v.extent[3] || o.extent[0] != n || o.extent[1] != drafts || o.extent[2] != heads ||
            t.extent[0] != n || v.extent[0] != k.extent[0] || v.extent[1] != k.extent[1] || v.extent[2] != key_heads || heads % key_heads != 0 ||
            m.extent[0] != n || m.extent[1] != drafts || m.extent[2] != (drafts + 31) / 32)
            return BTC_ERR_EXTENT_MISMATCH;
        if (q.extent[3] > kAttnMaxDim || v.extent[3] > kAttnMaxDim || drafts > kMaxDrafts) return BTC_ERR_NOT_SUPPORTED;
        if (window > 0 && window < drafts) return BTC_ERR_INVALID_ARGUMENT;
        if (k.extent[0] > INT32_MAX || k.extent[1] > INT32_MAX || t.extent[1] > INT32_MAX || n > kAttnMaxSequences ||
            heads * drafts > INT32_MAX / 2 || heads * drafts * o.extent[3] > INT32_MAX / 2)
            return BTC_ERR_NOT_SUPPORTED;
        for (const TensorDesc *d : {&q, &k, &v, &t, &m, &o})
            if (!spans_fit(*d)) return BTC_ERR_NOT_SUPPORTED;
        if (d_may_alias(o)) return BTC_ERR_D_ALIASING;
        btc_tree_attention_s op;
        op.handle = *handle;
        op.q = q; op.k = k; op.v = v; op.table = t; op.masks = m; op.o = o;
        op.scale = scale;
        op.window = window;
        const int64_t dim = std::max(q.extent[3], v.extent[3]), rows = drafts * (heads / key_heads);
        op.dp = dim <= 64 ? 64 : (dim <= 96 && q.dtype == BTC_F32 ? 96 : (dim <= 128 ? 128 : 256));
        op.nt = rows > 8 && op.dp <= 128 ? 2 : 1;
        op.blocks = (rows + 8 * op.nt - 1) / (8 * op.nt);
        if (__int128(n) * key_heads * op.blocks > INT32_MAX) return BTC_ERR_NOT_SUPPORTED;
        // tiles of all sequences: 38 bits of the kernel's prefix sum
        if (__int128(n) * (std::min(t.extent[1] * k.extent[1], kMaxTokens) / kAttnTok + 1) >= (__int128(1) << 38)) return BTC_ERR_NOT_SUPPORTED;
        btc_tree_attention_s *kept = new (std::nothrow) btc_tree_attention_s(std::move(op));
        if (!kept) return BTC_ERR_OUT_OF_MEMORY;
        *out = kept;
        return BTC_SUCCESS;
    });
}

btc_error_t btc_destroy_tree_attention(btc_tree_attention_t *op)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    delete *op;
    *op = nullptr;
    return BTC_SUCCESS;
}

btc_error_t btc_tree_attention_workspace_size(btc_tree_attention_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = workspace_bytes_of(*op);
    return BTC_SUCCESS;
}

btc_error_t btc_tree_attention_set_attr(btc_tree_attention_t op, int32_t key, const void *value, size_t len)
{
    if (!op || !value || len != sizeof(int32_t) || key != BTC_ATTR_POLL_LIMIT) return BTC_ERR_INVALID_ARGUMENT;
    int32_t v;
    std::memcpy(&v, value, sizeof v);
    if (v < 0) return BTC_ERR_INVALID_ARGUMENT;
    op->poll_limit = uint32_t(v);
    return BTC_SUCCESS;
}

btc_error_t btc_tree_attention_execute(btc_tree_attention_t op, void *cuda_stream, const void *Q, const void *K, const void *V,
                                       const int32_t *table, const int32_t *lengths, const int32_t *masks, void *O, float *lse,
                                       void *workspace, size_t workspace_bytes, int32_t *flags)
{
    if (!op || !Q || !K || !V || !table || !lengths || !masks || !O) return BTC_ERR_INVALID_ARGUMENT;
    const size_t es = esize(op->q.dtype);
    for (const void *x : {Q, K, V, static_cast<const void *>(O)})
        if (!aligned_to(x, es)) return BTC_ERR_MISALIGNED;
    if (!aligned_to(table, 4) || !aligned_to(lengths, 4) || !aligned_to(masks, 4) || !aligned_to(lse, 4) || !aligned_to(flags, 4)) return BTC_ERR_MISALIGNED;
    if (!workspace || workspace_bytes < workspace_bytes_of(*op)) return BTC_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned_to(workspace, 256)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;

    AttentionParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.q = Q; p.k = K; p.v = V; p.o = O;
    p.table = table; p.lengths = lengths; p.masks = masks; p.lse = lse; p.flags = flags;
    const int64_t ctas = ctas_of(*op);
    p.partial = static_cast<float *>(workspace);
    p.partial_item = reinterpret_cast<int32_t *>(p.partial + ctas * 2 * slot_floats(*op));
    p.q_n = op->q.stride[0]; p.q_t = op->q.stride[1]; p.q_h = op->q.stride[2]; p.q_d = op->q.stride[3];
    p.o_n = op->o.stride[0]; p.o_t = op->o.stride[1]; p.o_h = op->o.stride[2]; p.o_d = op->o.stride[3];
    p.m_n = op->masks.stride[0]; p.m_t = op->masks.stride[1]; p.m_w = op->masks.stride[2];
    p.k_page = op->k.stride[0]; p.k_slot = op->k.stride[1]; p.k_head = op->k.stride[2]; p.k_d = op->k.stride[3];
    p.v_page = op->v.stride[0]; p.v_slot = op->v.stride[1]; p.v_head = op->v.stride[2]; p.v_d = op->v.stride[3];
    p.table_n = op->table.stride[0]; p.table_j = op->table.stride[1];
    p.sequences = int32_t(op->q.extent[0]);
    p.drafts = int32_t(op->q.extent[1]);
    p.words = int32_t(op->masks.extent[2]);
    p.heads = int32_t(op->q.extent[2]);
    p.key_heads = int32_t(op->k.extent[2]);
    p.sharing.set(p.heads / p.key_heads);
    p.group = p.drafts * (p.heads / p.key_heads);
    p.blocks = int32_t(op->blocks);
    p.dim_k = int32_t(op->k.extent[3]);
    p.dim_v = int32_t(op->v.extent[3]);
    p.pages = int32_t(op->k.extent[0]);
    p.columns = int32_t(op->table.extent[1]);
    p.window = op->window;
    p.page.set(op->k.extent[1]);
    p.room = int32_t(std::min(op->table.extent[1] * op->k.extent[1], kMaxTokens));
    const int64_t vec = int64_t(16 / es);
    p.vec_k = rows_allow_vectors(op->k, vec) && aligned_to(K, 16);
    p.vec_v = rows_allow_vectors(op->v, vec) && aligned_to(V, 16);
    p.whole_tiles = !(p.vec_k && p.vec_v) ? 0 : (op->k.extent[1] % kAttnTok == 0 ? kAttnTok : (op->k.extent[1] % 8 == 0 ? 8 : 0));
    p.vec_q = es == 2 && p.dim_k % 2 == 0 && rows_allow_vectors(op->q, 2) && aligned_to(Q, 4);
    p.scale_log2 = float(op->scale * kLog2E);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (umma_fits(*op) && p.vec_k && p.vec_v) {
        TreeParams tp;
        std::memset(static_cast<void *>(&tp), 0, sizeof tp);
        p.blocks = (p.group + 2 * kTreeRows - 1) / (2 * kTreeRows);
        tp.a = p;
        tp.poll_limit = op->poll_limit;
        tp.partial = static_cast<float *>(workspace);
        tp.partial_item = reinterpret_cast<int32_t *>(tp.partial + ctas * 4 * umma_part_floats(*op));
        tp.k_page16 = uint32_t(p.k_page / 8); tp.k_slot16 = uint32_t(p.k_slot / 8);
        tp.v_page16 = uint32_t(p.v_page / 8); tp.v_slot16 = uint32_t(p.v_slot / 8);
        tp.vec_q = rows_allow_vectors(op->q, 8) && aligned_to(Q, 16);
        tp.vec_o = rows_allow_vectors(op->o, 8) && aligned_to(O, 16);
        TreeMaps maps;
        encode_maps(*op, tp, maps);
        const int dev = op->handle.device;
        if (op->q.dtype == BTC_F16) return op->dp == 64 ? launch_umma<__half, 64>(tp, maps, dev, int(ctas), st) : launch_umma<__half, 128>(tp, maps, dev, int(ctas), st);
        return op->dp == 64 ? launch_umma<__nv_bfloat16, 64>(tp, maps, dev, int(ctas), st) : launch_umma<__nv_bfloat16, 128>(tp, maps, dev, int(ctas), st);
    }
    switch (op->q.dtype) {
    case BTC_F32: return launch_typed<float>(*op, p, st);
    case BTC_F16: return launch_typed<__half>(*op, p, st);
    default: return launch_typed<__nv_bfloat16>(*op, p, st);
    }
}

}  // extern "C"
