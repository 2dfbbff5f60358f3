// C entry points of the residual addition with the norm after it (add_norm_kernel.cuh).
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cstring>

#include "add_norm_kernel.cuh"
#include "decoder_host.h"

using namespace btc;

struct btc_add_norm_s {
    btc_handle_s handle;
    TensorDesc x, y, r, h, s;
    bool residual = false, e4m3 = false, x_aliases = false;
    int32_t group = 0;
    double eps = 0.0;
};

namespace {

size_t esize(btc_dtype_t t) { return t == BTC_F32 ? 4 : (t == BTC_E4M3 ? 1 : 2); }

const TensorDesc &stream_of(const btc_add_norm_s &op) { return op.residual ? op.h : op.x; }

// Do rows of this tensor allow accesses of ch elements?  (At most 16 bytes are one access.)
bool rows_allow(const TensorDesc &t, const void *at, int ch)
{
    const int64_t es = int64_t(esize(t.dtype)), bytes = std::min<int64_t>(16, ch * es);
    return (t.extent[1] == 1 || t.stride[1] == 1) && (t.extent[0] == 1 || t.stride[0] * es % bytes == 0) && aligned_to(at, size_t(bytes));
}

// How a row is laid over threads: `chunks` of ch elements, `count` per thread; 32 threads: a warp to a row
struct Shape {
    int ch, count, threads;
    int32_t chunks;
};

// Many rows: two chunks a thread (16 elements of a 16-bit type, 8 of fp32), few: one, so that a row is spread over as many
// threads as there are; rows that fit a warp take a warp.  A row needs at most 1024 threads.
Shape shape_for(const btc_add_norm_s &op, bool vectors, int usual)
{
    Shape f;
    f.ch = vectors ? int(16 / esize(op.x.dtype)) : 1;
    const int64_t dim = op.x.extent[1];
    f.chunks = int32_t((dim + f.ch - 1) / f.ch);
    const int most = f.ch == 8 ? 2 : (f.ch == 4 ? 4 : 16);
    f.count = f.ch == 1 ? (f.chunks <= 4 * 1024 ? 4 : 16) : std::min(usual, most);
    while (f.count < most && f.chunks > f.count * 1024) f.count *= 2;
    const int64_t need = (f.chunks + f.count - 1) / f.count;
    f.threads = need <= 32 ? 32 : int((need + 31) / 32 * 32);
    return f;
}

template <typename TX, typename TR, bool E4M3, int CH, int C>
btc_error_t launch_forward(const AddNormParams &p, const Shape &f, cudaStream_t st)
{
    if (f.threads == 32)
        return launch_early(add_norm_forward_kernel<TX, TR, E4M3, CH, C, true>, dim3(unsigned((p.rows + kNormWarpRows - 1) / kNormWarpRows)),
                            32 * kNormWarpRows, 0, st, p);
    return launch_early(add_norm_forward_kernel<TX, TR, E4M3, CH, C, false>, dim3(unsigned(p.rows)), unsigned(f.threads), 0, st, p);
}
template <typename TX, typename TR, bool E4M3> btc_error_t forward(const AddNormParams &p, const Shape &f, cudaStream_t st)
{
    constexpr int CH = 16 / int(sizeof(TX));
    if (f.ch == 1) return f.count == 4 ? launch_forward<TX, TR, E4M3, 1, 4>(p, f, st) : launch_forward<TX, TR, E4M3, 1, 16>(p, f, st);
    if (f.count == 1) return launch_forward<TX, TR, E4M3, CH, 1>(p, f, st);
    if constexpr (CH == 4)
        if (f.count == 4) return launch_forward<TX, TR, E4M3, CH, 4>(p, f, st);
    return launch_forward<TX, TR, E4M3, CH, 2>(p, f, st);
}

template <typename TX, typename TR, int CH, int C>
btc_error_t launch_backward(const AddNormParams &p, const Shape &f, unsigned ctas, cudaStream_t st)
{
    if (f.threads == 32) return launch_early(add_norm_backward_kernel<TX, TR, CH, C, true>, dim3(ctas), 32 * kNormWarpRows, 0, st, p);
    return launch_early(add_norm_backward_kernel<TX, TR, CH, C, false>, dim3(ctas), unsigned(f.threads), 0, st, p);
}
template <typename TX, typename TR> btc_error_t backward(const AddNormParams &p, const Shape &f, unsigned ctas, cudaStream_t st)
{
    constexpr int CH = 16 / int(sizeof(TX));
    if (f.ch == 1) return f.count == 4 ? launch_backward<TX, TR, 1, 4>(p, f, ctas, st) : launch_backward<TX, TR, 1, 16>(p, f, ctas, st);
    if (f.count == 1) return launch_backward<TX, TR, CH, 1>(p, f, ctas, st);
    if constexpr (CH == 4)
        if (f.count == 4) return launch_backward<TX, TR, CH, 4>(p, f, ctas, st);
    return launch_backward<TX, TR, CH, 2>(p, f, ctas, st);
}

// CTAs of the backward pass: what runs at once with 64 registers a thread, and no more than there are rows to take (four rows to a CTA
// at least, for fewer partial sums of dW, is slower where there are few: 777 rows of 1001 in fp32 14.2 -> 18.0 us)
unsigned backward_ctas(const btc_add_norm_s &op, const Shape &f)
{
    const int64_t per_sm = f.threads == 32 ? 8 : std::max(1, 1024 / f.threads);
    const int64_t units = f.threads == 32 ? (op.x.extent[0] + kNormWarpRows - 1) / kNormWarpRows : op.x.extent[0];
    return unsigned(std::min(units, op.handle.sm_count * per_sm));
}

size_t workspace_bytes_of(const btc_add_norm_s &op)
{
    // whichever accesses the addresses of a call allow
    size_t most = 0;
    for (bool vectors : {false, true}) {
        const Shape f = shape_for(op, vectors, 1);
        most = std::max(most, size_t(backward_ctas(op, f)));
    }
    return most * size_t(op.x.extent[1]) * sizeof(float);
}

void set_rows(const TensorDesc &t, int64_t &row, int64_t &element)
{
    row = t.stride[0];
    element = t.stride[1];
}

}  // namespace

extern "C" {

btc_error_t btc_create_add_norm(btc_handle_t handle, btc_tensor_info_t X, btc_tensor_info_t R, btc_tensor_info_t H,
                                btc_tensor_info_t Y, btc_tensor_info_t S, int32_t group, double eps, btc_add_norm_t *out)
{
    if (!handle || !X || !Y || !out || (R == nullptr) != (H == nullptr)) return BTC_ERR_INVALID_ARGUMENT;
    if (!(eps == 0.0 || (eps >= double(FLT_MIN) && fits_f32(eps)))) return BTC_ERR_INVALID_ARGUMENT;
    return guarded([&]() -> btc_error_t {
        btc_add_norm_s op;
        op.handle = *handle;
        op.x = X->desc; op.y = Y->desc;
        op.residual = R != nullptr;
        op.e4m3 = op.y.dtype == BTC_E4M3;
        op.group = group;
        op.eps = eps;
        if (op.e4m3 != (S != nullptr)) return BTC_ERR_INVALID_ARGUMENT;
        if (group != 0 && (!op.e4m3 || (group != 32 && group != 64 && group != 128))) return BTC_ERR_INVALID_ARGUMENT;
        if (R) { op.r = R->desc; op.h = H->desc; }
        if (S) op.s = S->desc;
        for (const TensorDesc *t : {&op.x, &op.y, R ? &op.r : nullptr, H ? &op.h : nullptr, S ? &op.s : nullptr})
            if (t && t->extent.size() != 2) return BTC_ERR_INVALID_ARGUMENT;
        if (!decoder_type(op.x.dtype) || (!op.e4m3 && op.y.dtype != op.x.dtype)) return BTC_ERR_NOT_SUPPORTED;
        if (R && (op.r.dtype != op.h.dtype || (op.r.dtype != op.x.dtype && op.r.dtype != BTC_F32))) return BTC_ERR_NOT_SUPPORTED;
        if (S && op.s.dtype != BTC_F32) return BTC_ERR_NOT_SUPPORTED;
        const int64_t rows = op.x.extent[0], dim = op.x.extent[1];
        if (op.y.extent != op.x.extent || (R && (op.r.extent != op.x.extent || op.h.extent != op.x.extent))) return BTC_ERR_EXTENT_MISMATCH;
        if (S && (op.s.extent[0] != rows || op.s.extent[1] != (group ? (dim + group - 1) / group : 1))) return BTC_ERR_EXTENT_MISMATCH;
        if (dim > kNormMaxDim || rows > INT32_MAX) return BTC_ERR_NOT_SUPPORTED;
        for (const TensorDesc *t : {&op.x, &op.y, R ? &op.r : nullptr, H ? &op.h : nullptr, S ? &op.s : nullptr})
            if (t && !spans_fit(*t)) return BTC_ERR_NOT_SUPPORTED;
        if (d_may_alias(op.y) || (H && d_may_alias(op.h)) || (S && d_may_alias(op.s))) return BTC_ERR_D_ALIASING;
        op.x_aliases = d_may_alias(op.x);
        btc_add_norm_s *kept = new (std::nothrow) btc_add_norm_s(std::move(op));
        if (!kept) return BTC_ERR_OUT_OF_MEMORY;
        *out = kept;
        return BTC_SUCCESS;
    });
}

btc_error_t btc_destroy_add_norm(btc_add_norm_t *op)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    delete *op;
    *op = nullptr;
    return BTC_SUCCESS;
}

btc_error_t btc_add_norm_workspace_size(btc_add_norm_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = op->e4m3 ? 0 : workspace_bytes_of(*op);
    return BTC_SUCCESS;
}

btc_error_t btc_add_norm_execute(btc_add_norm_t op, void *cuda_stream, const void *X, const void *W, const void *R, void *H,
                                 void *Y, float *S)
{
    if (!op || !X || !Y) return BTC_ERR_INVALID_ARGUMENT;
    if ((R != nullptr) != op->residual || (H != nullptr) != op->residual || (S != nullptr) != op->e4m3) return BTC_ERR_INVALID_ARGUMENT;
    const size_t es = esize(op->x.dtype), rs = op->residual ? esize(op->r.dtype) : 1;
    if (!aligned_to(X, es) || !aligned_to(W, es) || !aligned_to(Y, esize(op->y.dtype)) || !aligned_to(R, rs) || !aligned_to(H, rs) ||
        !aligned_to(S, 4))
        return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;
    const int ch = int(16 / es);
    const bool vectors = op->x.extent[1] % ch == 0 && rows_allow(op->x, X, ch) && rows_allow(op->y, Y, ch) && aligned_to(W, 16) &&
                         (!op->residual || (rows_allow(op->r, R, ch) && rows_allow(op->h, H, ch)));
    const Shape f = shape_for(*op, vectors, op->x.extent[0] >= 2 * op->handle.sm_count ? 2 : 1);
    AddNormParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.x = X; p.w = W; p.r = R; p.h = H; p.y = Y; p.s = S;
    set_rows(op->x, p.x_t, p.x_d);
    set_rows(op->y, p.y_t, p.y_d);
    if (op->residual) {
        set_rows(op->r, p.r_t, p.r_d);
        set_rows(op->h, p.h_t, p.h_d);
    }
    if (op->e4m3) set_rows(op->s, p.s_t, p.s_g);
    p.rows = op->x.extent[0];
    p.dim = int32_t(op->x.extent[1]);
    p.chunks = f.chunks;
    p.group = op->group;
    p.inv_dim = 1.f / float(p.dim);
    p.eps = float(op->eps);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool wide = op->residual && op->r.dtype != op->x.dtype;
    switch (op->x.dtype) {
    case BTC_F32: return op->e4m3 ? forward<float, float, true>(p, f, st) : forward<float, float, false>(p, f, st);
    case BTC_F16:
        if (wide) return op->e4m3 ? forward<__half, float, true>(p, f, st) : forward<__half, float, false>(p, f, st);
        return op->e4m3 ? forward<__half, __half, true>(p, f, st) : forward<__half, __half, false>(p, f, st);
    default:
        if (wide) return op->e4m3 ? forward<__nv_bfloat16, float, true>(p, f, st) : forward<__nv_bfloat16, float, false>(p, f, st);
        return op->e4m3 ? forward<__nv_bfloat16, __nv_bfloat16, true>(p, f, st) : forward<__nv_bfloat16, __nv_bfloat16, false>(p, f, st);
    }
}

btc_error_t btc_add_norm_backward(btc_add_norm_t op, void *cuda_stream, const void *H, const void *W, const void *dY,
                                  const void *dH, void *dX, void *dR, float *dW, void *workspace, size_t workspace_bytes)
{
    if (!op || !H || !dY || (!dX && !dR)) return BTC_ERR_INVALID_ARGUMENT;
    if (op->e4m3) return BTC_ERR_NOT_SUPPORTED;
    if (!op->residual && (dH || dR)) return BTC_ERR_INVALID_ARGUMENT;
    if (dW && !W) return BTC_ERR_INVALID_ARGUMENT;
    if (dX && op->x_aliases) return BTC_ERR_D_ALIASING;
    const TensorDesc &kept = stream_of(*op);
    const size_t es = esize(op->x.dtype), rs = esize(kept.dtype);
    if (!aligned_to(H, rs) || !aligned_to(dH, rs) || !aligned_to(dR, rs) || !aligned_to(W, es) || !aligned_to(dY, es) || !aligned_to(dX, es) ||
        !aligned_to(dW, 4))
        return BTC_ERR_MISALIGNED;
    if (dW && (!workspace || workspace_bytes < workspace_bytes_of(*op))) return BTC_ERR_WORKSPACE_TOO_SMALL;
    if (dW && !aligned_to(workspace, 256)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;
    const int ch = int(16 / es);
    const bool vectors = op->x.extent[1] % ch == 0 && rows_allow(op->y, dY, ch) && rows_allow(kept, H, ch) && aligned_to(W, 16) &&
                         (!dX || rows_allow(op->x, dX, ch)) && (!dH || rows_allow(kept, dH, ch)) && (!dR || rows_allow(kept, dR, ch));
    const Shape f = shape_for(*op, vectors, 1);
    AddNormParams p;
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.x = H; p.w = W; p.dy = dY; p.dh = dH; p.y = dX; p.h = dR;
    p.partial = dW ? static_cast<float *>(workspace) : nullptr;
    set_rows(kept, p.x_t, p.x_d);
    set_rows(kept, p.dh_t, p.dh_d);
    set_rows(kept, p.h_t, p.h_d);
    set_rows(op->y, p.dy_t, p.dy_d);
    set_rows(op->x, p.y_t, p.y_d);
    p.rows = op->x.extent[0];
    p.dim = int32_t(op->x.extent[1]);
    p.chunks = f.chunks;
    p.inv_dim = 1.f / float(p.dim);
    p.eps = float(op->eps);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const unsigned ctas = backward_ctas(*op, f);
    const bool wide = kept.dtype != op->x.dtype;
    btc_error_t rc;
    switch (op->x.dtype) {
    case BTC_F32: rc = backward<float, float>(p, f, ctas, st); break;
    case BTC_F16: rc = wide ? backward<__half, float>(p, f, ctas, st) : backward<__half, __half>(p, f, ctas, st); break;
    default: rc = wide ? backward<__nv_bfloat16, float>(p, f, ctas, st) : backward<__nv_bfloat16, __nv_bfloat16>(p, f, ctas, st); break;
    }
    if (rc != BTC_SUCCESS || !dW) return rc;
    return launch_early(add_norm_weight_gradient_kernel, dim3(unsigned((p.dim + 31) / 32)), 1024, 0, st, static_cast<const float *>(p.partial), int(ctas), int(p.dim), dW);
}

}  // extern "C"
