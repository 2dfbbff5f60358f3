// C entry points of the cache page operator (pages_kernel.cuh).
#include <algorithm>
#include <climits>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "decoder_host.h"
#include "pages_kernel.cuh"

using namespace btc;

namespace {

// One page of a tensor in parts (the smallest real type among the operation's tensors): dimensions in order of
// increasing |stride|, chained ones fused.
struct PageShape {
    int64_t part = 4;                      // bytes
    int64_t page_stride = 0;               // in parts
    std::vector<int64_t> extent, stride;   // in parts
};

}  // namespace

struct btc_pages_s {
    btc_handle_s handle;
    std::vector<PageShape> layouts;
    int64_t pages = 0, sequences = 0, columns = 0, page_tokens = 0;
    int64_t table_n = 0, table_j = 0;
};

namespace {

int64_t part_of(btc_dtype_t t) { return int64_t(dtype_size(t)) / (dtype_is_complex(t) ? 2 : 1); }

bool shape_of(const TensorDesc &t, int64_t part, PageShape &out)
{
    const int64_t per = int64_t(dtype_size(t.dtype)) / part;
    out.part = part;
    out.page_stride = t.stride[0] * per;
    std::vector<std::pair<int64_t, int64_t>> dims;      // stride, extent
    if (per > 1) dims.emplace_back(1, per);
    for (size_t i = 1; i < t.extent.size(); ++i)
        if (t.extent[i] > 1) dims.emplace_back(t.stride[i] * per, t.extent[i]);
    std::sort(dims.begin(), dims.end(), [](const std::pair<int64_t, int64_t> &a, const std::pair<int64_t, int64_t> &b) {
        return std::llabs(a.first) < std::llabs(b.first);
    });
    if (dims.empty()) dims.emplace_back(1, 1);
    for (const auto &d : dims) {
        if (!out.extent.empty() && d.first == out.stride.back() * out.extent.back()) {
            out.extent.back() *= d.second;
        } else {
            out.stride.push_back(d.first);
            out.extent.push_back(d.second);
        }
    }
    __int128 all = 1;
    for (int64_t e : out.extent) all *= e;
    return out.extent.size() <= size_t(kPagesMaxDims) && all < (__int128(1) << 31);
}

// workspace: counts, pairs, holes, movers, map, rank (int32), then begin (int64)
struct Workspace {
    size_t count, pairs, holes, movers, map, rank, begin, bytes;
};
Workspace workspace_of(const btc_pages_s &op)
{
    const size_t n = size_t(op.sequences), p = size_t(op.pages);
    Workspace w;
    w.count = 0;
    w.pairs = 64;
    w.holes = w.pairs + 2 * std::max(n, p / 2 + 1);
    w.movers = w.holes + p;
    w.map = w.movers + p / 2 + 1;
    w.rank = w.map + p;
    w.begin = (w.rank + n + 1) / 2 * 2;
    w.bytes = w.begin * 4 + n * 8;
    return w;
}

btc_error_t check_state(const btc_pages_s &op, const void *a, const void *b, const void *c, const void *flags)
{
    if (!a || !b || !c) return BTC_ERR_INVALID_ARGUMENT;
    for (const void *x : {a, b, c, flags})
        if (!aligned_to(x, 4)) return BTC_ERR_MISALIGNED;
    return op.handle.device < 0 ? BTC_ERR_CUDA : BTC_SUCCESS;
}

btc_error_t check_tensors(const btc_pages_s &op, void *const *tensors, int32_t count)
{
    if (count < 0 || count % int32_t(op.layouts.size()) != 0 || (count > 0 && !tensors)) return BTC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < count; ++i) {
        if (!tensors[i]) return BTC_ERR_INVALID_ARGUMENT;
        if (!aligned_to(tensors[i], size_t(op.layouts[size_t(i) % op.layouts.size()].part))) return BTC_ERR_MISALIGNED;
    }
    return BTC_SUCCESS;
}

void fill_state(const btc_pages_s &op, PagesParams &p)
{
    std::memset(static_cast<void *>(&p), 0, sizeof p);
    p.table_n = op.table_n; p.table_j = op.table_j;
    p.sequences = int32_t(op.sequences); p.columns = int32_t(op.columns); p.pages = int32_t(op.pages);
    p.page.set(op.page_tokens);
    p.page_tokens = int32_t(op.page_tokens);
    p.room = int32_t(std::min<int64_t>(op.columns * op.page_tokens, INT32_MAX));
}
void fill_workspace(const btc_pages_s &op, void *workspace, PagesParams &p)
{
    const Workspace w = workspace_of(op);
    int32_t *base = static_cast<int32_t *>(workspace);
    p.count = base + w.count; p.pairs = base + w.pairs; p.holes = base + w.holes; p.movers = base + w.movers;
    p.map = base + w.map; p.rank = base + w.rank;
    p.begin = reinterpret_cast<int64_t *>(base + w.begin);
}

// Launches the copies (and the renumbering when p.table is set).  `pairs_most`: as many pairs as there can be.
btc_error_t launch_copies(const btc_pages_s &op, PagesCopyParams &p, void *const *tensors, int32_t count, int64_t pairs_most,
                          cudaStream_t st)
{
    const int32_t layouts = int32_t(op.layouts.size());
    // the largest unit that every run, stride and address of this call allows (pages whose smallest stride is not one
    // move part by part)
    int64_t unit = 16;
    for (int32_t i = 0; i < layouts; ++i) {
        const PageShape &s = op.layouts[size_t(i)];
        if (s.stride[0] != 1) unit = std::min(unit, s.part);
        while (unit > s.part) {
            bool ok = s.extent[0] * s.part % unit == 0 && s.page_stride * s.part % unit == 0;
            for (size_t d = 1; d < s.stride.size(); ++d) ok = ok && s.stride[d] * s.part % unit == 0;
            for (int32_t t = i; t < count; t += layouts) ok = ok && aligned_to(tensors[t], size_t(unit));
            if (ok) break;
            unit /= 2;
        }
    }
    p.layouts = layouts;
    p.chunks = 0;
    for (int32_t i = 0; i < layouts; ++i) {
        const PageShape &s = op.layouts[size_t(i)];
        PagesLayout &l = p.layout[i];
        l.dims = int32_t(s.extent.size());
        l.page_stride = s.page_stride * s.part / unit;
        int64_t units = 1;
        for (size_t d = 0; d < s.extent.size(); ++d) {
            const int64_t e = d == 0 ? s.extent[0] * s.part / unit : s.extent[d];
            l.dim[d].set(e);
            l.dim_stride[d] = d == 0 && s.stride[0] == 1 ? 1 : s.stride[d] * s.part / unit;
            units *= e;
        }
        if (units >= (int64_t(1) << 31) - kPagesCopyThreads * kPagesCopyUnits) return BTC_ERR_NOT_SUPPORTED;
        l.units = uint32_t(units);
        l.chunks = uint32_t((units + kPagesCopyThreads * kPagesCopyUnits - 1) / (kPagesCopyThreads * kPagesCopyUnits));
        p.chunks += l.chunks;
    }
    const int64_t most = int64_t(op.handle.sm_count) * 8;
    int32_t at = 0;
    do {
        const int32_t n = std::min<int32_t>(count - at, kPagesMaxTensors / layouts * layouts);
        p.tensors = n;
        for (int32_t i = 0; i < n; ++i) p.tensor[i] = tensors[at + i];
        __int128 steps = __int128(pairs_most) * (n / layouts) * p.chunks;
        if (p.table) steps = std::max<__int128>(steps, (__int128(p.sequences) * p.columns + kPagesCopyThreads - 1) / kPagesCopyThreads);
        const int64_t blocks = int64_t(std::max<__int128>(1, std::min<__int128>(steps, most)));
        btc_error_t rc;
        switch (unit) {
        case 16: rc = launch_early(pages_copy_kernel<uint4>, unsigned(blocks), kPagesCopyThreads, 0, st, p); break;
        case 8: rc = launch_early(pages_copy_kernel<uint2>, unsigned(blocks), kPagesCopyThreads, 0, st, p); break;
        case 4: rc = launch_early(pages_copy_kernel<uint32_t>, unsigned(blocks), kPagesCopyThreads, 0, st, p); break;
        default: rc = launch_early(pages_copy_kernel<uint16_t>, unsigned(blocks), kPagesCopyThreads, 0, st, p); break;
        }
        if (rc != BTC_SUCCESS) return rc;
        p.table = nullptr;                 // renumbered once
        at += n;
    } while (at < count);
    return BTC_SUCCESS;
}

}  // namespace

extern "C" {

btc_error_t btc_create_pages(btc_handle_t handle, int32_t layouts, const btc_tensor_info_t *pages, btc_tensor_info_t table,
                             int32_t page_tokens, btc_pages_t *out)
{
    if (!handle || !pages || !table || !out || layouts < 1 || layouts > kPagesMaxLayouts || page_tokens < 1) return BTC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < layouts; ++i)
        if (!pages[i]) return BTC_ERR_INVALID_ARGUMENT;
    return guarded([&]() -> btc_error_t {
        btc_pages_s op;
        op.handle = *handle;
        const TensorDesc &t = table->desc;
        if (t.extent.size() != 2) return BTC_ERR_INVALID_ARGUMENT;
        if (t.dtype != BTC_I32 || !spans_fit(t)) return BTC_ERR_NOT_SUPPORTED;
        if (d_may_alias(t)) return BTC_ERR_D_ALIASING;
        op.page_tokens = page_tokens;
        op.sequences = t.extent[0]; op.columns = t.extent[1];
        op.table_n = t.stride[0]; op.table_j = t.stride[1];
        int64_t part = 16;
        for (int32_t i = 0; i < layouts; ++i) part = std::min(part, part_of(pages[i]->desc.dtype));
        for (int32_t i = 0; i < layouts; ++i) {
            const TensorDesc &d = pages[i]->desc;
            if (d.extent.empty()) return BTC_ERR_INVALID_ARGUMENT;
            if (i == 0) op.pages = d.extent[0];
            if (d.extent[0] != op.pages) return BTC_ERR_EXTENT_MISMATCH;
            if (!spans_fit(d)) return BTC_ERR_NOT_SUPPORTED;
            if (d_may_alias(d)) return BTC_ERR_D_ALIASING;
            PageShape s;
            if (!shape_of(d, part, s)) return BTC_ERR_NOT_SUPPORTED;
            op.layouts.push_back(std::move(s));
        }
        if (op.pages > INT32_MAX - 4 * kPagesThreads || __int128(op.pages) * page_tokens > INT32_MAX || op.columns > INT32_MAX / 2 ||
            op.sequences > (int64_t(1) << 29))
            return BTC_ERR_NOT_SUPPORTED;
        btc_pages_s *kept = new (std::nothrow) btc_pages_s(std::move(op));
        if (!kept) return BTC_ERR_OUT_OF_MEMORY;
        *out = kept;
        return BTC_SUCCESS;
    });
}

btc_error_t btc_destroy_pages(btc_pages_t *op)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    delete *op;
    *op = nullptr;
    return BTC_SUCCESS;
}

btc_error_t btc_pages_workspace_size(btc_pages_t op, size_t *bytes)
{
    if (!op || !bytes) return BTC_ERR_INVALID_ARGUMENT;
    *bytes = workspace_of(*op).bytes;
    return BTC_SUCCESS;
}

btc_error_t btc_pages_extend(btc_pages_t op, void *cuda_stream, const int32_t *new_tokens, int32_t *table, int32_t *lengths,
                             int32_t *refs, int32_t *slots, int32_t max_new, void *const *tensors, int32_t count,
                             void *workspace, size_t workspace_bytes, int32_t *flags)
{
    if (!op || !new_tokens || !slots || max_new < 1) return BTC_ERR_INVALID_ARGUMENT;
    btc_error_t rc = check_tensors(*op, tensors, count);
    if (rc != BTC_SUCCESS) return rc;
    if (!workspace || workspace_bytes < workspace_of(*op).bytes) return BTC_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned_to(workspace, 256) || !aligned_to(new_tokens, 4) || !aligned_to(slots, 4)) return BTC_ERR_MISALIGNED;
    rc = check_state(*op, table, lengths, refs, flags);
    if (rc != BTC_SUCCESS) return rc;
    PagesParams p;
    fill_state(*op, p);
    fill_workspace(*op, workspace, p);
    p.table = table; p.lengths = lengths; p.refs = refs; p.flags = flags;
    p.fresh = new_tokens; p.slots = slots; p.most = max_new;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    rc = launch_early(pages_extend_kernel, kPagesCluster, kPagesThreads, 0, st, p);
    if (rc != BTC_SUCCESS || count == 0) return rc;
    PagesCopyParams c;
    std::memset(static_cast<void *>(&c), 0, sizeof c);
    c.pairs = p.pairs; c.count = p.count; c.pages = p.pages; c.flags = flags;
    return launch_copies(*op, c, tensors, count, op->sequences, st);
}

btc_error_t btc_pages_fork(btc_pages_t op, void *cuda_stream, const int32_t *src, const int32_t *dst, int32_t count,
                           int32_t *table, int32_t *lengths, int32_t *refs, int32_t *flags)
{
    if (!op || count < 0 || (count > 0 && (!src || !dst))) return BTC_ERR_INVALID_ARGUMENT;
    if (!aligned_to(src, 4) || !aligned_to(dst, 4)) return BTC_ERR_MISALIGNED;
    const btc_error_t rc = check_state(*op, table, lengths, refs, flags);
    if (rc != BTC_SUCCESS || count == 0) return rc;
    PagesParams p;
    fill_state(*op, p);
    p.table = table; p.lengths = lengths; p.refs = refs; p.flags = flags;
    return launch_early(pages_fork_kernel, unsigned(count), 128, 0, static_cast<cudaStream_t>(cuda_stream), p, src, dst);
}

btc_error_t btc_pages_free(btc_pages_t op, void *cuda_stream, const int32_t *sequences, int32_t count, int32_t *table,
                           int32_t *lengths, int32_t *refs, int32_t *flags)
{
    if (!op || count < 0 || (count > 0 && !sequences)) return BTC_ERR_INVALID_ARGUMENT;
    if (!aligned_to(sequences, 4)) return BTC_ERR_MISALIGNED;
    const btc_error_t rc = check_state(*op, table, lengths, refs, flags);
    if (rc != BTC_SUCCESS || count == 0) return rc;
    PagesParams p;
    fill_state(*op, p);
    p.table = table; p.lengths = lengths; p.refs = refs; p.flags = flags;
    return launch_early(pages_free_kernel, unsigned(count), 128, 0, static_cast<cudaStream_t>(cuda_stream), p, sequences);
}

btc_error_t btc_pages_compact(btc_pages_t op, void *cuda_stream, int32_t *table, int32_t *refs, void *const *tensors,
                              int32_t count, void *workspace, size_t workspace_bytes, int32_t *flags)
{
    if (!op) return BTC_ERR_INVALID_ARGUMENT;
    btc_error_t rc = check_tensors(*op, tensors, count);
    if (rc != BTC_SUCCESS) return rc;
    if (!workspace || workspace_bytes < workspace_of(*op).bytes) return BTC_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned_to(workspace, 256)) return BTC_ERR_MISALIGNED;
    rc = check_state(*op, table, refs, refs, flags);
    if (rc != BTC_SUCCESS) return rc;
    PagesParams p;
    fill_state(*op, p);
    fill_workspace(*op, workspace, p);
    p.table = table; p.refs = refs; p.flags = flags;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    rc = launch_early(pages_compact_kernel, kPagesCluster, kPagesThreads, 0, st, p);
    if (rc != BTC_SUCCESS) return rc;
    PagesCopyParams c;
    std::memset(static_cast<void *>(&c), 0, sizeof c);
    c.pairs = p.pairs; c.count = p.count; c.pages = p.pages; c.flags = flags;
    c.table = table; c.map = p.map; c.live = p.count + 1;
    c.table_n = p.table_n; c.table_j = p.table_j; c.sequences = p.sequences; c.columns = p.columns;
    return launch_copies(*op, c, tensors, count, op->pages / 2, st);
}

btc_error_t btc_pages_copy(btc_pages_t op, void *cuda_stream, const int32_t *pairs, int32_t pair_count,
                           void *const *tensors, int32_t count, int32_t *flags)
{
    if (!op || pair_count < 0 || (pair_count > 0 && !pairs)) return BTC_ERR_INVALID_ARGUMENT;
    const btc_error_t rc = check_tensors(*op, tensors, count);
    if (rc != BTC_SUCCESS) return rc;
    if (!aligned_to(pairs, 4) || !aligned_to(flags, 4)) return BTC_ERR_MISALIGNED;
    if (op->handle.device < 0) return BTC_ERR_CUDA;
    if (pair_count == 0 || count == 0) return BTC_SUCCESS;
    PagesCopyParams c;
    std::memset(static_cast<void *>(&c), 0, sizeof c);
    c.pairs = pairs; c.most = pair_count; c.pages = int32_t(op->pages); c.flags = flags;
    return launch_copies(*op, c, tensors, count, pair_count, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
