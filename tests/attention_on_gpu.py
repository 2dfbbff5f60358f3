"""Attention over a paged cache in 64 bits on the GPU, for caches that the loops of decoder_reference would take too long
over, and the calls that the tests of large caches share."""
import torch


def info(api, handle, t):
    return api.TensorInfo(handle, api.dtype_code(t.dtype), t.shape, t.stride())


def cache(seed, N, Hq, Hk, D, Dv, S, lengths, dtype, window=0):
    """Queries, pages, table and lengths on the GPU; pages in random order, what no sequence sees is NaN."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-n // S) for n in lengths]
    M, P = max(1, max(need)), sum(need) + 2
    at = torch.arange(M * S, device="cuda").view(1, M, S)
    ln = torch.tensor(lengths, device="cuda")
    held = torch.arange(M, device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]
    table = torch.full((N, M), -1, dtype=torch.int32, device="cuda")
    table[held] = torch.randperm(P, generator=g, device="cuda")[:int(held.sum())].to(torch.int32)
    low = (ln - window).clamp(min=0) if window else torch.zeros_like(ln)
    seen = (at >= low.view(-1, 1, 1)) & (at < ln.view(-1, 1, 1))
    hidden = torch.ones(P, S, dtype=torch.bool, device="cuda")
    hidden[table[held].long()] = ~seen[held]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    q = (randn(N, Hq, D) * 1.5).to(dtype)
    k, v = randn(P, S, Hk, D).to(dtype), randn(P, S, Hk, Dv).to(dtype)
    k[hidden], v[hidden] = float("nan"), float("nan")
    return q, k, v, table, ln.to(torch.int32)


def definition(q, k, v, table, lengths, scale, window, dtype=torch.float64):
    """o, lse, and the scale of the error bound as decoder_reference.attention has them; `dtype` is that of the arithmetic."""
    N, Hq, D = q.shape
    S, Hk, Dv = k.shape[1], k.shape[2], v.shape[3]
    group = Hq // Hk
    make = lambda *s: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    o, size, lse = make(N, Hq, Dv), make(N, Hq, Dv), make(N, Hq) - float("inf")
    moduli, top, count = make(N, Hq), make(N, Hq), make(N, Hq)
    for n, length in enumerate(lengths.tolist()):
        low = max(0, length - window) if window else 0
        if length <= low:
            continue
        rows = table[n, low // S:-(-length // S)].long()
        cut = slice(low - low // S * S, length - low // S * S)
        kk, vv = (t[rows].flatten(0, 1)[cut].to(dtype) for t in (k, v))
        qq = q[n].to(dtype).view(Hk, group, D)
        s = torch.einsum("hgd,thd->hgt", qq, kk) * scale
        p = torch.exp(s - s.amax(-1, keepdim=True))
        total = p.sum(-1, keepdim=True)
        o[n] = (torch.einsum("hgt,thd->hgd", p, vv) / total).flatten(0, 1)
        size[n] = (torch.einsum("hgt,thd->hgd", p, vv.abs()) / total).flatten(0, 1)
        lse[n] = (s.amax(-1) + torch.log(total[..., 0])).flatten()
        moduli[n] = (torch.einsum("hgd,thd->hgt", qq.abs(), kk.abs()).amax(-1) * abs(scale)).flatten()
        top[n], count[n] = s.abs().amax(-1).flatten(), float(length - low)
    return o, lse, size, moduli, top, count


def run(api, handle, q, k, v, table, lengths, scale, window=0):
    """The library's o, lse and flags (the workspace holds garbage before)."""
    o = torch.full((*q.shape[:2], v.shape[-1]), float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    op = api.PagedAttention(handle, *(info(api, handle, t) for t in (q, k, v, table, o)), scale=scale, window=window)
    ws = torch.full((op.workspace_size(),), 0x7f, dtype=torch.uint8, device="cuda")
    op.execute(torch.cuda.current_stream().cuda_stream, q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(),
               lengths.data_ptr(), o.data_ptr(), lse=lse.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel(),
               flags=flags.data_ptr())
    torch.cuda.synchronize()
    return o, lse, flags.item()


def tiles(lengths, window, key_heads, blocks=1):
    """Tiles of 16 tokens in the whole call."""
    low = [max(0, n - window) if window else 0 for n in lengths]
    return sum(-(-n // 16) - a // 16 for n, a in zip(lengths, low)) * key_heads * blocks


def warps():
    """As many warps as a launch can have (eight to an SM; fewer where tiles are large)."""
    return 8 * torch.cuda.get_device_properties(0).multi_processor_count
