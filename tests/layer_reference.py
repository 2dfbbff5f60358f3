"""Plain 64-bit implementations of the residual norm, the 4-bit products and the tree attention, and the bounds that the
tests hold the kernels to (see decoder_reference.py: u is the unit roundoff of a storage type, e = 2^-24)."""
import math

import torch

from decoder_reference import E32, FLOOR, UNIT

# e4m3: half a step is 2^-4 of the value, and 2^-10 below 2^-6
E4M3_UNIT, E4M3_FLOOR = 2.0 ** -4, 2.0 ** -10


def info(api, handle, t):
    return api.TensorInfo(handle, api.dtype_code(t.dtype), t.shape, t.stride())


def check(got, want, bound):
    half = got.dtype == torch.float16
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    if half:
        # f16 rounds 65520 and more to infinity: what is certainly beyond has to be infinite, what may be is allowed to
        bound = bound.expand(want.shape)
        beyond = torch.where(want > 0, math.inf, -math.inf).double()
        may = (want.abs() + bound >= 65520.0) & (got == beyond)
        want = torch.where(may | (want.abs() - bound >= 65520.0), beyond, want)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    special = ~finite & ~torch.isnan(want)
    assert torch.equal(got[special], want[special])
    off = (got - want).abs()[finite]
    bad = off > bound.expand(want.shape)[finite] + 1e-300
    assert not bad.any(), (int(bad.sum()), float((off / (bound.expand(want.shape)[finite] + 1e-300)).max()))


# ---- residual norm ----------------------------------------------------------------------------------------

def norm_forward(x, w, r, eps):
    """(h, y) in 64 bits."""
    h = x.double() + (r.double() if r is not None else 0.0)
    n = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, n * w.double() if w is not None else n


def norm_backward(h, w, dy, dh, eps):
    """Gradients (dx = dr, dw) by the formula, and the moduli that their bounds need."""
    h, dy = h.double(), dy.double()
    inv = 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    n, g = h * inv, dy * (w.double() if w is not None else 1.0)
    dx = inv * (g - n * (g * n).mean(-1, keepdim=True)) + (dh.double() if dh is not None else 0.0)
    size = (dh.double().abs() if dh is not None else 0.0) + inv * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True))
    return dx, (dy * n).sum(0), size, (dy * n).abs().sum(0)


# The sum of squares of a row: at most 16 elements one after the other in a thread, then 10 halvings; h itself is rounded once
# (two units of its square), mean, eps and the reciprocal root (2 units of 2^-23) add 2 + 1 + 4: the root takes half of
# 16 + 10 + 2 + 3 and all of 4 < 20; h's own rounding and two products make 23.
NORM_CHAIN = 24
# backward: the same root three times (20 each, of h as it is kept), the sum of products (one rounding each) 27, four products and sums
GRAD_CHAIN = 96


def norm_grad_chain(rows):
    """dw: n (24), a product, then the rows of a CTA one after the other (at least 148 CTAs where there are so many rows), up to
    8 * 148 CTAs by 32 warps and 5 halvings."""
    return 26 + rows / 148 + 2 + 8 * 148 / 32 + 5


def e4m3_scales(y, group):
    """(scales, scale of each element) of 64-bit values."""
    d = y.shape[-1]
    size = group or d
    top = torch.stack([p.abs().amax(-1) for p in y.split(size, -1)], -1)
    s = (top / 448.0).clamp(min=2.0 ** -126)
    bad = ~torch.isfinite(torch.stack([p.abs().sum(-1) for p in y.split(size, -1)], -1))
    s = torch.where(bad, torch.tensor(math.nan, dtype=s.dtype), s)
    return s, s.repeat_interleave(size, -1)[..., :d]


def check_e4m3(codes, scales, y, group, chain):
    """Codes and scales against the 64-bit values y: the scale within `chain` + 2 roundings, each value within half a step."""
    want, each = e4m3_scales(y, group)
    check(scales, want, (chain + 2) * E32 * want.nan_to_num(0.0))
    codes = codes.cpu()
    lost = torch.isnan(each)
    assert not codes.view(torch.uint8)[lost].any()
    got = codes.double() * scales.double().cpu().repeat_interleave(group or y.shape[-1], -1)[..., :y.shape[-1]]
    y = torch.where(lost, 0.0, y)
    # the value before rounding is off by chain + 2 units itself; the step is that of the value or of the next binade
    bound = torch.maximum(E4M3_UNIT * y.abs(), E4M3_FLOOR * each) * (1 + 2.0 ** -16) + 2 * (chain + 4) * E32 * y.abs()
    check(torch.where(lost, 0.0, got), y, torch.where(lost, 0.0, bound))


# ---- 4-bit products -----------------------------------------------------------------------------------------

def linear4_weights(codes, scales, zeros, group, k):
    """(code - zero) * scale in 64 bits, [rows, k]."""
    at = torch.arange(k)
    code = (codes[:, at // 2].int() >> (4 * (at % 2))) & 15
    which = at // group if group else torch.zeros_like(at)
    zero = zeros[:, which].double() if zeros is not None else 8.0
    return (code.double() - zero) * scales.double()[:, which]


def activation(x, kind):
    if kind == "silu":
        return x * torch.sigmoid(x)
    return torch.nn.functional.gelu(x, approximate="tanh")


def linear4(x, xs, x_group, weights, kind, out):
    """(y, bound) in 64 bits.  A block of 64 k is 4 products of 16 (three times as many for fp32, whose values are three parts), in
    which the tensor core may cut off two units for each k; blocks, warps and CTAs are then added one after the other in fp32 with a
    product by the scale each, x's scale one more."""
    k = x.shape[1]
    v = x.double()
    if xs is not None:
        v = v * xs.double()[:, (torch.arange(k) // x_group) if x_group else torch.zeros(k, dtype=torch.long)]
    parts = 3 if x.dtype == torch.float32 else 1
    chain = 2 * 64 * parts + k / 32 + 64 + 8
    z, size = v @ weights.T, v.abs() @ weights.abs().T
    off = chain * E32 * size
    if kind == "none":
        return z, UNIT[out] * z.abs() + off + FLOOR[out]
    n = z.shape[1] // 2
    g, u, dg, du = z[:, :n], z[:, n:], off[:, :n], off[:, n:]
    a = activation(g, kind)
    # both activations have slopes below 1.13; exponential, division and products: 16 units, of x itself where it is tiny
    y = a * u
    return y, UNIT[out] * y.abs() + 1.13 * dg * (u.abs() + du) + (a.abs() + 1.13 * dg) * du + 16 * E32 * (g * u).abs() + FLOOR[out]


# ---- tree attention -----------------------------------------------------------------------------------------

def mask_words(sees):
    """bool [N, T, T] -> int32 words [N, T, ceil(T / 32)]."""
    n, t, _ = sees.shape
    words = -(-t // 32)
    bits = torch.zeros(n, t, words * 32, dtype=torch.int64)
    bits[:, :, :t] = sees
    packed = (bits.view(n, t, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)


def random_trees(n, t, seed, unused=0):
    """bool [N, T, T]: every draft continues an earlier one or the last cached token; the last `unused` rows of every second
    sequence hold none."""
    g = torch.Generator().manual_seed(seed)
    sees = torch.zeros(n, t, t, dtype=torch.bool)
    for i in range(n):
        for j in range(t - (unused if i % 2 == 0 else 0)):
            parent = int(torch.randint(-1, j, (1,), generator=g)) if j else -1
            if parent >= 0:
                sees[i, j] = sees[i, parent]
            sees[i, j, j] = True
    return sees


def tree_attention(q, k, v, table, lengths, sees, scale, window):
    """q [N, T, Hq, D], k / v [P, S, Hk, *] (any device, computed there); returns what decoder_reference.attention returns, with
    [N, T, Hq] in the place of [N, Hq]."""
    N, T, Hq, _ = q.shape
    P, S, Hk, _ = k.shape
    Dv, dev, room = v.shape[-1], q.device, table.shape[1] * k.shape[1]
    o = torch.zeros(N, T, Hq, Dv, dtype=torch.float64, device=dev)
    lse = torch.full((N, T, Hq), -math.inf, dtype=torch.float64, device=dev)
    size = torch.zeros(N, T, Hq, Dv, dtype=torch.float64, device=dev)
    moduli, top, count = (torch.zeros(N, T, Hq, dtype=torch.float64, device=dev) for _ in range(3))
    for n in range(N):
        cached = max(0, min(int(lengths[n]), room))
        end = min(cached + T, room)
        at = torch.arange(end)
        page = table[n].cpu().long()[at // S]
        there = (page >= 0) & (page < P)
        row = sees[n].cpu()
        drafts = row.sum(-1)
        visible = torch.zeros(T, end, dtype=torch.bool)
        visible[:, :cached] = (drafts > 0)[:, None]
        if window:
            visible[:, :cached] &= at[None, :cached] >= cached + drafts[:, None] - window
        visible[:, cached:end] = row[:, :end - cached]
        visible &= there[None, :]
        used = visible.any(0)
        if not used.any():
            continue
        at, visible = at[used], visible[:, used].to(dev)
        pg, rw = page[used].to(dev), (at % S).to(dev)
        some = visible.any(-1)
        for h in range(Hq):
            kk, vv, qq = k[pg, rw, h // (Hq // Hk)].double(), v[pg, rw, h // (Hq // Hk)].double(), q[n, :, h].double()
            s = (qq @ kk.T * scale).masked_fill(~visible, -math.inf)
            p = torch.softmax(s, -1)
            p = torch.where(some[:, None], p, 0.0)
            o[n, :, h] = p @ vv
            lse[n, :, h] = torch.logsumexp(s, -1)
            size[n, :, h] = p @ vv.abs()
            moduli[n, :, h] = torch.where(visible, qq.abs() @ kk.abs().T, 0.0).amax(-1) * abs(scale)
            top[n, :, h] = torch.where(visible, s.abs(), 0.0).amax(-1)
            count[n, :, h] = visible.sum(-1).double()
    return tuple(t.cpu() for t in (o, lse, size, moduli, top, count))
