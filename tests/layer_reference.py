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
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
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
