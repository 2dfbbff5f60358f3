"""Plain 64-bit implementations of the decoder operators (loops and numpy / torch double, on the CPU) and the
error bounds that the tests hold the kernels to.

Bounds.  u is the unit roundoff of the storage type (2^-8 bf16, 2^-11 f16, 2^-24 fp32) and e = 2^-24.  A value computed in fp32 through a chain of n roundings and rounded once to its type is
off by at most u |y| + n e S, with S the sum of the moduli of the terms; n is stated where it is used.
"""
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# f16 subnormals: half the spacing below 2^-14
FLOOR = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
E32 = 2.0 ** -24


def rotary_forward(x, w, pos, freq, mult, interleaved, norm, eps):
    """x [T, H, D] in its storage type; returns float64 [T, H, D]."""
    x = x.double()
    if norm:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w.double()
    pairs = len(freq)
    if pairs == 0:
        return x
    angle = pos.double()[:, None, None] * torch.tensor(freq, dtype=torch.float64)
    c, s = torch.cos(angle) * mult, torch.sin(angle) * mult
    i = torch.arange(pairs)
    a_at, b_at = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    a, b = x[..., a_at], x[..., b_at]
    y = x.clone()
    y[..., a_at] = a * c - b * s
    y[..., b_at] = b * c + a * s
    return y


def rotary_backward(x, w, pos, freq, mult, interleaved, norm, eps, dy):
    """Formula of the gradients (float64): dx, dw."""
    dm = rotary_forward(dy, None, pos, [-f for f in freq], mult, interleaved, False, eps)
    if not norm:
        return dm, None
    xd = x.double()
    r = 1.0 / torch.sqrt((xd * xd).mean(-1, keepdim=True) + eps)
    n = xd * r
    g = dm * w.double() if w is not None else dm
    return r * (g - n * (g * n).mean(-1, keepdim=True)), (dm * n).sum((0, 1))
