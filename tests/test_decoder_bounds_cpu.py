"""What the bounds of the attention tests can see: mistakes planted in emulations of the products and sums, on the CPU."""
import math

import torch

E32 = 2.0 ** -24


def tf32_parts(x):
    """x = hi + lo as the tensor core takes them: hi rounded to 11 significant bits, lo cut off to 11."""
    bits = x.view(torch.int32)
    hi = ((bits + 0x1000) & ~0x1fff).view(torch.float32)
    lo = ((x - hi).view(torch.int32) & ~0x1fff).view(torch.float32)
    return hi.double(), lo.double()


def product(a, b, parts):
    """a b^T from one or three products of TF32 parts (sums in 64 bits)."""
    ah, al = tf32_parts(a)
    bh, bl = tf32_parts(b)
    return ah @ bh.T + (al @ bh.T + ah @ bl.T if parts == 3 else 0)


def test_missing_low_parts_exceed_the_fp32_bound():
    """The norm of the error against 1.5 times plain fp32's and 2^-24, for both products of the attention."""
    g = torch.Generator().manual_seed(1)
    for dim, tokens in ((64, 300), (96, 5000), (128, 2500), (256, 6000)):
        q, k, v = torch.randn(24, dim, generator=g) * 1.5, torch.randn(tokens, dim, generator=g), torch.randn(tokens, dim, generator=g)
        want = torch.softmax(q.double() @ k.double().T / math.sqrt(dim), -1) @ v.double()
        plain = torch.softmax(q @ k.T / math.sqrt(dim), -1) @ v
        error = lambda y: float((y.double() - want).norm() / want.norm())  # noqa: E731
        allowed = 1.5 * error(plain) + E32

        def emulated(scores, values):
            p = torch.softmax(product(q, k, scores) / math.sqrt(dim), -1).float()
            return product(p, v.T.contiguous(), values)

        assert error(emulated(3, 3)) <= allowed
        assert error(emulated(1, 3)) > 10 * allowed
        assert error(emulated(3, 1)) > 10 * allowed


def cut_off(x):
    """To 24 significant bits, towards zero."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.trunc(m * 2.0 ** 24), e - 24)


def test_cut_off_sums_exceed_the_bounds_of_long_chains():
    """7000 additions of a steady growth: the mean error against the bounds of single fp32 sums and of 16-bit outputs."""
    n, outputs = 7000, 2000
    g = torch.Generator().manual_seed(2)
    total, cut, rounded = torch.zeros(outputs).double(), torch.zeros(outputs).double(), torch.zeros(outputs)
    for _ in range(n):
        x = (24 + 16 * torch.randn(outputs, generator=g)).double()
        total += x
        cut = cut_off(cut + x)
        rounded += x.float()
    sums = 2 * math.sqrt(n) * E32 + 2.0 ** -20
    bf16 = sums + 6 * 2.0 ** -8 / math.sqrt(3) / math.sqrt(32 * 64 * 64 / 4)
    assert abs(float(((rounded.double() - total) / total).mean())) < E32 * math.sqrt(n)
    assert ((rounded.double() - total) / total).abs().max() <= sums
    shortfall = -float(((cut - total) / total).mean())
    assert shortfall > 1.2 * bf16 > 1.2 * sums


def test_cut_off_scores_exceed_the_bound_of_one_sign():
    """32 steps of 8 positive products each, cut off at every step or rounded after every second one."""
    g = torch.Generator().manual_seed(3)
    a, b = 1 + torch.rand(4000, 32, 8, generator=g), 1 + torch.rand(4000, 32, 8, generator=g)
    steps = (a.double() * b.double()).sum(-1)
    total = steps.sum(-1)
    cut, rounded = torch.zeros(4000).double(), torch.zeros(4000)
    for i in range(0, 32, 2):
        cut = cut_off(cut_off(cut + steps[:, i]) + steps[:, i + 1])
        rounded += cut_off(cut_off(steps[:, i]) + steps[:, i + 1]).float()
    bound = 2.0 ** -22 + 2.0 ** -24
    assert -float(((cut - total) / total).mean()) > bound
    assert abs(float(((rounded.double() - total) / total).mean())) <= bound
