"""What the bound of the fp32 4-bit products can see: a missing part of the inputs in an emulation of the products, on the CPU.

Bound.  x enters as three bf16 parts, exactly.  Blocks of 64 k are summed in the tensor core, a product of 16 k at a time, which may cut off the sum by
up to 2^-23 of its largest term or partial sum, always towards zero.  Only the four products of the leading parts weigh (the others are 2^-8 and 2^-16 of
them): 4 * 2^-23 of a block.  Blocks have signs of their own and so have their errors: in the norm of all outputs 2^-21 of the whole.
What follows in fp32 is 1.5 times what plain fp32 loses."""
import math

import torch

BOUND = 2.0 ** -21


def inputs(t, k, seed):
    return torch.randn(t, k, generator=torch.Generator().manual_seed(seed)) * 2


def relative(y, want):
    return float((y.double() - want).norm() / want.norm())


def plain(x, weights):
    return x @ weights.float().T


def parts(x, count):
    """The first `count` parts of x: each the leading 8 bits (16 of the word) of what those before leave."""
    out, rest = [], x.clone()
    for _ in range(count):
        lead = (rest.view(torch.int32) & -65536).view(torch.float32)
        out.append(lead.double())
        rest = rest - lead
    return out


def cut_off(x):
    """To 24 significant bits, towards zero."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.trunc(m * 2.0 ** 24), e - 24)


def emulated(x, codes, scales, group, count):
    """Products with whole numbers, 16 k at a time with the smallest parts first, cut off after each; a block's sum times its scale, added in fp32."""
    t, k = x.shape
    total = torch.zeros(t, codes.shape[0])
    pieces = parts(x, count)
    for k0 in range(0, k, 64):
        s = torch.zeros(t, codes.shape[0], dtype=torch.float64)
        for piece in reversed(pieces):
            for a in range(k0, min(k, k0 + 64), 16):
                s = cut_off(s + piece[:, a:a + 16] @ codes[:, a:a + 16].double().T)
        total += s.float() * scales[:, k0 // group][None, :]
    return total


def test_three_parts_are_the_whole_value():
    x = inputs(4, 999, 1)
    assert torch.equal(sum(parts(x, 3)), x.double())


def test_a_missing_part_exceeds_the_bound():
    for t, n, k, group in ((1, 300, 1024, 64), (5, 200, 1024, 128), (16, 100, 4096, 64)):
        g = torch.Generator().manual_seed(n)
        codes = torch.randint(-8, 8, (n, k), generator=g)
        scales = (0.5 + torch.rand(n, k // group, generator=g)) / math.sqrt(20 * k)
        weights = codes.double() * scales.double().repeat_interleave(group, 1)
        x = inputs(t, k, n)
        want = x.double() @ weights.T
        allowed = 1.5 * relative(plain(x, weights), want) + BOUND
        assert relative(emulated(x, codes, scales, group, 3), want) <= allowed
        assert relative(emulated(x, codes, scales, group, 2), want) > 10 * allowed
