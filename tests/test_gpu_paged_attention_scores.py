"""Scores far from zero: every probability is relative to the largest score, however large that is.

The scores here are exact in fp32: queries and keys are whole numbers whose products sum to less than 2^24, and the scale
is a power of two in units of log2, so that the probabilities are powers of two.  Left are the roundings of the sums:
4 (tokens / 16 + 64) units of sum p|v| for tiles and joins (any order, the tensor core may truncate), 8 units for
exp2 and the division, and one rounding to the type; log-sum-exp: 4 units of its size and the sums'."""
import math

import pytest
import torch

import helpers
from attention_on_gpu import definition, run, tiles, warps
from decoder_reference import E32, FLOOR, UNIT

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("exponent", [-3, 0, 1, 2, 3, 4])
@pytest.mark.parametrize("shape", [(1, 4, 1, 40), (3, 4, 2, 500), (64, 32, 8, 2000)])
def test_distance_from_zero_does_not_matter(api, handle, shape, exponent, sign, dtype):
    """Largest scores of 14680064 * 2^exponent (in log2), that is up to 2^27.8, which rises in steps of 2^exponent
    along the sequence: neighbouring fp32 values are up to 16 apart there.  All sequences share their pages."""
    N, Hq, Hk, T = shape
    D, S = 64, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    P = -(-T // S)
    q = torch.zeros(N, Hq, D, device="cuda")
    q[..., :4], q[..., 4] = 2048, 1
    step = (torch.arange(P * S, device="cuda") // max(1, T // 8)).view(P, S, 1)
    k = torch.zeros(P, S, Hk, D, device="cuda")
    k[..., :3], k[..., 3], k[..., 4] = 2048, 1024, step * sign          # rises along the sequence for either sign
    q = (q * sign).to(dtype)
    k = k.to(dtype)
    v = torch.randn(P, S, Hk, D, generator=g, device="cuda").to(dtype)
    table = torch.randperm(P, generator=g, device="cuda").to(torch.int32).expand(N, P).contiguous()
    k[table[0].long()], v[table[0].long()] = k.clone(), v.clone()
    lengths = torch.full((N,), T, dtype=torch.int32, device="cuda")
    if N == 64:
        assert tiles([T] * N, 0, Hk) > 20 * warps()
    scale = 2.0 ** exponent / 1.4426950408889634
    o, lse, flags = run(api, handle, q, k, v, table, lengths, scale)
    want, want_lse, size, *_ = definition(q, k, v, table, lengths, scale, 0)
    sums = 4 * (T / 16 + 64) * E32
    bound = UNIT[dtype] * want.abs() + (sums + 8 * E32) * size + FLOOR[dtype]
    assert flags == 0
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    assert ((o.double() - want).abs() <= bound).all()
    assert ((lse.double() - want_lse).abs() <= 4 * E32 * want_lse.abs() + sums).all()


def test_finite_f16_inputs_never_give_nan(api, handle):
    """All of 128 elements at 3500, the default scale: scores near 2^27 that are all alike give the average of V."""
    N, T, D, S = 2, 300, 128, 16
    P = -(-T // S)
    for value in (3500.0, -3500.0, 6000.0, 65504.0):
        q, k = torch.full((N, 8, D), value, device="cuda").half(), torch.full((P, S, 2, D), abs(value), device="cuda").half()
        v = torch.randn(P, S, 2, D, device="cuda").half()
        table = torch.arange(P, dtype=torch.int32, device="cuda").expand(N, P).contiguous()
        lengths = torch.full((N,), T, dtype=torch.int32, device="cuda")
        o, lse, _ = run(api, handle, q, k, v, table, lengths, 1 / math.sqrt(D))
        want = v.flatten(0, 1)[:T].double().mean(0).repeat_interleave(4, 0).expand(N, 8, D)
        size = v.flatten(0, 1)[:T].double().abs().mean(0).repeat_interleave(4, 0).expand(N, 8, D)
        assert ((o.double() - want).abs() <= UNIT[torch.float16] * want.abs() + 4 * (T / 16 + 66) * E32 * size + FLOOR[torch.float16]).all()
        assert torch.isfinite(lse).all()
