"""Long chains of sums: thousands of tiles in one warp.

64 sequences of 2^18 tokens share their pages, so that the cache is small enough to hold and its tokens differ within every
sequence (the rounding errors of a sum over repeated values would repeat as well).

Bounds.  V has a mean of 1 to 2 everywhere, so each sum grows steadily and a sum that is cut off instead of rounded falls
short by half a unit of its size per addition, all in one direction: 1e-4 and more for 7000 additions.  Sums in fp32
that are rounded to nearest make independent errors of at most a unit of what is there: over n additions 6 standard
deviations are 2 sqrt(n) 2^-24 (one is 2^-24 sqrt(n / 3) / sqrt(3)); 2^-20 is left for the products of a tile, the
probabilities and the joins.  Single outputs: that, of sum p|v|, and the rounding to the type.  The mean of the relative
errors: that and 6 standard deviations of the mean of the type's roundings, of which a quarter is taken as independent."""
import math

import pytest
import torch

import helpers
from attention_on_gpu import definition, run, tiles, warps
from decoder_reference import E32, UNIT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads", [(32, 8), (96, 8)])
def test_sums_over_thousands_of_tiles(heads, dtype):
    api = helpers.api()
    N, (Hq, Hk), D, S, T = 64, heads, 64, 16, 1 << 18
    P = T // S
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    q, k = (randn(N, Hq, D) * 1.5).to(dtype), randn(P, S, Hk, D).to(dtype)
    v = (1 + torch.rand(1, 1, Hk, D, generator=g, device="cuda") + 4 * randn(P, S, Hk, D)).to(dtype)
    table = torch.randperm(P, generator=g, device="cuda").to(torch.int32).expand(N, P).contiguous()
    lengths = torch.full((N,), T, dtype=torch.int32, device="cuda")
    scale = 1 / math.sqrt(D)
    chain = tiles([T] * N, 0, Hk) / warps()
    assert chain > 5000
    o, lse, flags = run(api, api.Handle(), q, k, v, table, lengths, scale)
    want, want_lse, size, *_ = definition(q, k, v, table, lengths, scale, 0)
    sums = 2 * math.sqrt(chain) * E32 + 2.0 ** -20
    error = (o.double() - want) / want
    assert flags == 0
    assert (error.abs() <= UNIT[dtype] + sums * size / want).all(), float(error.abs().max())
    rounding = UNIT[dtype] / math.sqrt(3) if dtype != torch.float32 else 0.0
    assert abs(float(error.mean())) <= sums + 6 * rounding / math.sqrt(o.numel() / 4), float(error.mean())
    assert ((lse.double() - want_lse).abs() <= sums + 4 * E32 * want_lse.abs()).all()
