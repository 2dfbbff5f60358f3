"""fp32 scores are sums of fp32 quality, not the tensor core's cut-off ones.

Queries and keys between 1 and 2: all products of a score are positive, so a sum that is cut off instead of rounded falls
short every time, by a quarter of 2^-23 of the whole on average for each of the 32 steps of a head of 256 (7e-7 and more).  The
scale is a power of two in units of log2, so that it adds no error.  Bound for the mean of the relative errors of log-sum-exp
(the largest score but for the sum's logarithm): two steps are added in the tensor core, each loses less than 2^-23 of them:
2^-22; rounding errors and the dropped parts of the products have either sign: 2^-24 for their mean."""
import pytest
import torch

import helpers
from attention_on_gpu import cache, definition, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(256, 24, 8), (192, 16, 2), (128, 96, 8), (96, 40, 8)])
def test_scores_of_one_sign(heads):
    api = helpers.api()
    D, Hq, Hk = heads
    N = 64
    q, k, v, table, lengths = cache(3, N, Hq, Hk, D, 64, 16, [200 + 17 * n for n in range(N)], torch.float32)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    q = 1 + torch.rand(q.shape, generator=g, device="cuda")
    k = torch.where(torch.isnan(k), k, 1 + torch.rand(k.shape, generator=g, device="cuda"))
    scale = 2.0 ** -4 / 1.4426950408889634
    o, lse, flags = run(api, api.Handle(), q, k, v, table, lengths, scale)
    want = definition(q, k, v, table, lengths, scale, 0)
    error = (lse.double() - want[1]) / want[1]
    assert flags == 0
    assert abs(float(error.mean())) <= 2.0 ** -22 + 2.0 ** -24, float(error.mean())
