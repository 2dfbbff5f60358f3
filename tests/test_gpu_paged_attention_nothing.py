"""Sequences whose scores are all -inf have the output 0 and the log-sum-exp -inf whatever V holds, wherever their tiles
were cut: within one warp, between the warps of a CTA, between CTAs."""
import math

import pytest
import torch

import helpers
from attention_on_gpu import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head", [40, 80, 128, 256])
@pytest.mark.parametrize("shape", [(1, 5), (3, 16), (2, 33), (1, 3000), (900, 90), (40, 700)])
def test_all_scores_minus_infinity(api, shape, head, dtype):
    N, T = shape
    S, Hk, Hq = 16, 2, 6
    P = -(-T // S)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    q = torch.randn(N, Hq, head, generator=g, device="cuda")
    k, v = torch.randn(P, S, Hk, head, generator=g, device="cuda"), torch.randn(P, S, Hk, head, generator=g, device="cuda")
    q[..., 0] = 1
    k[..., 0] = -math.inf
    v.view(-1)[::3], v.view(-1)[1::7], v.view(-1)[2::5] = math.inf, math.nan, -math.inf
    table = torch.arange(P, dtype=torch.int32, device="cuda").expand(N, P).contiguous()
    lengths = torch.full((N,), T, dtype=torch.int32, device="cuda")
    o, lse, _ = run(api, api.Handle(), q.to(dtype), k.to(dtype), v.to(dtype), table, lengths, 0.1)
    assert (o == 0).all() and (lse == -math.inf).all()
