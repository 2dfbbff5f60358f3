"""The largest inputs that the 4-bit products take: moduli up to 2^117, where 64 products with whole numbers of 15 still fit fp32."""
import pytest
import torch

import helpers
from layer_reference import check, linear4, linear4_weights
from test_gpu_linear4 import BF16, F32, Weights, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [1, 12, 40])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_largest_inputs(t, group, dtype):
    api = helpers.api()
    n, k = 50, 520
    w = Weights(n, k, group, F32, True, "none", 7)
    w.codes[0], w.zeros[0] = 255, 0                      # every factor is 15
    w.scales *= 2.0 ** -20
    w.exact = linear4_weights(w.codes, w.scales, w.zeros, group, k)
    x = ((torch.rand(t, k, generator=torch.Generator().manual_seed(1)) - 0.5) * 2.0 ** 118).to(dtype)
    x[0] = 2.0 ** 117                                    # all of one sign
    y = run(api, api.Handle(), w, x.cuda(), None, 0, F32)
    want, bound = linear4(x, None, 0, w.exact, "none", F32)
    assert torch.isfinite(want.float()).all() and torch.isfinite(y).all()
    check(y, want, bound)
