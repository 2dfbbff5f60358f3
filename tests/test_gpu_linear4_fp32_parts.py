"""fp32 inputs of the 4-bit products keep their 24 bits: error in the norm, against plain fp32 and against what two of the three parts would give."""
import pytest
import torch

import helpers
from test_gpu_linear4 import F32, Weights, run
from test_linear4_bounds_cpu import BOUND, inputs, plain, relative

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,n,k,group,zeros", [(1, 300, 1001, 32, True), (5, 777, 1001, 128, True), (16, 200, 4096, 64, False), (40, 130, 2050, 0, True)])
def test_error_in_the_norm(t, n, k, group, zeros):
    api = helpers.api()
    w = Weights(n, k, group, F32, zeros, "none", k)
    x = inputs(t, k, k)
    y = run(api, api.Handle(), w, x.cuda(), None, 0, F32)
    want = x.double() @ w.exact.T
    assert relative(y.cpu(), want) <= 1.5 * relative(plain(x, w.exact), want) + BOUND
