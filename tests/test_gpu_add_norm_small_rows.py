"""The norm's backward pass of rows whose squares are the smallest that fp32 holds: gradients that fp32 holds come out finite."""
import math

import pytest
import torch

import helpers
from layer_reference import GRAD_CHAIN, check, info, norm_backward, norm_grad_chain
from decoder_reference import E32, UNIT
from test_gpu_add_norm import BF16, F32, at, now

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D", [(5, 512), (3, 1001), (2, 4096)])
def test_gradients_of_small_rows(T, D, dtype):
    """Moduli of 2^-62 and eps = 0: the reciprocal root is 2^62 and its square, times a mean of 500, beyond fp32's range."""
    api = helpers.api()
    handle = api.Handle()
    g = torch.Generator().manual_seed(D)
    sign = torch.where(torch.rand(T, D, generator=g) < 0.5, -1.0, 1.0)
    x = (sign * (1 + torch.rand(T, D, generator=g)) * 2.0 ** -62).to(dtype)
    w = (1 + 0.3 * torch.rand(D, generator=g)).to(dtype)
    dy = (sign * 400 * (1 + 0.1 * torch.randn(T, D, generator=g))).to(dtype)
    cx, cw, cdy = x.cuda(), w.cuda(), dy.cuda()
    i = info(api, handle, cx)
    op = api.AddNorm(handle, i, i, eps=0.0)
    dx, dw = torch.full_like(cx, math.nan), torch.full((D,), math.nan, device="cuda")
    ws = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")
    op.backward(now(), at(cx), at(cw), at(cdy), dX=at(dx), dW=at(dw), workspace=at(ws), workspace_bytes=ws.numel())
    edx, edw, size, moduli = norm_backward(x, w, dy, None, 0.0)
    assert torch.isfinite(edx.float()).all()
    check(dx, edx, UNIT[dtype] * edx.abs() + GRAD_CHAIN * E32 * size)
    check(dw, edw, norm_grad_chain(T) * E32 * moduli)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_whose_squares_vanish(dtype):
    """With eps = 0 the reciprocal root is infinite: infinities, NaN for zeros, scales lost; with the smallest eps zeros and values times 2^63."""
    api = helpers.api()
    handle = api.Handle()
    x = torch.full((2, 64), 2.0 ** -80, dtype=dtype, device="cuda")
    x[1] = 0
    i = info(api, handle, x)
    for eps in (0.0, 2.0 ** -126):
        y = torch.full_like(x, 7.0)
        api.AddNorm(handle, i, i, eps=eps).execute(now(), at(x), 0, at(y))
        q, s = torch.ones(2, 64, device="cuda").to(torch.float8_e4m3fn), torch.zeros(2, 2, device="cuda")
        api.AddNorm(handle, i, info(api, handle, q), S=info(api, handle, s), group=32, eps=eps).execute(now(), at(x), 0, at(q), S=at(s))
        codes = q.view(torch.uint8)
        if eps == 0.0:
            assert (y[0] == math.inf).all() and torch.isnan(y[1]).all() and torch.isnan(s).all() and not codes.any()
        else:
            assert (y[0] == 2.0 ** -17).all() and not y[1].any() and not codes[1].any()
            assert (s[1] == 2.0 ** -126).all() and (q[0].float() == 448).all()
