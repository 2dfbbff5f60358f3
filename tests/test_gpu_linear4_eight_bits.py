"""Products of 8-bit inputs with 4-bit weights on the GPU: finite codes throughout, results into memory that holds finite values."""
import math

import pytest
import torch

import helpers
from layer_reference import check, linear4
from test_gpu_linear4 import BF16, E4M3, F16, F32, Weights, at, now, operation, pieces, work_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def codes(t, k, x_group, seed):
    """Codes up to 448 (a cast does not saturate: larger values would become NaN) and scales, as a norm leaves them."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(t, k, generator=g) * 150).clamp(-448, 448).to(E4M3)
    x[:, ::37] = torch.tensor([448.0, -448.0, 2.0 ** -9, 0.0]).to(E4M3)[torch.randint(0, 4, (t, pieces(k, 37)), generator=g)]
    assert torch.isfinite(x.float()).all()
    return x, (torch.rand(t, pieces(k, x_group), generator=g) + 0.5) / 64


def run(api, handle, w, x, xs, x_group, out, y=None):
    """y comes in full of a value that no result has."""
    if y is None:
        y = torch.full((x.shape[0], w.n), -60000.0, dtype=out, device="cuda")
    op = operation(api, handle, w, x, xs, x_group, y)
    ws, packed = work_of(op), w.pack(op)
    op.execute(now(), at(packed), at(x), at(y), XS=at(xs), workspace=at(ws), workspace_bytes=ws.numel())
    return y


def compare(y, x, xs, x_group, w, out):
    want, bound = linear4(x, xs, x_group, w.exact, w.kind, out)
    assert torch.isfinite(want).all() and torch.isfinite(y).all()
    check(y, want, bound)


@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
@pytest.mark.parametrize("out,scale,group,x_group,zeros", [
    (BF16, F16, 128, 0, False), (F16, BF16, 64, 128, True), (F32, F32, 256, 32, False), (BF16, F16, 0, 64, True), (BF16, F16, 32, 128, False),
    (F32, BF16, 128, 256, True)])
@pytest.mark.parametrize("t,n,k", [(1, 1, 1), (2, 5, 31), (8, 33, 129), (7, 777, 1001), (17, 200, 640), (33, 130, 257), (1, 4096, 4096), (40, 1000, 4160),
                                   (64, 256, 8192), (130, 520, 320)])
def test_products(api, handle, t, n, k, out, scale, group, x_group, zeros, kind):
    w = Weights(n, k, group, scale, zeros, kind, t + n + k)
    x, xs = codes(t, k, x_group, k)
    compare(run(api, handle, w, x.cuda(), xs.cuda(), x_group, out), x, xs, x_group, w, out)


@pytest.mark.parametrize("t", [3, 19, 40])
@pytest.mark.parametrize("x_group", [0, 32, 64])
def test_strides_and_alignment(api, handle, t, x_group):
    n, k = 77, 520
    w = Weights(n, k, 128, F16, True, "none", 3)
    x, xs = codes(t, k, x_group, 4)
    for extra, first, apart in ((16, 0, 1), (3, 0, 1), (0, 1, 1), (0, 0, 2), (24, 8, 1)):
        room = torch.zeros(first + t * (k * apart + extra), dtype=E4M3, device="cuda")
        v = room[first:].view(t, -1)[:, :k * apart:apart]
        v.copy_(x)
        s = torch.zeros(xs.shape[1], t + 1, device="cuda").T[:t]
        s.copy_(xs)
        y = torch.full((n, t + 2), -60000.0, dtype=BF16, device="cuda").T[:t]
        compare(run(api, handle, w, v, s, x_group, BF16, y), x, xs, x_group, w, BF16)
        assert (y.as_strided((n, 2), (t + 2, 1), y.storage_offset() + t) == torch.tensor(-60000.0).to(BF16).cuda()).all()
    one, s = x[:1].cuda().expand(t, k), xs[:1].cuda().expand(t, -1)      # one row for all tokens
    compare(run(api, handle, w, one, s, x_group, BF16), x[:1].expand(t, k), xs[:1].expand(t, -1), x_group, w, BF16)


@pytest.mark.parametrize("t", [2, 12, 48])
def test_a_lost_scale_stays_in_its_token(api, handle, t):
    """As a norm leaves a group that holds an infinity: scale NaN, codes of zero."""
    n, k = 60, 300
    w = Weights(n, k, 128, F32, False, "none", 5)
    for x_group in (0, 64):
        x, xs = codes(t, k, x_group, 6)
        xs[1, -1] = math.nan
        x[1, (xs.shape[1] - 1) * x_group:] = 0
        y = run(api, handle, w, x.cuda(), xs.cuda(), x_group, F32)
        assert torch.isnan(y[1]).all()
        keep = [i for i in range(t) if i != 1]
        compare(y[keep], x[keep], xs[keep], x_group, w, F32)
