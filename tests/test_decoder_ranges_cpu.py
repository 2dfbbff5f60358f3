"""Numbers given as doubles that the kernels' fp32 arithmetic cannot hold are refused at creation (they became infinities or
zeros there: outputs of NaN for finite inputs)."""
import pytest

from test_decoder_refusals_cpu import code, dense


@pytest.fixture(scope="module")
def api():
    from paper_2601_07827_b200 import build
    build.build()
    from paper_2601_07827_b200 import api as _api
    return _api


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def test_scale(api, handle):
    t = lambda *s: dense(api, handle, api.BF16, *s)  # noqa: E731
    args = t(3, 8, 64), t(9, 16, 2, 64), t(9, 16, 2, 32), dense(api, handle, api.I32, 3, 5), t(3, 8, 32)
    for scale in (1e39, -1e39, 3e38):                                    # (3e38 log2(e) is beyond fp32)
        assert code(api, lambda: api.PagedAttention(handle, *args, scale=scale)) == api.ERR_INVALID_ARGUMENT
    for scale in (2e38, -2e38, 1.0, 0.0, 1e-50):
        api.PagedAttention(handle, *args, scale=scale)


def test_multiplier_and_eps(api, handle):
    x = dense(api, handle, api.F32, 4, 2, 8)
    make = lambda **k: api.Rotary(handle, [0.1], x, x, **k)  # noqa: E731
    for bad in (dict(multiplier=1e39), dict(multiplier=-4e38), dict(norm=True, eps=1e-50), dict(norm=True, eps=1e-39), dict(norm=True, eps=1e39)):
        assert code(api, lambda: make(**bad)) == api.ERR_INVALID_ARGUMENT
    for good in (dict(multiplier=-3e38), dict(multiplier=0.0), dict(norm=True, eps=0.0), dict(norm=True, eps=1.2e-38), dict(norm=True, eps=1.0),
                 dict(norm=False, eps=1e-50)):                           # eps is not used without a norm
        make(**good)
