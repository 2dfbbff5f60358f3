"""The tree attention's attribute: what is refused, no GPU needed."""
import ctypes

from test_decoder_refusals_cpu import api, code, dense, handle  # noqa: F401


def test_poll_limit(api, handle):  # noqa: F811
    t = lambda *s: dense(api, handle, api.BF16, *s)  # noqa: E731
    i = lambda *s: dense(api, handle, api.I32, *s)  # noqa: E731
    op = api.TreeAttention(handle, t(3, 40, 8, 64), t(9, 16, 2, 64), t(9, 16, 2, 32), i(3, 5), i(3, 40, 2), t(3, 40, 8, 32))
    op.set_attr(api.ATTR_POLL_LIMIT, 0)
    op.set_attr(api.ATTR_POLL_LIMIT, 1 << 22)
    assert code(api, lambda: op.set_attr(api.ATTR_POLL_LIMIT, -1)) == api.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.set_attr(api.ATTR_SPLIT_K, 1)) == api.ERR_INVALID_ARGUMENT
    v, set_attr = ctypes.c_int64(1), api._lib.btc_tree_attention_set_attr
    assert set_attr(op._op, api.ATTR_POLL_LIMIT, ctypes.byref(v), 8) == api.ERR_INVALID_ARGUMENT
    assert set_attr(op._op, api.ATTR_POLL_LIMIT, None, 4) == api.ERR_INVALID_ARGUMENT
    assert set_attr(None, api.ATTR_POLL_LIMIT, ctypes.byref(v), 4) == api.ERR_INVALID_ARGUMENT
