"""What the decoder operators refuse, and their host-side helpers: no GPU needed."""
import math

import pytest


@pytest.fixture(scope="module")
def api():
    from paper_2601_07827_b200 import build
    build.build()
    from paper_2601_07827_b200 import api as _api
    return _api


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def code(api, fn):
    with pytest.raises(api.BtcError) as e:
        fn()
    return e.value.code


def dense(api, h, dtype, *shape, strides=None):
    if strides is None:
        strides, s = [], 1
        for x in reversed(shape):
            strides.insert(0, s)
            s *= x
    return api.TensorInfo(h, dtype, shape, strides)


def test_decoder_types_are_refused_by_contractions(api, handle):
    for dt in (api.F16, api.BF16, api.I32):
        a = dense(api, handle, dt, 4, 4)
        assert code(api, lambda: api.Contraction(handle, a, "ik", a, "kj", None, None, a, "ij", alpha=None)) == api.ERR_NOT_SUPPORTED
        assert code(api, lambda: api.Elementwise(handle, a, "ij", None, a, "ji", alpha=None, beta=None)) == api.ERR_NOT_SUPPORTED


def test_rotary_refusals(api, handle):
    E, B = api, api.BF16
    t = lambda *s, dt=B, st=None: dense(api, handle, dt, *s, strides=st)  # noqa: E731
    f = [0.1] * 4
    make = lambda *a, **k: code(api, lambda: api.Rotary(handle, *a, **k))  # noqa: E731
    assert make(f, t(4, 2, 8, dt=E.F64), t(4, 2, 8, dt=E.F64)) == E.ERR_NOT_SUPPORTED
    assert make(f, t(4, 2, 8), t(4, 2, 8, dt=E.F16)) == E.ERR_NOT_SUPPORTED
    assert make(f, t(4, 2, 8), t(4, 3, 8)) == E.ERR_EXTENT_MISMATCH
    assert make(f, t(4, 2, 8), t(5, 2, 8)) == E.ERR_EXTENT_MISMATCH
    assert make(f, t(4, 2, 6), t(4, 2, 6)) == E.ERR_INVALID_ARGUMENT            # more pairs than the head has
    assert make(f, t(4, 2, 264), t(4, 2, 264)) == E.ERR_NOT_SUPPORTED
    assert make(f, t(8, 8), t(8, 8)) == E.ERR_INVALID_ARGUMENT
    assert make(f, t(2, 3, 2, 8), t(2, 3, 2, 8)) == E.ERR_INVALID_ARGUMENT
    assert make(f, t(6, 2, 8), t(2, 3, 2, 8)) == E.ERR_INVALID_ARGUMENT         # queries go to no pages
    assert make(f, t(4, 2, 8), t(4, 2, 8, st=(16, 0, 1))) == E.ERR_D_ALIASING
    assert make(f, t(4, 2, 8), t(4, 2, 8), Xk=t(4, 1, 8)) == E.ERR_INVALID_ARGUMENT
    assert make(f, t(4, 2, 8), t(4, 2, 8), Xk=t(4, 1, 16), Yk=t(4, 1, 16)) == E.ERR_EXTENT_MISMATCH
    assert make(f, t(4, 2, 8), t(4, 2, 8), Xk=t(4, 1, 8), Yk=t(9, 16, 1, 8), Xv=t(4, 1, 8), Yv=t(9, 8, 1, 8)) == E.ERR_EXTENT_MISMATCH
    assert make(f, t(4, 2, 8), t(4, 2, 8), Xk=t(4, 1, 8), Yk=t(1 << 28, 16, 1, 8)) == E.ERR_NOT_SUPPORTED
    assert make(f, t(4, 2, 8, st=(1 << 62, 8, 1)), t(4, 2, 8)) == E.ERR_NOT_SUPPORTED
    assert make([float("nan")], t(4, 2, 8), t(4, 2, 8)) == E.ERR_INVALID_ARGUMENT
    assert make(f, t(4, 2, 8), t(4, 2, 8), multiplier=float("inf")) == E.ERR_INVALID_ARGUMENT
    assert make(f, t(4, 2, 8), t(4, 2, 8), norm=True, eps=-1.0) == E.ERR_INVALID_ARGUMENT

    op = api.Rotary(handle, f, t(4, 2, 8), t(4, 2, 8), t(4, 1, 8), t(9, 16, 1, 8))
    run = lambda *a, **k: code(api, lambda: op.execute(0, *a, **k))  # noqa: E731
    assert run(0, 0, 0, 256, 512, 256, 512, slots=256) == E.ERR_INVALID_ARGUMENT     # no positions
    assert run(256, 0, 0, 256, 512, 256, 512) == E.ERR_INVALID_ARGUMENT              # no slots
    assert run(256, 0, 0, 256, 512, 0, 0, slots=256) == E.ERR_INVALID_ARGUMENT       # no keys
    assert run(256, 256, 0, 256, 512, 256, 512, slots=256) == E.ERR_INVALID_ARGUMENT  # a weight without a norm
    assert run(256, 0, 0, 257, 512, 256, 512, slots=256) == E.ERR_MISALIGNED
    assert run(258, 0, 0, 256, 512, 256, 512, slots=256) == E.ERR_MISALIGNED
    assert code(api, lambda: op.backward(0, 256, 0, 0, 256, 256, 256, 256, 256, 256)) == E.ERR_NOT_SUPPORTED   # paged

    op = api.Rotary(handle, f, t(4, 2, 8), t(4, 2, 8), norm=True)
    back = lambda *a, **k: code(api, lambda: op.backward(0, *a, **k))  # noqa: E731
    assert op.workspace_size() > 0
    assert back(256, 0, 0, 0, 256, 256) == E.ERR_INVALID_ARGUMENT                    # a norm needs X
    assert back(256, 0, 0, 256, 256, 256, dWq=256) == E.ERR_WORKSPACE_TOO_SMALL
    assert back(256, 0, 0, 256, 256, 256, dWq=256, workspace=128, workspace_bytes=1 << 30) == E.ERR_MISALIGNED
    assert back(256, 0, 0, 256, 256, 256, dWq=258, workspace=256, workspace_bytes=1 << 30) == E.ERR_MISALIGNED
    plain = api.Rotary(handle, f, t(4, 2, 8), t(4, 2, 8))
    assert plain.workspace_size() == 0
    assert code(api, lambda: plain.backward(0, 256, 0, 0, 0, 256, 256, dWq=256)) == E.ERR_INVALID_ARGUMENT


def test_rotary_frequencies(api):
    f, m = api.rotary_frequencies(8)
    assert m == 1.0 and f == [10000.0 ** (-i / 4) for i in range(4)]
    g, m = api.rotary_frequencies(8, scaling="linear", factor=4.0)
    assert m == 1.0 and all(math.isclose(a, b / 4) for a, b in zip(g, f))
    g, m = api.rotary_frequencies(8, scaling="base", factor=4.0)
    assert m == 1.0 and g[0] == f[0] and math.isclose(g[-1], f[-1] / 4)
    g, m = api.rotary_frequencies(64, scaling="bands", factor=8.0, original_length=4096)
    f, _ = api.rotary_frequencies(64)
    assert g[0] == f[0] and math.isclose(g[-1], f[-1] / 8) and math.isclose(m, 0.1 * math.log(8) + 1)
    assert all(a / 8 * (1 - 1e-12) <= b <= a for a, b in zip(f, g))
    for bad in (dict(rotary_dim=7), dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, scaling="other")):
        with pytest.raises(ValueError):
            api.rotary_frequencies(**bad)


def test_paged_attention_refusals(api, handle):
    E, B = api, api.BF16
    t = lambda *s, dt=B, st=None: dense(api, handle, dt, *s, strides=st)  # noqa: E731
    i = lambda *s: dense(api, handle, api.I32, *s)  # noqa: E731
    make = lambda *a, **k: code(api, lambda: api.PagedAttention(handle, *a, **k))  # noqa: E731
    q, k, v, tab, o = t(3, 8, 64), t(9, 16, 2, 64), t(9, 16, 2, 32), i(3, 5), t(3, 8, 32)
    op = api.PagedAttention(handle, q, k, v, tab, o)
    assert op.workspace_size() > 0
    assert make(t(3, 8, 64, dt=E.F64), k, v, tab, o) == E.ERR_NOT_SUPPORTED
    assert make(q, t(9, 16, 2, 64, dt=E.F16), v, tab, o) == E.ERR_NOT_SUPPORTED
    assert make(q, k, v, t(3, 5, dt=E.F32), o) == E.ERR_NOT_SUPPORTED
    assert make(t(8, 64), k, v, tab, o) == E.ERR_INVALID_ARGUMENT
    assert make(q, k, v, i(4, 5), o) == E.ERR_EXTENT_MISMATCH
    assert make(t(3, 7, 64), k, v, tab, t(3, 7, 32)) == E.ERR_EXTENT_MISMATCH        # 7 heads over 2 key heads
    assert make(q, k, t(9, 8, 2, 32), tab, o) == E.ERR_EXTENT_MISMATCH
    assert make(q, k, t(8, 16, 2, 32), tab, o) == E.ERR_EXTENT_MISMATCH
    assert make(q, t(9, 16, 2, 32), v, tab, o) == E.ERR_EXTENT_MISMATCH
    assert make(q, k, v, tab, t(3, 8, 64)) == E.ERR_EXTENT_MISMATCH
    assert make(t(3, 8, 257), t(9, 16, 2, 257), v, tab, o) == E.ERR_NOT_SUPPORTED
    assert make(q, k, v, tab, t(3, 8, 32, st=(0, 32, 1))) == E.ERR_D_ALIASING
    assert make(q, k, v, tab, o, window=-1) == E.ERR_INVALID_ARGUMENT
    assert make(q, k, v, tab, o, scale=float("nan")) == E.ERR_INVALID_ARGUMENT
    assert make(q, t(9, 16, 2, 64, st=(1 << 61, 128, 64, 1)), v, tab, o) == E.ERR_NOT_SUPPORTED
    n = op.workspace_size()
    run = lambda *a, **k: code(api, lambda: op.execute(0, *a, **k))  # noqa: E731
    assert run(256, 256, 256, 256, 0, 256, workspace=256, workspace_bytes=n) == E.ERR_INVALID_ARGUMENT
    assert run(256, 256, 256, 256, 256, 256) == E.ERR_WORKSPACE_TOO_SMALL
    assert run(256, 256, 256, 256, 256, 256, workspace=256, workspace_bytes=n - 1) == E.ERR_WORKSPACE_TOO_SMALL
    assert run(256, 256, 256, 256, 256, 256, workspace=128, workspace_bytes=n) == E.ERR_MISALIGNED
    assert run(257, 256, 256, 256, 256, 256, workspace=256, workspace_bytes=n) == E.ERR_MISALIGNED
    assert run(256, 256, 256, 258, 256, 256, workspace=256, workspace_bytes=n) == E.ERR_MISALIGNED


def test_pages_refusals(api, handle):
    E = api
    t = lambda *s, dt=api.BF16, st=None: dense(api, handle, dt, *s, strides=st)  # noqa: E731
    tab = dense(api, handle, api.I32, 3, 5)
    make = lambda *a: code(api, lambda: api.Pages(handle, *a))  # noqa: E731
    op = api.Pages(handle, [t(9, 16, 2, 64), t(9, 16, 2, 32, dt=E.F64)], tab, 16)
    n = op.workspace_size()
    assert n > 0
    assert make([], tab, 16) == E.ERR_INVALID_ARGUMENT
    assert make([t(9, 4)] * 5, tab, 16) == E.ERR_INVALID_ARGUMENT
    assert make(t(9, 4), tab, 0) == E.ERR_INVALID_ARGUMENT
    assert make(t(), tab, 16) == E.ERR_INVALID_ARGUMENT
    assert make(t(9, 4), t(3, 5), 16) == E.ERR_NOT_SUPPORTED
    assert make(t(9, 4), dense(api, handle, api.I32, 3, 5, 2), 16) == E.ERR_INVALID_ARGUMENT
    assert make([t(9, 4), t(8, 4)], tab, 16) == E.ERR_EXTENT_MISMATCH
    assert make(t(9, 4, st=(4, 0)), tab, 16) == E.ERR_D_ALIASING
    assert make(t(9, 4), dense(api, handle, api.I32, 3, 5, strides=(0, 1)), 16) == E.ERR_D_ALIASING
    assert make(t(1 << 28, 4), tab, 16) == E.ERR_NOT_SUPPORTED
    assert make(t(2, 1 << 16, 1 << 16), tab, 16) == E.ERR_NOT_SUPPORTED
    many = (3, 2, 2, 2, 2, 2, 2, 2, 2, 2)
    assert make(t(*many, st=[3 ** 10] + [3 ** i for i in range(9)]), tab, 16) == E.ERR_NOT_SUPPORTED
    ok = dict(workspace=256, workspace_bytes=n)
    ext = lambda *a, **k: code(api, lambda: op.extend(0, *a, **k))  # noqa: E731
    assert ext(0, 256, 256, 256, 256, 1, [256, 256], **ok) == E.ERR_INVALID_ARGUMENT
    assert ext(256, 256, 256, 256, 256, 0, [256, 256], **ok) == E.ERR_INVALID_ARGUMENT
    assert ext(256, 256, 256, 256, 256, 1, [256], **ok) == E.ERR_INVALID_ARGUMENT           # two layouts, one tensor
    assert ext(256, 256, 256, 256, 256, 1, [256, 0], **ok) == E.ERR_INVALID_ARGUMENT
    assert ext(256, 256, 256, 256, 256, 1, [257, 256], **ok) == E.ERR_MISALIGNED
    assert ext(256, 256, 256, 256, 256, 1, [256, 256]) == E.ERR_WORKSPACE_TOO_SMALL
    assert ext(256, 256, 256, 256, 256, 1, [256, 256], workspace=128, workspace_bytes=n) == E.ERR_MISALIGNED
    assert ext(256, 258, 256, 256, 256, 1, [256, 256], **ok) == E.ERR_MISALIGNED
    assert code(api, lambda: op.compact(0, 256, 0, [256, 256], **ok)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.compact(0, 256, 256, [256, 256])) == E.ERR_WORKSPACE_TOO_SMALL
    assert code(api, lambda: op.fork(0, 0, 256, 1, 256, 256, 256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.fork(0, 256, 256, -1, 256, 256, 256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.free(0, 0, 1, 256, 256, 256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.free(0, 256, 1, 256, 0, 256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.copy(0, 0, 1, [256, 256])) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: op.copy(0, 256, 1, [256, 256, 256])) == E.ERR_INVALID_ARGUMENT


def test_paged_attention_limits(api, handle):
    """More sequences, or more tokens in all, than the kernel's counters hold."""
    E = api
    t = lambda *s, st=None: dense(api, handle, api.BF16, *s, strides=st)  # noqa: E731
    n = (1 << 23) + 1
    one = dense(api, handle, api.I32, n, 1)
    assert code(api, lambda: api.PagedAttention(handle, t(n, 1, 8), t(9, 16, 1, 8), t(9, 16, 1, 8), one, t(n, 1, 8))) == E.ERR_NOT_SUPPORTED
    n = 1 << 22
    wide = dense(api, handle, api.I32, n, 1)
    long_page = t(1, 1 << 21, 1, 8)
    assert code(api, lambda: api.PagedAttention(handle, t(n, 1, 8), long_page, long_page, wide, t(n, 1, 8))) == E.ERR_NOT_SUPPORTED
