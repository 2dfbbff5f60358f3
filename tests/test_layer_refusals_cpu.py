"""What the residual norm, the 4-bit products and the tree attention refuse, and the norm's 64-bit reference against differences: no GPU needed."""
import pytest
import torch

from test_decoder_refusals_cpu import api, code, dense, handle  # noqa: F401


def test_types_of_the_layer_are_refused_by_contractions(api, handle):  # noqa: F811
    a = dense(api, handle, api.E4M3, 4, 4)
    assert code(api, lambda: api.Contraction(handle, a, "ik", a, "kj", None, None, a, "ij", alpha=None)) == api.ERR_NOT_SUPPORTED
    assert code(api, lambda: api.Elementwise(handle, a, "ij", None, a, "ji", alpha=None, beta=None)) == api.ERR_NOT_SUPPORTED
    assert code(api, lambda: dense(api, handle, 8, 4, 4)) == api.ERR_INVALID_ARGUMENT


def test_add_norm_refusals(api, handle):  # noqa: F811
    E, B = api, api.BF16
    t = lambda *s, dt=B, st=None: dense(api, handle, dt, *s, strides=st)  # noqa: E731
    make = lambda *a, **k: code(api, lambda: api.AddNorm(handle, *a, **k))  # noqa: E731
    x = t(4, 64)
    assert make(t(4, 64, dt=E.F64), t(4, 64, dt=E.F64)) == E.ERR_NOT_SUPPORTED
    assert make(x, t(4, 64, dt=E.F16)) == E.ERR_NOT_SUPPORTED
    assert make(x, t(4, 64, dt=E.F32)) == E.ERR_NOT_SUPPORTED
    assert make(t(4, 64, dt=E.E4M3), x) == E.ERR_NOT_SUPPORTED
    assert make(x, x, R=x) == E.ERR_INVALID_ARGUMENT
    assert make(x, x, H=x) == E.ERR_INVALID_ARGUMENT
    assert make(x, x, R=x, H=t(4, 64, dt=E.F32)) == E.ERR_NOT_SUPPORTED
    assert make(x, x, R=t(4, 64, dt=E.F16), H=t(4, 64, dt=E.F16)) == E.ERR_NOT_SUPPORTED
    assert make(x, t(4, 63)) == E.ERR_EXTENT_MISMATCH
    assert make(x, x, R=t(5, 64), H=t(4, 64)) == E.ERR_EXTENT_MISMATCH
    assert make(t(4, 2, 32), t(4, 2, 32)) == E.ERR_INVALID_ARGUMENT
    assert make(t(2, 16385), t(2, 16385)) == E.ERR_NOT_SUPPORTED
    assert make(x, t(4, 64, st=(0, 1))) == E.ERR_D_ALIASING
    assert make(x, x, R=x, H=t(4, 64, st=(32, 1))) == E.ERR_D_ALIASING
    assert make(t(4, 64, st=(1 << 62, 1)), x) == E.ERR_NOT_SUPPORTED
    assert make(x, x, eps=-1.0) == E.ERR_INVALID_ARGUMENT
    assert make(x, x, eps=1e-39) == E.ERR_INVALID_ARGUMENT
    assert make(x, x, eps=float("nan")) == E.ERR_INVALID_ARGUMENT
    q, s = t(4, 64, dt=E.E4M3), t(4, 1, dt=E.F32)
    assert make(x, q) == E.ERR_INVALID_ARGUMENT                           # no scales
    assert make(x, x, S=s) == E.ERR_INVALID_ARGUMENT
    assert make(x, x, group=32) == E.ERR_INVALID_ARGUMENT
    assert make(x, q, S=s, group=16) == E.ERR_INVALID_ARGUMENT
    assert make(x, q, S=s, group=-32) == E.ERR_INVALID_ARGUMENT
    assert make(x, q, S=s, group=32) == E.ERR_EXTENT_MISMATCH
    assert make(x, q, S=t(4, 1)) == E.ERR_NOT_SUPPORTED
    assert make(x, q, S=t(4, 1, dt=E.F32, st=(0, 1))) == E.ERR_D_ALIASING

    op = api.AddNorm(handle, x, x, R=x, H=x)
    run = lambda *a, **k: code(api, lambda: op.execute(0, *a, **k))  # noqa: E731
    assert run(256, 256, 256) == E.ERR_INVALID_ARGUMENT                    # no stream of residuals
    assert run(256, 256, 256, R=256) == E.ERR_INVALID_ARGUMENT
    assert run(0, 256, 256, R=256, H=256) == E.ERR_INVALID_ARGUMENT
    assert run(256, 256, 256, R=256, H=256, S=256) == E.ERR_INVALID_ARGUMENT
    assert run(257, 256, 256, R=256, H=256) == E.ERR_MISALIGNED
    assert run(256, 257, 256, R=256, H=256) == E.ERR_MISALIGNED
    back = lambda *a, **k: code(api, lambda: op.backward(0, *a, **k))  # noqa: E731
    assert op.workspace_size() > 0
    assert back(256, 256, 256) == E.ERR_INVALID_ARGUMENT                   # nothing wanted
    assert back(0, 256, 256, dX=256) == E.ERR_INVALID_ARGUMENT
    assert back(256, 0, 256, dX=256, dW=256, workspace=256, workspace_bytes=1 << 30) == E.ERR_INVALID_ARGUMENT   # dW without W
    assert back(256, 256, 256, dX=256, dW=256) == E.ERR_WORKSPACE_TOO_SMALL
    assert back(256, 256, 256, dX=256, dW=256, workspace=256, workspace_bytes=op.workspace_size() - 1) == E.ERR_WORKSPACE_TOO_SMALL
    assert back(256, 256, 256, dX=256, dW=256, workspace=128, workspace_bytes=1 << 30) == E.ERR_MISALIGNED
    assert back(256, 256, 256, dX=256, dW=258, workspace=256, workspace_bytes=1 << 30) == E.ERR_MISALIGNED
    assert back(256, 256, 257, dX=256) == E.ERR_MISALIGNED
    alone = api.AddNorm(handle, x, x)
    assert code(api, lambda: alone.execute(0, 256, 256, 256, R=256, H=256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: alone.backward(0, 256, 256, 256, dX=256, dH=256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: alone.backward(0, 256, 256, 256, dR=256)) == E.ERR_INVALID_ARGUMENT
    eight = api.AddNorm(handle, x, q, S=s)
    assert eight.workspace_size() == 0
    assert code(api, lambda: eight.execute(0, 256, 256, 256)) == E.ERR_INVALID_ARGUMENT
    assert code(api, lambda: eight.backward(0, 256, 256, 256, dX=256)) == E.ERR_NOT_SUPPORTED
    spread = api.AddNorm(handle, t(4, 64, st=(0, 1)), x)
    assert code(api, lambda: spread.backward(0, 256, 256, 256, dX=256)) == E.ERR_D_ALIASING


def test_linear4_refusals(api, handle):  # noqa: F811
    E, B = api, api.BF16
    t = lambda *s, dt=B, st=None: dense(api, handle, dt, *s, strides=st)  # noqa: E731
    make = lambda *a, **k: code(api, lambda: api.Linear4(handle, *a, **k))  # noqa: E731
    x, y = t(4, 256), t(4, 100)
    assert make(x, y, group=16) == E.ERR_INVALID_ARGUMENT
    assert make(x, y, group=512) == E.ERR_INVALID_ARGUMENT
    assert make(x, y, group=96) == E.ERR_INVALID_ARGUMENT
    assert make(x, y, group=-128) == E.ERR_INVALID_ARGUMENT
    assert make(x, y, x_group=128) == E.ERR_INVALID_ARGUMENT                       # only inputs in 8 bits have scales
    assert make(x, y, XS=t(4, 1, dt=E.F32)) == E.ERR_INVALID_ARGUMENT
    assert make(t(4, 256, dt=E.E4M3), y) == E.ERR_INVALID_ARGUMENT
    assert make(t(4, 256, dt=E.E4M3), y, XS=t(4, 1)) == E.ERR_NOT_SUPPORTED
    assert make(t(4, 256, dt=E.E4M3), y, XS=t(4, 1, dt=E.F32), x_group=128) == E.ERR_EXTENT_MISMATCH
    assert make(t(4, 256, dt=E.E4M3), y, XS=t(3, 1, dt=E.F32)) == E.ERR_EXTENT_MISMATCH
    assert make(x, t(5, 100)) == E.ERR_EXTENT_MISMATCH
    assert make(x, t(4, 100, dt=E.E4M3)) == E.ERR_NOT_SUPPORTED
    assert make(t(4, 256, dt=E.F64), y) == E.ERR_NOT_SUPPORTED
    assert make(x, y, scale_type=E.F64) == E.ERR_NOT_SUPPORTED
    assert make(t(4, 2, 128), y) == E.ERR_INVALID_ARGUMENT
    assert make(x, t(4, 100, st=(50, 1))) == E.ERR_D_ALIASING
    assert make(t(4, 256, st=(1 << 62, 1)), y) == E.ERR_NOT_SUPPORTED
    assert make(t(4, (1 << 24) + 1), y) == E.ERR_NOT_SUPPORTED
    assert make(x, t(4, (1 << 24) + 1)) == E.ERR_NOT_SUPPORTED
    assert make(t((1 << 19) + 1, 256), t((1 << 19) + 1, 100)) == E.ERR_NOT_SUPPORTED
    with pytest.raises(ValueError):
        api.Linear4(handle, x, y, activation="other")

    op = api.Linear4(handle, x, y, group=64)
    assert op.packed_size() == 7 * 4 * (512 + 16 * 2)
    assert api.Linear4(handle, x, y, group=64, zeros=True).packed_size() == op.packed_size() + 7 * 4 * 16
    assert api.Linear4(handle, t(9, 256, dt=E.F32), t(9, 100, dt=E.F16), group=64).packed_size() == op.packed_size()
    run = lambda *a, **k: code(api, lambda: op.execute(0, *a, **k))  # noqa: E731
    big = dict(workspace=256, workspace_bytes=1 << 40)
    assert run(0, 256, 256, **big) == E.ERR_INVALID_ARGUMENT
    assert run(256, 0, 256, **big) == E.ERR_INVALID_ARGUMENT
    assert run(256, 256, 0, **big) == E.ERR_INVALID_ARGUMENT
    assert run(256, 256, 256, XS=256, **big) == E.ERR_INVALID_ARGUMENT
    assert run(128, 256, 256, **big) == E.ERR_MISALIGNED
    assert run(256, 257, 256, **big) == E.ERR_MISALIGNED
    assert run(256, 256, 257, **big) == E.ERR_MISALIGNED
    pack = lambda *a: code(api, lambda: op.pack(0, *a))  # noqa: E731
    assert pack(0, 256, 0, 256) == E.ERR_INVALID_ARGUMENT
    assert pack(256, 256, 256, 256) == E.ERR_INVALID_ARGUMENT                      # zeros that the operation does not have
    assert pack(256, 257, 0, 256) == E.ERR_MISALIGNED
    assert pack(256, 256, 0, 128) == E.ERR_MISALIGNED


def test_tree_attention_refusals(api, handle):  # noqa: F811
    E, B = api, api.BF16
    t = lambda *s, dt=B, st=None: dense(api, handle, dt, *s, strides=st)  # noqa: E731
    i = lambda *s: dense(api, handle, api.I32, *s)  # noqa: E731
    make = lambda *a, **k: code(api, lambda: api.TreeAttention(handle, *a, **k))  # noqa: E731
    q, k, v, tab, m, o = t(3, 40, 8, 64), t(9, 16, 2, 64), t(9, 16, 2, 32), i(3, 5), i(3, 40, 2), t(3, 40, 8, 32)
    op = api.TreeAttention(handle, q, k, v, tab, m, o)
    assert op.workspace_size() > 0
    assert make(t(3, 40, 8, 64, dt=E.F64), k, v, tab, m, o) == E.ERR_NOT_SUPPORTED
    assert make(t(3, 40, 8, 64, dt=E.E4M3), k, v, tab, m, o) == E.ERR_NOT_SUPPORTED
    assert make(q, t(9, 16, 2, 64, dt=E.F16), v, tab, m, o) == E.ERR_NOT_SUPPORTED
    assert make(q, k, v, tab, t(3, 40, 2), o) == E.ERR_NOT_SUPPORTED
    assert make(t(3, 8, 64), k, v, tab, m, o) == E.ERR_INVALID_ARGUMENT
    assert make(q, k, v, tab, i(3, 40), o) == E.ERR_INVALID_ARGUMENT
    assert make(q, k, v, i(4, 5), m, o) == E.ERR_EXTENT_MISMATCH
    assert make(q, k, v, tab, i(3, 40, 1), o) == E.ERR_EXTENT_MISMATCH
    assert make(q, k, v, tab, i(3, 39, 2), o) == E.ERR_EXTENT_MISMATCH
    assert make(t(3, 40, 7, 64), k, v, tab, m, t(3, 40, 7, 32)) == E.ERR_EXTENT_MISMATCH
    assert make(q, k, t(9, 8, 2, 32), tab, m, o) == E.ERR_EXTENT_MISMATCH
    assert make(q, k, v, tab, m, t(3, 41, 8, 32)) == E.ERR_EXTENT_MISMATCH
    assert make(t(3, 129, 8, 64), k, v, tab, i(3, 129, 5), t(3, 129, 8, 32)) == E.ERR_NOT_SUPPORTED
    assert make(t(3, 40, 8, 264), t(9, 16, 2, 264), v, tab, m, o) == E.ERR_NOT_SUPPORTED
    assert make(q, k, v, tab, m, t(3, 40, 8, 32, st=(1280 * 8, 0, 32, 1))) == E.ERR_D_ALIASING
    assert make(q, t(9, 16, 2, 64, st=(1 << 62, 128, 64, 1)), v, tab, m, o) == E.ERR_NOT_SUPPORTED
    assert make(q, k, v, tab, m, o, window=39) == E.ERR_INVALID_ARGUMENT                # shorter than a tree
    assert make(q, k, v, tab, m, o, window=-1) == E.ERR_INVALID_ARGUMENT
    assert make(q, k, v, tab, m, o, scale=1e39) == E.ERR_INVALID_ARGUMENT
    api.TreeAttention(handle, q, k, v, tab, m, o, window=40)
    run = lambda *a, **k: code(api, lambda: op.execute(0, *a, **k))  # noqa: E731
    big = dict(workspace=256, workspace_bytes=1 << 40)
    assert run(0, 256, 256, 256, 256, 256, 256, **big) == E.ERR_INVALID_ARGUMENT
    assert run(256, 256, 256, 256, 256, 0, 256, **big) == E.ERR_INVALID_ARGUMENT
    assert run(257, 256, 256, 256, 256, 256, 256, **big) == E.ERR_MISALIGNED
    assert run(256, 256, 256, 256, 256, 258, 256, **big) == E.ERR_MISALIGNED
    assert run(256, 256, 256, 256, 256, 256, 256, lse=258, **big) == E.ERR_MISALIGNED
    assert run(256, 256, 256, 256, 256, 256, 256) == E.ERR_WORKSPACE_TOO_SMALL
    assert run(256, 256, 256, 256, 256, 256, 256, workspace=256, workspace_bytes=op.workspace_size() - 1) == E.ERR_WORKSPACE_TOO_SMALL
    assert run(256, 256, 256, 256, 256, 256, 256, workspace=128, workspace_bytes=1 << 40) == E.ERR_MISALIGNED
    for bad in ([0], [-3], [-1, 1], [-2, 0]):
        with pytest.raises(ValueError):
            api.tree_masks(bad)


def test_norm_reference_against_differences():
    from layer_reference import norm_backward, norm_forward
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g).double()  # noqa: E731
    x, rr, w, dy, dh, v, u = r(3, 17), r(3, 17), r(17), r(3, 17), r(3, 17), r(3, 17), r(17)
    step = 1e-5
    f = lambda a, b: float((norm_forward(a, b, rr, 1e-3)[1] * dy).sum() + (norm_forward(a, b, rr, 1e-3)[0] * dh).sum())  # noqa: E731
    dx, dw, _, _ = norm_backward(x + rr, w, dy, dh, 1e-3)
    assert abs((f(x + step * v, w) - f(x - step * v, w)) / (2 * step) - float((dx * v).sum())) < 1e-7
    assert abs((f(x, w + step * u) - f(x, w - step * u)) / (2 * step) - float((dw * u).sum())) < 1e-7
