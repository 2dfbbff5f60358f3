"""The residual's addition and norm on the GPU against a plain 64-bit implementation."""
import math

import pytest
import torch

import helpers
from decoder_reference import E32, FLOOR, UNIT
from layer_reference import (GRAD_CHAIN, NORM_CHAIN, check, check_e4m3, info, norm_backward, norm_forward, norm_grad_chain)

pytestmark = pytest.mark.gpu
F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def now():
    return torch.cuda.current_stream().cuda_stream


def at(t):
    return t.data_ptr() if t is not None else 0


def make(T, D, dtype, stream, seed, weight=True):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, D, generator=g) * 2).to(dtype)
    r = (torch.randn(T, D, generator=g) * 3).to(stream) if stream is not None else None
    w = (1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if weight else None
    dy = torch.randn(T, D, generator=g).to(dtype)
    dh = torch.randn(T, D, generator=g).to(stream) if stream is not None else None
    return x, r, w, dy, dh


def padded(t, extra, first=0):
    """A copy of t on the GPU whose rows lie `extra` elements further apart, begun `first` elements into the memory."""
    if t is None:
        return None
    room = torch.zeros(first + t.shape[0] * (t.shape[1] + extra), dtype=t.dtype, device="cuda")
    v = room[first:].view(t.shape[0], -1)[:, :t.shape[1]]
    v.copy_(t)
    return v


SIZES = [(1, 1), (1, 8), (3, 64), (5, 100), (2, 256), (7, 257), (4, 520), (3, 1001), (2, 4096), (3, 5120), (2, 8192), (2, 8200), (2, 16384),
         (1, 16383), (310, 96), (450, 1024), (700, 72), (301, 2056)]


@pytest.mark.parametrize("dtype,stream", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32), (BF16, None), (F32, None)])
@pytest.mark.parametrize("T,D", SIZES)
def test_forward_and_backward(api, handle, T, D, dtype, stream):
    eps = 1e-5
    x, r, w, dy, dh = make(T, D, dtype, stream, T * 31 + D)
    cx, cr, cw, cdy, cdh = (t.cuda() if t is not None else None for t in (x, r, w, dy, dh))
    y, h = torch.full_like(cx, math.nan), torch.full_like(cr, math.nan) if r is not None else None
    op = api.AddNorm(handle, info(api, handle, cx), info(api, handle, y), R=info(api, handle, cr) if r is not None else None,
                     H=info(api, handle, h) if r is not None else None, eps=eps)
    op.execute(now(), at(cx), at(cw), at(y), R=at(cr), H=at(h))
    eh, ey = norm_forward(x, w, r, eps)
    check(y, ey, UNIT[dtype] * ey.abs() + NORM_CHAIN * E32 * ey.abs() + FLOOR[dtype])
    kept = x
    if r is not None:
        check(h, eh, (UNIT[stream] + E32) * eh.abs() + FLOOR[stream])
        kept = h.cpu()
    dx, dw = torch.full_like(cx, math.nan), torch.full((D,), math.nan, device="cuda")
    dr = torch.full_like(cr, math.nan) if r is not None else None
    ws = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")
    source = h if r is not None else cx
    op.backward(now(), at(source), at(cw), at(cdy), dH=at(cdh), dX=at(dx), dR=at(dr), dW=at(dw), workspace=at(ws), workspace_bytes=ws.numel())
    edx, edw, size, moduli = norm_backward(kept, w, dy, dh, eps)
    check(dx, edx, UNIT[dtype] * edx.abs() + GRAD_CHAIN * E32 * size + FLOOR[dtype])
    if r is not None:
        check(dr, edx, UNIT[stream] * edx.abs() + GRAD_CHAIN * E32 * size + FLOOR[stream])
    check(dw, edw, norm_grad_chain(T) * E32 * moduli)
    first = dw.clone()
    op.backward(now(), at(source), at(cw), at(cdy), dX=at(dx), dW=at(dw), workspace=at(ws), workspace_bytes=ws.numel())
    assert torch.equal(first, dw)                     # same sums, same bits; no gradient along the stream this time
    edx = norm_backward(kept, w, dy, None, eps)[0]
    check(dx, edx, UNIT[dtype] * edx.abs() + GRAD_CHAIN * E32 * size + FLOOR[dtype])


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("dtype,stream", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32), (BF16, None)])
@pytest.mark.parametrize("T,D", SIZES)
def test_eight_bits(api, handle, T, D, dtype, stream, group):
    eps = 1e-6
    x, r, w, _, _ = make(T, D, dtype, stream, T * 77 + D)
    cx, cr, cw = (t.cuda() if t is not None else None for t in (x, r, w))
    y = torch.full((T, D), 1.0, device="cuda").to(E4M3)
    h = torch.full_like(cr, math.nan) if r is not None else None
    s = torch.full((T, -(-D // group) if group else 1), math.nan, device="cuda")
    op = api.AddNorm(handle, info(api, handle, cx), info(api, handle, y), R=info(api, handle, cr) if r is not None else None,
                     H=info(api, handle, h) if r is not None else None, S=info(api, handle, s), group=group, eps=eps)
    op.execute(now(), at(cx), at(cw), at(y), R=at(cr), H=at(h), S=at(s))
    eh, ey = norm_forward(x, w, r, eps)
    check_e4m3(y, s, ey, group, NORM_CHAIN)
    if r is not None:
        check(h, eh, (UNIT[stream] + E32) * eh.abs() + FLOOR[stream])


@pytest.mark.parametrize("extra,first", [(8, 0), (16, 16), (3, 0), (0, 1), (16, 8), (1, 5)])
@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("eight", [False, True])
def test_strides_alignment_and_in_place(api, handle, dtype, stream, extra, first, eight):
    """Padded and shifted rows give what dense ones give (up to the order of sums); the stream is updated in place."""
    T, D, eps = 5, 512, 1e-5
    x, r, w, dy, dh = make(T, D, dtype, stream, 5)
    cx, cr, cw = padded(x, extra, first), padded(r, extra, first), w.cuda()
    y = padded(torch.zeros(T, D).to(E4M3 if eight else dtype), extra, first)
    s = torch.full((T, 2 * D // 64), math.nan, device="cuda")[:, ::2] if eight else None
    op = api.AddNorm(handle, info(api, handle, cx), info(api, handle, y), R=info(api, handle, cr), H=info(api, handle, cr),
                     S=info(api, handle, s) if eight else None, group=64 if eight else 0, eps=eps)
    op.execute(now(), at(cx), at(cw), at(y), R=at(cr), H=at(cr), S=at(s))
    eh, ey = norm_forward(x, w, r, eps)
    check(cr, eh, (UNIT[stream] + E32) * eh.abs() + FLOOR[stream])
    if eight:
        check_e4m3(y.contiguous(), s.contiguous(), ey, 64, NORM_CHAIN)
        return
    check(y, ey, UNIT[dtype] * ey.abs() + NORM_CHAIN * E32 * ey.abs() + FLOOR[dtype])
    # gradients over the gradients that came in, without weights' sums: no workspace
    gy, gh = padded(dy, extra, first), padded(dh, extra, first)
    op.backward(now(), at(cr), at(cw), at(gy), dH=at(gh), dX=at(gy), dR=at(gh))
    edx, _, size, _ = norm_backward(cr.cpu(), w, dy, dh, eps)
    check(gy, edx, UNIT[dtype] * edx.abs() + GRAD_CHAIN * E32 * size + FLOOR[dtype])
    check(gh, edx, UNIT[stream] * edx.abs() + GRAD_CHAIN * E32 * size + FLOOR[stream])


def test_columns_apart_reversed_rows_and_broadcast_input(api, handle):
    T, D, eps = 6, 40, 1e-5
    x, r, w, dy, dh = make(T, D, F32, F32, 9)
    wide = torch.zeros(T, 2 * D, device="cuda")
    wide[:, ::2] = x.cuda()
    y = torch.zeros(D, T, device="cuda").T
    # rows from the last to the first: negative strides
    ir = api.TensorInfo(handle, api.F32, (T, D), (-D, 1))
    cr, h, cw = r.flip(0).cuda(), torch.zeros(T, D, device="cuda"), w.cuda()
    op = api.AddNorm(handle, info(api, handle, wide[:, ::2]), info(api, handle, y), R=ir, H=ir, eps=eps)
    op.execute(now(), at(wide), at(cw), at(y), R=cr[T - 1].data_ptr(), H=h[T - 1].data_ptr())
    eh, ey = norm_forward(x, w, r, eps)
    check(y, ey, (1 + NORM_CHAIN) * E32 * ey.abs())
    check(h.flip(0), eh, 2 * E32 * eh.abs())
    # one row for all tokens, no weight; its gradient in its own layout would alias
    one = x[:1].cuda()
    op = api.AddNorm(handle, info(api, handle, one.expand(T, D)), info(api, handle, y), R=info(api, handle, h), H=info(api, handle, h), eps=eps)
    cr = r.cuda()
    op.execute(now(), at(one), 0, at(y), R=at(cr), H=at(h))
    eh, ey = norm_forward(x[:1].expand(T, D), None, r, eps)
    check(y, ey, (1 + NORM_CHAIN) * E32 * ey.abs())
    dyc = dy.cuda().T.contiguous().T
    dr = torch.zeros(T, D, device="cuda")
    with pytest.raises(api.BtcError) as e:
        op.backward(now(), at(h), 0, at(dyc), dX=at(one))
    assert e.value.code == api.ERR_D_ALIASING
    op.backward(now(), at(h), 0, at(dyc), dR=at(dr))
    edx, _, size, _ = norm_backward(h.cpu(), None, dy, None, eps)
    check(dr, edx, E32 * edx.abs() + GRAD_CHAIN * E32 * size)


def test_zeros_infinities_and_nan(api, handle):
    """A row of zeros gives zeros, a lost row or group stays alone, values down to the scale's smallest keep their codes."""
    T, D, group = 6, 256, 64
    x = torch.randn(T, D, generator=torch.Generator().manual_seed(2))
    x[0] = 0
    x[1, 5] = math.inf
    x[2, 200] = math.nan
    x[3, :64] = 0
    w = torch.ones(D)
    w[128:192] = 1e-38                                 # scales at their smallest
    for dtype in (F32, BF16):
        cx, cw = x.to(dtype).cuda(), w.to(dtype).cuda()
        y = torch.ones(T, D, device="cuda", dtype=dtype)
        op = api.AddNorm(handle, info(api, handle, cx), info(api, handle, y), eps=1e-6)
        op.execute(now(), at(cx), at(cw), at(y))
        assert not y[0].any() and torch.isnan(y[2]).all()
        assert torch.isnan(y[1, 5]) and not y[1, :5].any() and not y[1, 6:].any()
        ey = norm_forward(cx.cpu(), cw.cpu(), None, 1e-6)[1]
        check(y[3:], ey[3:], (UNIT[dtype] + NORM_CHAIN * E32) * ey[3:].abs() + 2.0 ** -133)
        for g in (0, group):
            q = torch.ones(T, D, device="cuda").to(E4M3)
            s = torch.zeros(T, D // g if g else 1, device="cuda")
            op = api.AddNorm(handle, info(api, handle, cx), info(api, handle, q), S=info(api, handle, s), group=g, eps=1e-6)
            op.execute(now(), at(cx), at(cw), at(q), S=at(s))
            codes = q.view(torch.uint8)
            assert not codes[0].any() and (s[0] == 2.0 ** -126).all()
            # the lost group has codes of zero; beside it the row's infinite root leaves zeros, which keep their signs
            assert torch.isnan(s[1, 0]) and not codes[1, :g or D].any() and not (codes[1] & 0x7f).any()
            assert torch.isnan(s[2]).all() and not codes[2].any()
            assert torch.isfinite(s[3:]).all() and (s[3:] >= 2.0 ** -126).all()
            if g:
                assert torch.isfinite(s[1, 1:]).all() and s[3, 0] == 2.0 ** -126 and not codes[3, :64].any()
            check_e4m3(q[4:], s[4:], ey[4:], g, NORM_CHAIN)


def test_gradient_against_differences(api, handle):
    """<dx, v> and <dw, u> against differences of the kernel's own forward pass in fp32."""
    T, D, eps, step = 4, 96, 1e-3, 2.0 ** -5
    x, r, w, dy, dh = make(T, D, F32, F32, 12)
    g = torch.Generator().manual_seed(3)
    v, u = torch.randn(T, D, generator=g), torch.randn(D, generator=g) * 0.2
    y, h = torch.zeros(T, D, device="cuda"), torch.zeros(T, D, device="cuda")
    like = info(api, handle, y)
    op = api.AddNorm(handle, like, like, R=like, H=like, eps=eps)

    def value(xx, ww):
        a, b, c = xx.cuda(), ww.cuda(), r.cuda()
        op.execute(now(), at(a), at(b), at(y), R=at(c), H=at(h))
        return float((y.double().cpu() * dy.double()).sum() + (h.double().cpu() * dh.double()).sum())

    def exact(xx, ww):
        hh, yy = norm_forward(xx, ww, r, eps)
        return float((yy * dy.double()).sum() + (hh * dh.double()).sum())

    value(x, w)
    dx, dw, ws = torch.zeros(T, D, device="cuda"), torch.zeros(D, device="cuda"), torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")
    cw, cdy, cdh = w.cuda(), dy.cuda(), dh.cuda()
    op.backward(now(), at(h), at(cw), at(cdy), dH=at(cdh), dX=at(dx), dW=at(dw), workspace=at(ws), workspace_bytes=ws.numel())
    eh, ey = norm_forward(x, w, r, eps)
    # each difference of two passes: every output within 26 units, over 2 steps; what the differences leave out is known from 64 bits
    noise = 2 * 27 * E32 * float((ey.abs() * dy.abs()).sum() + (eh.abs() * dh.abs()).sum()) / (2 * step) * 1.5
    for grad, a, b in ((dx, (x + step * v, w), (x - step * v, w)), (dw, (x, w + step * u), (x, w - step * u))):
        along = float((grad.double().cpu() * (v if grad is dx else u).double()).sum())
        curved = (exact(*a) - exact(*b)) / (2 * step)
        edx, edw, size, moduli = norm_backward(eh, w, dy, dh, eps)
        formula = float((edx * v.double()).sum()) if grad is dx else float((edw * u.double()).sum())
        measured = (value(*a) - value(*b)) / (2 * step)
        slack = GRAD_CHAIN * E32 * float(((size * v.double().abs()).sum()) if grad is dx else (moduli * u.double().abs()).sum())
        assert abs(measured - along) <= noise + slack + abs(curved - formula), (measured, along, curved, formula, noise)


def test_other_streams_graph_and_two_at_once(api, handle):
    """Two captured passes of one operation on two streams, with a workspace each, replayed at the same time."""
    T, D, eps = 300, 1024, 1e-5
    dtype = BF16
    sets = []
    like = torch.zeros(T, D, dtype=dtype, device="cuda")
    i = info(api, handle, like)
    op = api.AddNorm(handle, i, i, R=i, H=i, eps=eps)
    for seed in (1, 2):
        x, r, w, dy, dh = make(T, D, dtype, dtype, seed)
        c = [t.cuda() for t in (x, r, w, dy, dh)]
        out = [torch.zeros_like(like) for _ in range(4)] + [torch.zeros(D, device="cuda")]
        ws = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            op.execute(now(), at(c[0]), at(c[2]), at(out[1]), R=at(c[1]), H=at(out[0]))
            op.backward(now(), at(out[0]), at(c[2]), at(c[3]), dH=at(c[4]), dX=at(out[2]), dR=at(out[3]), dW=at(out[4]), workspace=at(ws),
                        workspace_bytes=ws.numel())
        sets.append((x, r, w, dy, dh, c, out, ws, stream, graph))
    for _ in range(3):
        for z in sets:
            with torch.cuda.stream(z[8]):
                z[9].replay()
    torch.cuda.synchronize()
    for x, r, w, dy, dh, c, out, ws, stream, graph in sets:
        eh, ey = norm_forward(x, w, r, eps)
        check(out[1], ey, (UNIT[dtype] + NORM_CHAIN * E32) * ey.abs())
        edx, edw, size, moduli = norm_backward(out[0].cpu(), w, dy, dh, eps)
        check(out[2], edx, UNIT[dtype] * edx.abs() + GRAD_CHAIN * E32 * size)
        assert torch.equal(out[2], out[3])
        check(out[4], edw, norm_grad_chain(T) * E32 * moduli)


def test_offsets_beyond_32_bits(api, handle):
    """Rows of one tensor more than 2^32 bytes apart."""
    T, D, far = 2, 512, (1 << 31) + 64
    g = torch.Generator().manual_seed(4)
    x = torch.randn(T, D, generator=g).to(F16)
    room = torch.empty(far + D, dtype=F16, device="cuda")
    v = room.as_strided((T, D), (far, 1))
    v.copy_(x)
    i = info(api, handle, v)
    op = api.AddNorm(handle, i, i, eps=1e-5)
    op.execute(now(), at(room), 0, at(room))           # in place
    ey = norm_forward(x, None, None, 1e-5)[1]
    check(v, ey, (UNIT[F16] + NORM_CHAIN * E32) * ey.abs() + FLOOR[F16])
