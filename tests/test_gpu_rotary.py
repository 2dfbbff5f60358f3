"""Head norm and rotary positions on the GPU against a plain 64-bit implementation: layouts, part of the head,
long positions, strides, alignment, pages, in place, backward (formula, differences), streams, graphs."""
import math

import pytest
import torch

import helpers
from decoder_reference import E32, FLOOR, UNIT, rotary_backward, rotary_forward

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def info(api, handle, t):
    return api.TensorInfo(handle, api.dtype_code(t.dtype), t.shape, t.stride())


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def close(got, want, scale, dtype, chain):
    """|got - want| <= u |want| + chain e scale (+ half the subnormal spacing of f16)."""
    got, want = got.double().cpu(), want.double()
    bound = UNIT[dtype] * want.abs() + chain * E32 * scale + FLOOR[dtype] + 1e-300
    bad = (got - want).abs() > bound
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / bound).max()))


def scale_of(y, mult):
    """Sum of moduli of the two terms of a rotated value is at most sqrt(2) times the pair's norm: bounded by
    the head's largest modulus."""
    return 2.0 * y.abs().amax(-1, keepdim=True).clamp(min=1e-30) * max(1.0, abs(mult))


# a rotated value: norm (mean of D squares, rsqrt: ~ 8 roundings), weight, cos / sin (argument of 2^-24 turns error,
# function 2 units, multiplier) and two products: below 24 + the angle's rounding pi 2^-25 / 2^-24 < 2
CHAIN = 32


CASES = [
    # T, Hq, Hk, D, pairs, interleaved, norm
    (1, 1, 1, 2, 1, False, True),
    (1, 1, 0, 1, 0, False, True),          # a head of one value, nothing rotated
    (3, 5, 1, 7, 3, True, True),           # odd head size
    (3, 5, 2, 9, 2, False, True),          # odd, half layout, part rotated
    (17, 4, 2, 64, 32, False, True),
    (17, 4, 2, 64, 32, True, True),
    (5, 32, 8, 128, 64, False, True),
    (5, 32, 8, 128, 64, True, False),
    (33, 6, 3, 80, 16, False, True),
    (33, 6, 3, 80, 18, True, True),
    (7, 3, 1, 96, 48, False, False),
    (7, 3, 1, 72, 36, True, True),
    (9, 2, 2, 256, 128, False, True),
    (9, 2, 2, 256, 128, True, True),
    (9, 2, 1, 256, 0, False, True),        # norm alone
    (300, 9, 3, 128, 32, False, True),     # ragged groups of heads
    (2000, 24, 8, 128, 64, False, True),   # several heads to a group of lanes
]


def make(case, dtype, seed, packed):
    T, Hq, Hk, D, pairs, inter, norm = case
    g = gen(seed)
    if packed:
        x = torch.randn(T, Hq + Hk, D, generator=g).to(dtype)
        xq, xk = x[:, :Hq], x[:, Hq:]
    else:
        xq, xk = torch.randn(T, Hq, D, generator=g).to(dtype), torch.randn(T, max(Hk, 1), D, generator=g).to(dtype)[:, :Hk]
    wq = (1 + 0.2 * torch.randn(D, generator=g)).to(dtype)
    wk = (1 + 0.2 * torch.randn(D, generator=g)).to(dtype)
    pos = torch.randint(0, 200000, (T,), generator=g, dtype=torch.int32)
    pos[0] = 0
    if T > 2:
        pos[1], pos[2] = 2 ** 31 - 1, -5
    freq = [10000.0 ** (-2.0 * i / max(2 * pairs, 1)) for i in range(pairs)]
    return xq, xk, wq, wk, pos, freq


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(api, handle, case, dtype):
    T, Hq, Hk, D, pairs, inter, norm = case
    xq, xk, wq, wk, pos, freq = make(case, dtype, 11, packed=True)
    mult, eps = 1.25, 1e-5
    packed = torch.cat((xq, xk), 1).cuda()
    dxq, dxk = packed[:, :Hq], packed[:, Hq:]
    yq, yk = torch.empty(T, Hq, D, dtype=dtype, device="cuda"), torch.empty(T, max(Hk, 1), D, dtype=dtype, device="cuda")
    k = dict(Xk=info(api, handle, dxk), Yk=info(api, handle, yk[:, :Hk])) if Hk else {}
    op = api.Rotary(handle, freq, info(api, handle, dxq), info(api, handle, yq), interleaved=inter, norm=norm, eps=eps,
                    multiplier=mult, **k)
    cw = [w.cuda() for w in (wq, wk)]
    cpos = pos.cuda()
    stream = torch.cuda.current_stream().cuda_stream
    w_at = [w.data_ptr() if norm else 0 for w in cw]
    keys = (dxk.data_ptr(), yk.data_ptr()) if Hk else (0, 0)
    op.execute(stream, cpos.data_ptr(), w_at[0], w_at[1] if Hk else 0, dxq.data_ptr(), yq.data_ptr(), *keys)
    want = rotary_forward(xq, wq, pos, freq, mult, inter, norm, eps)
    close(yq, want, scale_of(want, mult), dtype, CHAIN)
    if Hk:
        want = rotary_forward(xk, wk, pos, freq, mult, inter, norm, eps)
        close(yk[:, :Hk], want, scale_of(want, mult), dtype, CHAIN)

    # backward
    g = gen(12)
    gq, gk = torch.randn(T, Hq, D, generator=g).to(dtype), torch.randn(T, max(Hk, 1), D, generator=g).to(dtype)[:, :Hk]
    cgq, cgk = gq.cuda(), gk.contiguous().cuda()
    grads = torch.full_like(packed, float("nan"))
    dwq, dwk = torch.full((D,), float("nan"), device="cuda"), torch.full((D,), float("nan"), device="cuda")
    n = op.workspace_size()
    ws = torch.full((max(n, 1),), 0xff, dtype=torch.uint8, device="cuda")
    keys = (dxk.data_ptr(), cgk.data_ptr(), grads[:, Hq:].data_ptr()) if Hk else (0, 0, 0)
    args = (stream, cpos.data_ptr(), w_at[0], w_at[1] if Hk else 0, dxq.data_ptr(), cgq.data_ptr(), grads.data_ptr(), *keys)
    dw = dict(dWq=dwq.data_ptr() if norm else 0, dWk=dwk.data_ptr() if norm and Hk else 0, workspace=ws.data_ptr(), workspace_bytes=n)
    op.backward(*args, **dw)
    first = (grads.clone(), dwq.clone(), dwk.clone())
    for x, w, gy, got, gw in ((xq, wq, gq, grads[:, :Hq], dwq),) + (((xk, wk, gk, grads[:, Hq:], dwk),) if Hk else ()):
        dx, dwant = rotary_backward(x, w, pos, freq, mult, inter, norm, eps, gy)
        xd = x.double()
        r = 1 / torch.sqrt((xd * xd).mean(-1, keepdim=True) + eps) if norm else torch.ones(1, dtype=torch.float64)
        # terms of dx: r |g| + r |n| mean|g n|, every head bounded by its largest modulus times r
        big = gy.double().abs().amax(-1, keepdim=True) * 3 * r * (1 + (xd * r).abs().amax(-1, keepdim=True) ** 2 if norm else 1)
        close(got, dx, big, dtype, 2 * CHAIN)
        if norm:
            rows = x.shape[0] * x.shape[1]
            dm = rotary_backward(x, None, pos, freq, mult, inter, False, eps, gy)[0]
            moduli = ((dm.abs() + gy.double().abs().amax(-1, keepdim=True)) * (xd * r).abs()).sum((0, 1))
            # a term carries CHAIN roundings, the sum at most rows / (a thread's share) + 40 more; a thread adds at most rows
            assert ((gw.double().cpu() - dwant).abs() <= (CHAIN + min(rows, 512) + 40) * E32 * moduli + 1e-30).all()
    # same bits again
    grads.fill_(float("nan"))
    op.backward(*args, **dw)
    assert torch.equal(first[0].view(torch.int16 if dtype != torch.float32 else torch.int32),
                       grads.view(torch.int16 if dtype != torch.float32 else torch.int32))
    if norm:
        assert torch.equal(first[1], dwq) and (not Hk or torch.equal(first[2], dwk))


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("inter", [False, True])
def test_gradient_against_differences(api, handle, norm, inter):
    """d/dx and d/dw of sum(dy * forward) by central differences of the 64-bit forward (h^2 error ~ 1e-10)."""
    T, H, D, pairs, eps, mult = 3, 2, 12, 4, 1e-3, 0.8
    g = gen(3)
    x, w, dy = (torch.randn(*s, generator=g) for s in ((T, H, D), (D,), (T, H, D)))
    pos = torch.tensor([0, 7, 1234], dtype=torch.int32)
    freq = [0.5 ** i for i in range(pairs)]
    f = lambda xx, ww: (rotary_forward(xx, ww, pos, freq, mult, inter, norm, eps) * dy.double()).sum().item()  # noqa: E731
    step = 1e-5
    dx, dw = torch.zeros(T, H, D, dtype=torch.float64), torch.zeros(D, dtype=torch.float64)
    xd, wd = x.double(), w.double()
    for i in range(x.numel()):
        e = torch.zeros(x.numel(), dtype=torch.float64)
        e[i] = step
        e = e.view_as(xd)
        dx.view(-1)[i] = (f(xd + e, wd) - f(xd - e, wd)) / (2 * step)
    for i in range(D):
        e = torch.zeros(D, dtype=torch.float64)
        e[i] = step
        dw[i] = (f(xd, wd + e) - f(xd, wd - e)) / (2 * step)
    cx, cw, cdy, cpos = x.cuda(), w.cuda(), dy.cuda(), pos.cuda()
    gx, gw = torch.empty_like(cx), torch.zeros(D, device="cuda")
    op = api.Rotary(handle, freq, info(api, handle, cx), info(api, handle, cdy), interleaved=inter, norm=norm, eps=eps, multiplier=mult)
    ws = torch.empty(max(op.workspace_size(), 1), dtype=torch.uint8, device="cuda")
    op.backward(torch.cuda.current_stream().cuda_stream, cpos.data_ptr(), cw.data_ptr() if norm else 0, 0,
                cx.data_ptr() if norm else 0, cdy.data_ptr(), gx.data_ptr(),
                dWq=gw.data_ptr() if norm else 0, workspace=ws.data_ptr(), workspace_bytes=op.workspace_size())
    assert (gx.double().cpu() - dx).abs().max() < 2e-5
    if norm:
        assert (gw.double().cpu() - dw).abs().max() < 2e-5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(20, 3, 128, 64, 16), (20, 2, 80, 18, 12), (1, 1, 64, 32, 8), (600, 4, 128, 64, 16)])
def test_append_to_pages(api, handle, dtype, shape):
    """Keys and values land in their slots; skipped and bad slots write nothing; everything else keeps its bits."""
    T, H, D, pairs, S = shape
    g = gen(5)
    P = T // S * 2 + 3
    x = torch.randn(T, 3 * H, D, generator=g).to(dtype)
    x[T // 2, 2 * H:] = float("inf")       # values pass unchanged, whatever they are
    x[0, 2 * H, 0] = float("nan")
    w = (1 + 0.1 * torch.randn(D, generator=g)).to(dtype)
    pos = torch.arange(T, dtype=torch.int32) + 70000
    slots = torch.randperm(P * S, generator=g)[:T].to(torch.int32)
    if T > 3:
        slots[1], slots[2], slots[3] = -1, P * S, 2 ** 31 - 1
    freq = [10000.0 ** (-i / pairs) for i in range(pairs)]
    cx = x.cuda()
    kp, vp = (torch.randn(P, S, H, D, generator=g).to(dtype).cuda() for _ in range(2))
    k0, v0 = kp.cpu().clone(), vp.cpu().clone()
    yq = torch.empty(T, H, D, dtype=dtype, device="cuda")
    parts = [cx[:, i * H:(i + 1) * H] for i in range(3)]
    op = api.Rotary(handle, freq, info(api, handle, parts[0]), info(api, handle, yq), info(api, handle, parts[1]),
                    info(api, handle, kp), info(api, handle, parts[2]), info(api, handle, vp), norm=True)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    cw, cpos, cslots = w.cuda(), pos.cuda(), slots.cuda()
    op.execute(torch.cuda.current_stream().cuda_stream, cpos.data_ptr(), cw.data_ptr(), 0, parts[0].data_ptr(),
               yq.data_ptr(), parts[1].data_ptr(), kp.data_ptr(), parts[2].data_ptr(), vp.data_ptr(), slots=cslots.data_ptr(),
               flags=flags.data_ptr())
    want_q = rotary_forward(x[:, :H], w, pos, freq, 1.0, False, True, 1e-6)
    want_k = rotary_forward(x[:, H:2 * H], None, pos, freq, 1.0, False, True, 1e-6)
    close(yq, want_q, scale_of(want_q, 1.0), dtype, CHAIN)
    ok = (slots >= 0) & (slots < P * S)
    at = slots[ok].long()
    got_k, got_v = kp.cpu().reshape(P * S, H, D), vp.cpu().reshape(P * S, H, D)
    close(got_k[at], want_k[ok], scale_of(want_k[ok], 1.0), dtype, CHAIN)
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    assert torch.equal(got_v[at].view(bits), x[ok, 2 * H:].contiguous().view(bits))
    rest = torch.ones(P * S, dtype=torch.bool)
    rest[at] = False
    assert torch.equal(got_k[rest].view(bits), k0.reshape(P * S, H, D)[rest].view(bits))
    assert torch.equal(got_v[rest].view(bits), v0.reshape(P * S, H, D)[rest].view(bits))
    assert flags.item() == (api.FLAG_BAD_SLOT if T > 3 else 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_alignment_and_in_place(api, handle, dtype):
    """Head-size stride other than one, misaligned bases, broadcast input, heads-first pages, in place."""
    T, H, D, pairs = 13, 3, 64, 32
    g = gen(8)
    freq = [10000.0 ** (-i / pairs) for i in range(pairs)]
    x = torch.randn(T, H, D, generator=g).to(dtype)
    pos = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)
    cpos = pos.cuda()
    want = rotary_forward(x, None, pos, freq, 1.0, False, True, 1e-6)
    stream = torch.cuda.current_stream().cuda_stream

    def run(cx, y):
        op = api.Rotary(handle, freq, info(api, handle, cx), info(api, handle, y), norm=True)
        op.execute(stream, cpos.data_ptr(), 0, 0, cx.data_ptr(), y.data_ptr())
        close(y, want, scale_of(want, 1.0), dtype, CHAIN)

    # x transposed: heads of stride T * H
    run(x.permute(2, 0, 1).contiguous().cuda().permute(1, 2, 0), torch.empty(T, H, D, dtype=dtype, device="cuda"))
    # one element off 16-byte alignment, in and out
    flat = torch.zeros(T * H * D + 1, dtype=dtype, device="cuda")
    flat[1:] = x.reshape(-1).cuda()
    out = torch.full((T * H * D + 2,), 7.0, dtype=dtype, device="cuda")
    run(flat[1:].view(T, H, D), out[1:-1].view(T, H, D))
    assert out[0] == 7.0 and out[-1] == 7.0
    # padded rows
    wide = torch.zeros(T, H, D + 8, dtype=dtype, device="cuda")
    wide[..., :D] = x.cuda()
    run(wide[..., :D], torch.empty(T, H, D + 24, dtype=dtype, device="cuda")[..., :D])
    # reversed tokens (negative stride)
    back = x.flip(0).cuda().contiguous()
    op = api.Rotary(handle, freq, api.TensorInfo(handle, api.dtype_code(dtype), (T, H, D), (-H * D, D, 1)),
                    api.TensorInfo(handle, api.dtype_code(dtype), (T, H, D), (H * D, D, 1)), norm=True)
    y = torch.empty(T, H, D, dtype=dtype, device="cuda")
    op.execute(stream, cpos.data_ptr(), 0, 0, back[T - 1].data_ptr(), y.data_ptr())
    close(y, want, scale_of(want, 1.0), dtype, CHAIN)
    # in place
    y = x.cuda().clone()
    run(y, y)
    # one head broadcast over all (stride zero in X): forward only
    one = x[:, :1].cuda()
    y = torch.empty(T, H, D, dtype=dtype, device="cuda")
    wide_info = api.TensorInfo(handle, api.dtype_code(dtype), (T, H, D), (H * D if False else one.stride(0), 0, 1))
    op = api.Rotary(handle, freq, wide_info, info(api, handle, y), norm=True)
    op.execute(stream, cpos.data_ptr(), 0, 0, one.data_ptr(), y.data_ptr())
    w1 = rotary_forward(x[:, :1], None, pos, freq, 1.0, False, True, 1e-6).expand(T, H, D)
    close(y, w1, scale_of(w1, 1.0), dtype, CHAIN)
    with pytest.raises(api.BtcError) as e:
        op.backward(stream, cpos.data_ptr(), 0, 0, one.data_ptr(), y.data_ptr(), y.data_ptr())
    assert e.value.code == api.ERR_D_ALIASING
    # dX in place of dY
    dy = torch.randn(T, H, D, generator=g).to(dtype)
    cx, io = x.cuda(), dy.cuda()
    op = api.Rotary(handle, freq, info(api, handle, cx), info(api, handle, io), norm=True)
    op.backward(stream, cpos.data_ptr(), 0, 0, cx.data_ptr(), io.data_ptr(), io.data_ptr())
    dx, _ = rotary_backward(x, None, pos, freq, 1.0, False, True, 1e-6, dy)
    xd = x.double()
    r = 1 / torch.sqrt((xd * xd).mean(-1, keepdim=True) + 1e-6)
    big = dy.double().abs().amax(-1, keepdim=True) * 3 * r * (1 + (xd * r).abs().amax(-1, keepdim=True) ** 2)
    close(io, dx, big, dtype, 2 * CHAIN)


def test_unrotated_infinities_stay_in_place(api, handle):
    """An infinity beyond the rotated part must not leak into its neighbour (no 0 * inf)."""
    for dtype in TYPES:
        for D, pairs in ((64, 16), (9, 2)):
            x = torch.ones(2, 1, D, dtype=dtype)
            x[0, 0, D - 1] = float("inf")
            cx, y, pos = x.cuda(), torch.empty(2, 1, D, dtype=dtype, device="cuda"), torch.tensor([3, 4], dtype=torch.int32, device="cuda")
            op = api.Rotary(handle, [0.1] * pairs, info(api, handle, cx), info(api, handle, y))
            op.execute(torch.cuda.current_stream().cuda_stream, pos.data_ptr(), 0, 0, cx.data_ptr(), y.data_ptr())
            y = y.cpu()
            assert torch.isinf(y[0, 0, D - 1]) and torch.isfinite(y[0, 0, :D - 1]).all() and torch.isfinite(y[1]).all()
            assert (y[0, 0, 2 * pairs:D - 1] == 1).all()


def test_offsets_beyond_32_bits(api, handle):
    """More than 2^31 elements in one tensor (vector form), tokens 2^31 bytes and more apart (scalar form)."""
    T, H, D, pairs = 420_000, 40, 128, 64
    freq = [10000.0 ** (-i / pairs) for i in range(pairs)]
    x = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda").normal_()
    pos = (torch.arange(T, device="cuda") % 100_003).to(torch.int32)
    rows = torch.tensor([0, 1, T // 2, 2 ** 31 // (H * D), 2 ** 31 // (H * D) + 1, T - 2, T - 1])
    kept = x[rows.cuda()].cpu()
    op = api.Rotary(handle, freq, info(api, handle, x), info(api, handle, x), norm=True)
    op.execute(torch.cuda.current_stream().cuda_stream, pos.data_ptr(), 0, 0, x.data_ptr(), x.data_ptr())      # in place
    want = rotary_forward(kept, None, pos[rows.cuda()].cpu(), freq, 1.0, False, True, 1e-6)
    close(x[rows.cuda()], want, scale_of(want, 1.0), torch.bfloat16, CHAIN)
    del x
    stride = 1_200_000_000
    flat = torch.zeros(2 * stride + 4 * D, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(flat, (3, 4, D), (stride, D, 1))
    x.copy_(torch.randn(3, 4, D, generator=gen(2)))
    kept = x.cpu().clone()
    y = torch.empty(3, 4, D, dtype=torch.bfloat16, device="cuda")
    op = api.Rotary(handle, freq, info(api, handle, x), info(api, handle, y), norm=True)
    op.execute(torch.cuda.current_stream().cuda_stream, pos.data_ptr(), 0, 0, x.data_ptr(), y.data_ptr())
    want = rotary_forward(kept, None, pos[:3].cpu(), freq, 1.0, False, True, 1e-6)
    close(y, want, scale_of(want, 1.0), torch.bfloat16, CHAIN)


def test_other_stream_and_graph(api, handle):
    T, H, D = 64, 4, 128
    x = torch.randn(T, H, D, device="cuda", dtype=torch.bfloat16)
    y = torch.empty_like(x)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freq, mult = api.rotary_frequencies(D, scaling="bands", factor=4.0)
    op = api.Rotary(handle, freq, info(api, handle, x), info(api, handle, y), norm=True, multiplier=mult)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        op.execute(torch.cuda.current_stream().cuda_stream, pos.data_ptr(), 0, 0, x.data_ptr(), y.data_ptr())
    for seed in (1, 2):
        x.copy_(torch.randn(T, H, D, generator=gen(seed)).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = rotary_forward(x.cpu(), None, pos.cpu(), freq, mult, False, True, 1e-6)
        close(y, want, scale_of(want, mult), torch.bfloat16, CHAIN)
    assert math.isfinite(float(y.float().sum()))
