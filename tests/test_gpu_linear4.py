"""Products with 4-bit weights on the GPU against a plain 64-bit implementation."""
import math

import pytest
import torch

import helpers
from decoder_reference import E32, UNIT
from layer_reference import check, info, linear4, linear4_weights

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


def pieces(extent, group):
    return -(-extent // group) if group else 1


class Weights:
    def __init__(self, n, k, group, scale_type, zeros, kind, seed):
        g = torch.Generator().manual_seed(seed)
        rows = n if kind == "none" else 2 * n
        self.n, self.k, self.group, self.kind = n, k, group, kind
        self.codes = torch.randint(0, 256, (rows, (k + 1) // 2), generator=g, dtype=torch.uint8)
        self.scales = ((0.5 + torch.rand(rows, pieces(k, group), generator=g)) / math.sqrt(20 * k)).to(scale_type)
        self.zeros = torch.randint(0, 16, (rows, pieces(k, group)), generator=g, dtype=torch.uint8) if zeros else None
        self.exact = linear4_weights(self.codes, self.scales, self.zeros, group, k)

    def pack(self, op):
        packed = torch.full((op.packed_size(),), 255, dtype=torch.uint8, device="cuda")
        c, s, z = self.codes.cuda(), self.scales.cuda(), self.zeros.cuda() if self.zeros is not None else None
        op.pack(now(), at(c), at(s), at(z), at(packed))
        torch.cuda.synchronize()
        return packed


def inputs(t, k, dtype, x_group, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(t, k, generator=g) * 2
    if dtype != E4M3:
        return x.to(dtype), None
    return (x * 100).to(E4M3), torch.rand(t, pieces(k, x_group), generator=g) + 0.5


def operation(api, handle, w, x, xs, x_group, y):
    return api.Linear4(handle, info(api, handle, x), info(api, handle, y), scale_type=api.dtype_code(w.scales.dtype), group=w.group,
                       zeros=w.zeros is not None, activation=w.kind, XS=info(api, handle, xs) if xs is not None else None, x_group=x_group)


def work_of(op):
    return torch.empty(max(op.workspace_size(), 1), dtype=torch.uint8, device="cuda")


def run(api, handle, w, x, xs, x_group, out, y=None):
    if y is None:
        y = torch.full((x.shape[0], w.n), math.nan, dtype=out, device="cuda")
    op = operation(api, handle, w, x, xs, x_group, y)
    ws = work_of(op)
    op.execute(now(), at(w.pack(op)), at(x), at(y), XS=at(xs), workspace=at(ws), workspace_bytes=ws.numel())
    return y


SIZES = [(1, 1, 1), (1, 16, 64), (2, 5, 31), (3, 17, 33), (8, 33, 129), (9, 100, 100), (7, 777, 1001), (16, 48, 2048), (17, 200, 640), (33, 130, 257),
         (1, 4096, 4096), (8, 2056, 1024), (40, 1000, 4160), (64, 256, 8192), (5, 64, 9000), (65, 300, 512), (130, 520, 320)]


@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
@pytest.mark.parametrize("dtype,out,scale,group,x_group,zeros", [
    (F32, F32, F32, 32, 0, True), (F32, F32, F16, 128, 0, False), (F16, F16, F16, 128, 0, False), (F16, F16, F32, 64, 0, True), (BF16, BF16, BF16, 64, 0, True),
    (BF16, F32, F16, 32, 0, False), (BF16, BF16, BF16, 0, 0, True), (E4M3, BF16, F16, 128, 0, False), (E4M3, F16, BF16, 64, 128, True),
    (E4M3, F32, F32, 256, 32, False), (E4M3, BF16, F16, 0, 64, True), (E4M3, BF16, F16, 32, 128, False)])
@pytest.mark.parametrize("t,n,k", SIZES)
def test_products(api, handle, t, n, k, dtype, out, scale, group, x_group, zeros, kind):
    w = Weights(n, k, group, scale, zeros, kind, t + n + k)
    x, xs = inputs(t, k, dtype, x_group, k)
    y = run(api, handle, w, x.cuda(), xs.cuda() if xs is not None else None, x_group, out)
    want, bound = linear4(x, xs, x_group, w.exact, kind, out)
    check(y, want, bound)


@pytest.mark.parametrize("dtype", [F32, F16, BF16, E4M3])
@pytest.mark.parametrize("t", [3, 19, 40])
def test_strides_and_alignment(api, handle, dtype, t):
    n, k, group, x_group = 77, 520, 128, 64
    w = Weights(n, k, group, F16, True, "none", 3)
    x, xs = inputs(t, k, dtype, x_group if dtype == E4M3 else 0, 4)
    out = F32 if dtype == F32 else BF16
    want, bound = linear4(x, xs, x_group if dtype == E4M3 else 0, w.exact, "none", out)
    for extra, first, apart in ((16, 0, 1), (3, 0, 1), (0, 1, 1), (0, 0, 2), (24, 8, 1)):
        room = torch.zeros(first + t * (k * apart + extra), dtype=dtype, device="cuda")
        v = room[first:].view(t, -1)[:, :k * apart:apart]
        v.copy_(x)
        s = None
        if xs is not None:
            s = torch.zeros(xs.shape[1], t + 1, device="cuda").T[:t]
            s.copy_(xs)
        y = torch.full((n, t + 2), math.nan, dtype=out, device="cuda").T[:t]
        run(api, handle, w, v, s, x_group if dtype == E4M3 else 0, out, y)
        check(y, want, bound)
        assert torch.isnan(y.as_strided((n, 2), (t + 2, 1), y.storage_offset() + t)).all()       # what lies beside is left alone
    # one row for all tokens
    one = x[:1].cuda().expand(t, k)
    s = xs[:1].cuda().expand(t, -1) if xs is not None else None
    y = run(api, handle, w, one, s, x_group if dtype == E4M3 else 0, out)
    want, bound = linear4(x[:1].expand(t, k), xs[:1].expand(t, -1) if xs is not None else None, x_group if dtype == E4M3 else 0, w.exact, "none", out)
    check(y, want, bound)


def test_one_packing_for_any_number_of_tokens(api, handle):
    n, k = 400, 1500
    w = Weights(n, k, 64, BF16, True, "silu", 8)
    packed = None
    for t, dtype in ((1, BF16), (5, F16), (24, BF16), (64, F32), (100, E4M3)):
        x, xs = inputs(t, k, dtype, 0, t)
        cx, cs = x.cuda(), xs.cuda() if xs is not None else None
        y = torch.full((t, n), math.nan, dtype=BF16, device="cuda")
        op = operation(api, handle, w, cx, cs, 0, y)
        if packed is None:
            packed = w.pack(op)
        assert op.packed_size() == packed.numel()
        ws = work_of(op)
        op.execute(now(), at(packed), at(cx), at(y), XS=at(cs), workspace=at(ws), workspace_bytes=ws.numel())
        want, bound = linear4(x, xs, 0, w.exact, "silu", BF16)
        check(y, want, bound)


@pytest.mark.parametrize("t", [1, 12, 48])
def test_lost_scales_and_inputs_stay_in_their_rows(api, handle, t):
    """A scale or a token that is NaN spoils its column or row, nothing else; the largest inputs stay finite."""
    n, k = 60, 300
    w = Weights(n, k, 128, F32, False, "none", 5)
    w.scales[7, 1] = math.nan
    w.exact = linear4_weights(w.codes, w.scales, None, 128, k)
    for dtype in (F32, BF16, E4M3):
        x, xs = inputs(t, k, dtype, 0, 6)
        if xs is not None:
            xs[0] = math.nan
        else:
            x[0, 299] = math.nan
        y = run(api, handle, w, x.cuda(), xs.cuda() if xs is not None else None, 0, F32)
        assert torch.isnan(y[0]).all() and torch.isnan(y[:, 7]).all()
        keep = [i for i in range(n) if i != 7]
        want, bound = linear4(x[1:], xs[1:] if xs is not None else None, 0, w.exact[keep], "none", F32)
        if t > 1:
            check(y[1:, keep], want, bound)


@pytest.mark.parametrize("t", [1, 8, 32])
def test_graphs_on_two_streams_at_once(api, handle, t):
    n, k = 2000, 2048
    sets = []
    for seed in (1, 2):
        w = Weights(n, k, 128, F16, False, "silu", seed)
        x, _ = inputs(t, k, F16, 0, seed)
        cx, y = x.cuda(), torch.zeros(t, n, dtype=F16, device="cuda")
        op = operation(api, handle, w, cx, None, 0, y)
        packed, ws = w.pack(op), work_of(op)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                op.execute(now(), at(packed), at(cx), at(y), workspace=at(ws), workspace_bytes=ws.numel())
        sets.append((w, x, cx, y, op, packed, ws, stream, graph))
    for _ in range(4):
        for z in sets:
            with torch.cuda.stream(z[7]):
                z[8].replay()
    torch.cuda.synchronize()
    first = []
    for w, x, cx, y, *_ in sets:
        want, bound = linear4(x, None, 0, w.exact, "silu", F16)
        check(y, want, bound)
        first.append(y.clone())
    for z, was in zip(sets, first):
        z[8].replay()
        torch.cuda.synchronize()
        assert torch.equal(z[3], was)                    # same inputs, same bits


def test_offsets_beyond_32_bits(api, handle):
    """Rows of x and y more than 2^32 bytes apart."""
    t, n, k, far = 2, 40, 256, (1 << 31) + 64
    w = Weights(n, k, 64, F16, False, "none", 4)
    x, _ = inputs(t, k, F16, 0, 1)
    room = torch.empty(far + k, dtype=F16, device="cuda")
    v = room.as_strided((t, k), (far, 1))
    v.copy_(x)
    y = torch.empty(far + n, dtype=F16, device="cuda").as_strided((t, n), (far, 1))
    run(api, handle, w, v, None, 0, F16, y)
    want, bound = linear4(x, None, 0, w.exact, "none", F16)
    check(y, want, bound)
