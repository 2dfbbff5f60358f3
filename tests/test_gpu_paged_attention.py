"""Attention of one token over a paged cache against a plain 64-bit implementation.

Error bound (decoder_reference.attention_bounds), derived before the first run.  A score is a sum of D products
in fp32 (any order, the tensor core may truncate: 2 D + 8 units of the sum of moduli), scaled (4 units of |s|);
for fp32 each product misses at most 2^-22 of itself on either side (2^-20 taken).  exp2 of it and the sums keep
relative errors of the probabilities at twice the score's plus 8 units.  Probabilities enter the second product in
two parts (bf16: 2^-16 left out, 2^-15 taken; f16 and fp32 2^-20).  Output sums run over tiles of 16 tokens and
joins: 4 (tokens / 16 + 64) units of sum p|v|.  Then one rounding to the type."""
import math

import pytest
import torch

import helpers
from decoder_reference import attention, attention_bounds

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


def make(seed, N, Hq, Hk, D, Dv, S, lengths, dtype, spare=2, columns=None):
    """Inputs on the CPU; pages in random order, everything that no sequence sees is NaN."""
    g = torch.Generator()
    g.manual_seed(seed)
    need = [-(-max(0, n) // S) for n in lengths]
    P = sum(need) + spare
    M = columns or max(1, max(need))
    q = (torch.randn(N, Hq, D, generator=g) * 1.5).to(dtype)
    k = torch.full((P, S, Hk, D), float("nan"), dtype=dtype)
    v = torch.full((P, S, Hk, Dv), float("nan"), dtype=dtype)
    table = torch.full((N, M), -1, dtype=torch.int32)
    order = torch.randperm(P, generator=g)
    at = 0
    for n in range(N):
        for j in range(need[n]):
            page = int(order[at])
            at += 1
            table[n, j] = page
            rows = min(S, lengths[n] - j * S)
            k[page, :rows] = torch.randn(rows, Hk, D, generator=g).to(dtype)
            v[page, :rows] = torch.randn(rows, Hk, Dv, generator=g).to(dtype)
    return q, k, v, table, torch.tensor(lengths, dtype=torch.int32)


def run(api, handle, q, k, v, table, lengths, scale, window, o=None, lse=True):
    """Arguments on the GPU, any strides; returns o, lse, flags (workspace holds garbage before)."""
    N, Hq, _ = q.shape
    o = torch.full((N, Hq, v.shape[-1]), float("nan"), dtype=q.dtype, device="cuda") if o is None else o
    out = torch.full((N, Hq), float("nan"), device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    op = api.PagedAttention(handle, info(api, handle, q), info(api, handle, k), info(api, handle, v), info(api, handle, table),
                            info(api, handle, o), scale=scale, window=window)
    ws = torch.full((op.workspace_size(),), 0x7f, dtype=torch.uint8, device="cuda")
    op.execute(torch.cuda.current_stream().cuda_stream, q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(),
               lengths.data_ptr(), o.data_ptr(), lse=out.data_ptr() if lse else 0, workspace=ws.data_ptr(),
               workspace_bytes=ws.numel(), flags=flags.data_ptr())
    torch.cuda.synchronize()
    return o, out, flags.item()


def check(o, lse, want, dim, dtype):
    bo, bl = attention_bounds(*want, dim, dtype)
    eo = (o.double().cpu() - want[0]).abs()
    assert (eo <= bo).all(), float((eo / bo).max())
    if lse is not None:
        got, ref = lse.double().cpu(), want[1]
        empty = torch.isinf(ref)
        assert torch.equal(torch.isinf(got), empty) and (got[empty] < 0).all()
        el = (got - ref).abs()[~empty]
        assert (el <= bl[~empty]).all(), float((el / bl[~empty]).max())


SHAPES = [
    # N, Hq, Hk, D, Dv, S, lengths, window
    (1, 1, 1, 8, 8, 1, [1], 0),
    (3, 2, 1, 16, 16, 16, [0, 1, 2], 0),
    (6, 4, 2, 64, 64, 16, [15, 16, 17, 31, 32, 33], 0),
    (5, 8, 1, 128, 128, 8, [7, 8, 9, 63, 100], 0),
    (4, 32, 8, 128, 128, 16, [300, 0, 1, 77], 0),
    (2, 9, 1, 128, 128, 16, [130, 250], 0),          # more than 8 heads to a key head
    (2, 12, 1, 64, 64, 64, [65, 129], 0),
    (2, 20, 1, 96, 96, 32, [33, 200], 0),            # two blocks of 16
    (2, 33, 1, 128, 128, 16, [50, 17], 0),
    (2, 66, 2, 40, 40, 16, [50, 17], 0),
    (2, 10, 1, 256, 256, 16, [90, 33], 0),           # two blocks of 8
    (3, 5, 5, 80, 72, 24, [24, 25, 100], 0),
    (3, 3, 3, 192, 128, 16, [16, 40, 5], 0),
    (3, 6, 2, 72, 200, 12, [12, 13, 300], 0),
    (3, 14, 2, 20, 20, 5, [4, 5, 101], 0),           # rows of 40 bytes: no 16-byte copies
    (2, 3, 1, 7, 9, 3, [10, 50], 0),
    (2, 3, 1, 1, 1, 3, [10, 50], 0),
    (4, 8, 2, 128, 128, 16, [100, 5, 64, 200], 64),  # window
    (4, 8, 2, 64, 64, 16, [100, 1, 17, 16], 1),
    (4, 6, 2, 80, 80, 24, [100, 1, 50, 49], 49),
    (1, 8, 1, 128, 128, 16, [5000], 0),              # one sequence over all SMs
    (1, 3, 1, 64, 64, 16, [9001], 0),
    (2, 2, 1, 256, 256, 64, [3001, 10], 0),
    (3, 16, 2, 128, 128, 16, [1500, 2, 2300], 1400),
    (40, 2, 2, 32, 32, 16, [(37 * i) % 90 for i in range(40)], 0),
    (700, 2, 1, 64, 64, 16, [(i * 7) % 23 for i in range(700)], 0),   # more sequences than threads
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_against_definition(api, handle, shape, dtype):
    N, Hq, Hk, D, Dv, S, lengths, window = shape
    x = make(21, N, Hq, Hk, D, Dv, S, lengths, dtype)
    scale = 1.0 / math.sqrt(D)
    want = attention(*x, scale, window)
    gpu = [t.cuda() for t in x]
    o, lse, flags = run(api, handle, *gpu, scale, window)
    check(o, lse, want, D, dtype)
    assert flags == 0
    again, lse2, _ = run(api, handle, *gpu, scale, window)
    assert torch.equal(o.view(torch.uint8), again.view(torch.uint8)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))
    without, _, _ = run(api, handle, *gpu, scale, window, lse=False)
    assert torch.equal(o.view(torch.uint8), without.view(torch.uint8))


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(api, handle, dtype):
    """Heads-first pages, strided queries, outputs and tables, unaligned bases, keys and values in one buffer."""
    N, Hq, Hk, D, S, lengths = 3, 6, 2, 64, 16, [40, 3, 90]
    x = make(5, N, Hq, Hk, D, D, S, lengths, dtype)
    want = attention(*x, 0.2, 0)
    q, k, v, table, ln = (t.cuda() for t in x)

    def ok(q, k, v, table, o=None):
        o, lse, flags = run(api, handle, q, k, v, table, ln, 0.2, 0, o=o)
        check(o, lse, want, D, dtype)
        assert flags == 0

    heads_first = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    ok(q, heads_first(k), heads_first(v), table)
    both = torch.stack((k, v), 1)                                    # [P, 2, S, Hk, D]
    ok(q, both[:, 0], both[:, 1], table)
    packed = torch.zeros(N, 3 * Hq, D + 3, dtype=dtype, device="cuda")
    packed[:, Hq:2 * Hq, :D] = q
    ok(packed[:, Hq:2 * Hq, :D], k, v, table)
    ok(q.permute(2, 0, 1).contiguous().permute(1, 2, 0), k, v, table)
    ok(q, k.permute(3, 0, 1, 2).contiguous().permute(1, 2, 3, 0), v, table)      # head elements far apart
    ok(q, k, v, table.T.contiguous().T)
    wide = torch.full((N, 7), 123456789, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    ok(q, k, v, wide[:, :table.shape[1]])
    shifted = torch.zeros(k.numel() + 1, dtype=dtype, device="cuda")
    shifted[1:] = k.reshape(-1)
    ok(q, shifted[1:].view(k.shape), v, table)
    o = torch.full((N, Hq, D + 5), 7.0, dtype=dtype, device="cuda")
    ok(q, k, v, table, o=o[..., :D])
    assert (o[..., D:] == 7).all()
    ok(q, k, v, table, o=torch.empty(Hq, N, D, dtype=dtype, device="cuda").transpose(0, 1))


def test_bad_pages_and_lengths(api, handle):
    """Entries that are no pages are not visible and reported; lengths are clamped to what a row can hold."""
    N, Hq, Hk, D, S = 5, 4, 1, 64, 16
    x = list(make(9, N, Hq, Hk, D, D, S, [40, 40, 48, 48, 48], torch.bfloat16))
    x[3][0, 1], x[3][1, 0], x[3][1, 1], x[3][1, 2] = -1, 10 ** 9, -7, x[1].shape[0]
    x[4] = torch.tensor([40, 40, -3, 2 ** 31 - 1, 48], dtype=torch.int32)
    want = attention(*x, 0.125, 0)
    o, lse, flags = run(api, handle, *[t.cuda() for t in x], 0.125, 0)
    check(o, lse, want, D, torch.bfloat16)
    assert flags == api.FLAG_BAD_PAGE | api.FLAG_BAD_LENGTH
    assert (o[1] == 0).all() and (o[2] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinite_scores(api, handle, dtype):
    """A NaN among the visible keys reaches its sequence only; scores of -inf weigh nothing; all -inf gives zero."""
    N, D, S = 3, 64, 16
    x = make(13, N, 2, 1, D, D, S, [70, 70, 70], dtype)
    q, k, v, table, ln = x
    k[table[0, 2].item(), 5, 0, 3] = float("nan")
    q[1:, :, 0] = 1.0
    inf_rows = [(0, r) for r in range(16)] + [(3, 4)]
    for j, r in inf_rows:
        k[table[1, j].item(), r, 0, 0] = float("-inf")
    for j in range(5):
        k[table[2, j].item(), :, 0, 0] = float("-inf")
    scale = 0.125
    o, lse, _ = run(api, handle, *[t.cuda() for t in x], scale, 0)
    assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all()
    assert (o[2] == 0).all() and (lse[2] == -math.inf).all()
    keep = [(j, r) for j in range(5) for r in range(16) if j * 16 + r < 70 and (j, r) not in inf_rows]
    kk = torch.stack([k[table[1, j].item(), r, 0] for j, r in keep]).double()
    vv = torch.stack([v[table[1, j].item(), r, 0] for j, r in keep]).double()
    for h in range(2):
        p = torch.softmax(kk @ q[1, h].double() * scale, 0)
        assert ((o[1, h].double().cpu() - p @ vv).abs() < 2e-2).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_large_scores(api, handle, dtype):
    """Scores of several hundred: one key takes all; nothing overflows."""
    x = make(17, 1, 8, 1, 128, 128, 16, [900], dtype)
    x[0].mul_(30)
    want = attention(*x, 1.0 / math.sqrt(128), 0)
    o, lse, _ = run(api, handle, *[t.cuda() for t in x], 1.0 / math.sqrt(128), 0)
    check(o, lse, want, 128, dtype)


def test_offsets_beyond_32_bits(api, handle):
    """Pages more than 2^31 elements apart."""
    D, S, stride = 64, 16, 1_200_000_000
    flat = torch.zeros(2 * stride + S * D, dtype=torch.bfloat16, device="cuda")
    k = torch.as_strided(flat, (3, S, 1, D), (stride, D, D, 1))
    g = torch.Generator()
    g.manual_seed(1)
    rows = torch.randn(3, S, 1, D, generator=g).to(torch.bfloat16)
    k.copy_(rows)
    q = torch.randn(1, 4, D, generator=g).to(torch.bfloat16)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    ln = torch.tensor([45], dtype=torch.int32)
    want = attention(q, rows, rows, table, ln, 0.125, 0)
    o, lse, _ = run(api, handle, q.cuda(), k, k, table.cuda(), ln.cuda(), 0.125, 0)
    check(o, lse, want, D, torch.bfloat16)


def test_graph_of_a_growing_cache(api, handle):
    """One captured call on a stream of its own serves every length."""
    N, Hq, Hk, D, S = 4, 8, 2, 128, 16
    x = make(31, N, Hq, Hk, D, D, S, [200, 150, 170, 10], torch.bfloat16)
    q, k, v, table, ln = (t.cuda() for t in x)
    o, lse = torch.empty(N, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(N, Hq, device="cuda")
    op = api.PagedAttention(handle, *(info(api, handle, t) for t in (q, k, v, table, o)))
    ws = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")

    def call():
        op.execute(torch.cuda.current_stream().cuda_stream, q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(),
                   ln.data_ptr(), o.data_ptr(), lse=lse.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for lengths in ([200, 150, 170, 10], [1, 0, 16, 3], [64, 149, 33, 9]):
        ln.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = attention(x[0], x[1], x[2], x[3], torch.tensor(lengths), 1 / math.sqrt(D), 0)
        check(o, lse, want, D, torch.bfloat16)
