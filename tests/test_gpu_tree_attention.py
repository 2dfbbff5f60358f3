"""Attention of trees of drafted tokens on the GPU against a plain 64-bit implementation."""
import math

import pytest
import torch

import helpers
from decoder_reference import attention_bounds
from layer_reference import check, info, mask_words, random_trees, tree_attention

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def now():
    return torch.cuda.current_stream().cuda_stream


class Problem:
    """Queries, a pool with pages in random order, tables, lengths; what no row may see is NaN."""

    def __init__(self, n, t, hq, hk, d, dv, page, lengths, dtype, seed=0, columns=None, scale=1.5, sees=None, unused=0, heads_first=False):
        g = torch.Generator().manual_seed(seed)
        self.t, self.page, self.lengths = t, page, lengths
        held = [-(-(x + t) // page) for x in lengths]
        pool = sum(held) + 3
        columns = columns or max(held)
        order = torch.randperm(pool, generator=g)
        self.table = torch.full((n, columns), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(held):
            self.table[i, :min(c, columns)] = order[at:at + min(c, columns)].to(torch.int32)
            at += c
        self.sees = random_trees(n, t, seed + 1, unused) if sees is None else sees
        self.q = (torch.randn(n, t, hq, d, generator=g) * scale).to(dtype)
        self.k = torch.randn(pool, page, hk, d, generator=g).to(dtype)
        self.v = torch.randn(pool, page, hk, dv, generator=g).to(dtype)
        # behind the drafts, and in pages of nobody
        mine = torch.zeros(pool, page, dtype=torch.bool)
        for i, x in enumerate(lengths):
            for j in range(min(x + t, columns * page)):
                mine[self.table[i, j // page].long(), j % page] = True
        self.k[~mine], self.v[~mine] = math.nan, math.nan
        if heads_first:
            self.k, self.v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (self.k, self.v))

    def gpu(self):
        self.cq, self.ck, self.cv, self.ctable = self.q.cuda(), self.k.cuda(), self.v.cuda(), self.table.cuda()
        self.clengths, self.cmasks = torch.tensor(self.lengths, dtype=torch.int32, device="cuda"), mask_words(self.sees).cuda()
        return self


def run(api, handle, p, window=0, scale=None, o=None, lse=True, flags=0, stream=None, ws=None):
    n, t, hq, d = p.cq.shape
    if o is None:
        o = torch.full((n, t, hq, p.cv.shape[-1]), math.nan, dtype=p.cq.dtype, device="cuda")
    op = api.TreeAttention(handle, *(info(api, handle, x) for x in (p.cq, p.ck, p.cv, p.ctable, p.cmasks, o)), scale=scale, window=window)
    out = torch.full((n, t, hq), math.nan, device="cuda") if lse else None
    ws = torch.full((op.workspace_size(),), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
    op.execute(stream or now(), p.cq.data_ptr(), p.ck.data_ptr(), p.cv.data_ptr(), p.ctable.data_ptr(), p.clengths.data_ptr(),
               p.cmasks.data_ptr(), o.data_ptr(), lse=out.data_ptr() if lse else 0, workspace=ws.data_ptr(), workspace_bytes=ws.numel(),
               flags=flags)
    return o, out, (op, ws)


def compare(p, o, lse, window=0, scale=None):
    scale = p.q.shape[-1] ** -0.5 if scale is None else scale
    want = tree_attention(p.cq, p.ck, p.cv, p.table, p.lengths, p.sees, scale, window)
    bo, bl = attention_bounds(*want, p.q.shape[-1], p.q.dtype)
    check(o, want[0], bo)
    if lse is not None:
        check(lse, want[1], bl)


CASES = [
    # n, t, hq, hk, d, dv, page, lengths, window
    (1, 1, 1, 1, 1, 1, 1, [0], 0),
    (1, 1, 8, 1, 64, 64, 16, [1], 0),
    (2, 3, 4, 2, 64, 64, 16, [0, 37], 0),
    (3, 5, 6, 2, 80, 72, 24, [100, 0, 15], 0),
    (2, 7, 3, 3, 7, 9, 3, [10, 50], 0),
    (1, 16, 32, 8, 128, 128, 16, [1500], 0),
    (4, 16, 8, 2, 128, 128, 16, [3, 128, 129, 700], 0),
    (3, 33, 7, 1, 64, 64, 8, [31, 32, 333], 0),
    (2, 64, 16, 2, 128, 128, 64, [1000, 63], 0),
    (2, 128, 4, 2, 128, 64, 32, [517, 128], 0),
    (2, 40, 20, 4, 80, 72, 24, [10, 1100], 0),
    (2, 9, 8, 8, 256, 256, 16, [77, 300], 0),
    (2, 20, 4, 1, 192, 128, 16, [150, 260], 0),
    (5, 12, 8, 2, 96, 96, 128, [1, 2, 3, 127, 900], 0),
    (3, 6, 8, 2, 64, 64, 16, [5, 100, 900], 6),
    (3, 10, 8, 2, 128, 128, 16, [5, 260, 901], 100),
    (2, 32, 16, 2, 128, 128, 16, [700, 290], 257),
    (4, 70, 12, 3, 64, 32, 20, [99, 0, 1, 450], 128),
    (40, 4, 4, 2, 64, 64, 16, [13 * i % 211 for i in range(40)], 0),
    (2, 8, 8, 1, 128, 128, 16, [9000, 4000], 0),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_trees(api, handle, case, dtype):
    n, t, hq, hk, d, dv, page, lengths, window = case
    p = Problem(n, t, hq, hk, d, dv, page, lengths, dtype, seed=t + d, unused=t // 3, heads_first=n % 2 == 0).gpu()
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    o, lse, _ = run(api, handle, p, window=window, flags=flags.data_ptr())
    compare(p, o, lse, window)
    assert flags.item() == 0
    again, _, _ = run(api, handle, p, window=window, lse=False)
    assert torch.equal(o, again)                         # same inputs, same bits


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.11, 1.5])
def test_scales(api, handle, dtype, scale):
    p = Problem(2, 11, 8, 2, 64, 64, 16, [200, 30], dtype, seed=12).gpu()
    o, lse, _ = run(api, handle, p, scale=scale, window=50)
    compare(p, o, lse, 50, scale)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_masks_of_any_kind(api, handle, dtype):
    """Rows that see nothing, only others, everything; a sequence without drafts; bits beyond the last draft."""
    n, t = 3, 37
    sees = torch.zeros(n, t, t, dtype=torch.bool)
    sees[0] = True
    sees[1] = torch.rand(t, t, generator=torch.Generator().manual_seed(1)) < 0.4
    sees[1, 5] = False
    sees[1, 6] = False
    sees[1, 6, 30] = True
    p = Problem(n, t, 8, 2, 64, 64, 16, [40, 250, 90], dtype, seed=4, sees=sees).gpu()
    p.cmasks[:, :, 1] |= -(1 << (t - 32))               # bits of drafts 37 to 63
    o, lse, _ = run(api, handle, p)
    compare(p, o, lse)
    assert not o[2].any() and (lse[2] == -math.inf).all() and not o[1, 5].any()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_a_chain_of_one_is_the_attention_of_one_token(api, handle, dtype):
    """One draft that sees itself: PagedAttention with the draft counted among the tokens."""
    p = Problem(5, 1, 8, 2, 128, 128, 16, [0, 1, 63, 700, 2100], dtype, seed=7).gpu()
    o, lse, _ = run(api, handle, p)
    q, one = p.cq[:, 0], torch.zeros_like(p.cq[:, 0])
    op = api.PagedAttention(handle, info(api, handle, q), info(api, handle, p.ck), info(api, handle, p.cv), info(api, handle, p.ctable), info(api, handle, one))
    ws, l1 = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda"), torch.zeros(5, 8, device="cuda")
    lengths = p.clengths + 1
    op.execute(now(), q.data_ptr(), p.ck.data_ptr(), p.cv.data_ptr(), p.ctable.data_ptr(), lengths.data_ptr(), one.data_ptr(), lse=l1.data_ptr(),
               workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    want = tree_attention(p.cq, p.ck, p.cv, p.table, p.lengths, p.sees, 128 ** -0.5, 0)
    bo, bl = attention_bounds(*want, 128, dtype)
    check(o[:, 0], one.cpu().double(), 2 * bo[:, 0])
    check(lse[:, 0], l1.cpu().double(), 2 * bl[:, 0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [3, 40])
def test_strides_and_alignment(api, handle, dtype, t):
    """Rows apart, cache elements shifted or apart, heads and drafts exchanged in the output; what lies beside is left alone."""
    p = Problem(2, t, 4, 2, 64, 64, 16, [35, 300], dtype, seed=2).gpu()
    o, lse, _ = run(api, handle, p)
    compare(p, o, lse)
    for extra, first in ((8, 0), (0, 1), (3, 0)):
        s = Problem(2, t, 4, 2, 64, 64, 16, [35, 300], dtype, seed=2).gpu()
        for name in ("ck", "cv", "cq"):
            x = getattr(s, name)
            room = torch.full((first + x.numel() // x.shape[-1] * (x.shape[-1] + extra),), math.nan, dtype=dtype, device="cuda")
            v = room[first:].view(*x.shape[:-1], -1)[..., :x.shape[-1]]
            v.copy_(x)
            setattr(s, name, v)
        s.ctable = torch.full((2, 2 * s.ctable.shape[1]), -7, dtype=torch.int32, device="cuda")[:, ::2].copy_(s.ctable)
        s.cmasks = torch.full((t, 2, s.cmasks.shape[2] + 1), 0, dtype=torch.int32, device="cuda").transpose(0, 1)[:, :, :-1].copy_(s.cmasks)
        out = torch.full((4, 2, t, 66), math.nan, dtype=dtype, device="cuda").permute(1, 2, 0, 3)[..., :64]
        run(api, handle, s, o=out, lse=False)
        compare(s, out, None)
        assert torch.isnan(out.as_strided((4 * 2 * t, 2), (66, 1), out.storage_offset() + 64)).all()
    # elements of the cache two apart
    s = Problem(2, t, 4, 2, 64, 64, 16, [35, 300], dtype, seed=2).gpu()
    for name in ("ck", "cv", "cq"):
        x = getattr(s, name)
        setattr(s, name, torch.full((*x.shape[:-1], 2 * x.shape[-1]), math.nan, dtype=dtype, device="cuda")[..., ::2].copy_(x))
    out, lse, _ = run(api, handle, s)
    compare(s, out, lse)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("t", [4, 48])
def test_bad_lengths_and_pages(api, handle, dtype, t):
    """Lengths below zero and beyond the row, pages that do not exist: reported, not followed, the other sequences as ever."""
    p = Problem(5, t, 8, 2, 64, 64, 16, [20, 100, 64, 150, 128 - t], dtype, seed=3, columns=8).gpu()
    p.table[1, 2] = p.k.shape[0] + 5
    p.table[1, 4] = -3
    p.lengths[0], p.lengths[2], p.lengths[3] = -4, 10 ** 9, 128 - t + 2
    # every token of the row may be read now: pages of its own, no NaN
    spare = torch.randn(p.k.shape, generator=torch.Generator().manual_seed(1)).to(dtype)
    p.k, p.v = torch.where(torch.isnan(p.k), spare, p.k), torch.where(torch.isnan(p.v), spare[..., :p.v.shape[-1]], p.v)
    p.table[2], p.table[3] = torch.arange(8, dtype=torch.int32), torch.arange(8, dtype=torch.int32) + 1
    p.gpu()
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    o, lse, _ = run(api, handle, p, flags=flags.data_ptr())
    compare(p, o, lse)
    assert flags.item() == api.FLAG_BAD_LENGTH | api.FLAG_BAD_PAGE
    o2, _, _ = run(api, handle, p, window=max(t, 20))
    compare(p, o2, None, max(t, 20))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_large_and_infinite_scores(api, handle, dtype):
    """Scores far apart from one another, rows whose visible scores are all -inf, infinities and NaN in drafts that nobody sees."""
    t = 24
    sees = torch.zeros(2, t, t, dtype=torch.bool)
    for i in range(t - 4):
        sees[:, i, i] = True
        if i:
            sees[:, i, i - 1] = True
    p = Problem(2, t, 8, 2, 64, 64, 16, [300, 41], dtype, seed=6, sees=sees, scale=30.0)
    flat = p.k.view(-1, 2, 64)
    for i, x in enumerate(p.lengths):
        for j in range(t - 4, t):                        # drafts that no row sees
            slot = int(p.table[i, (x + j) // 16]) * 16 + (x + j) % 16
            flat[slot], p.v.view(-1, 2, 64)[slot] = math.inf, math.nan
    p.gpu()
    o, lse, _ = run(api, handle, p)
    compare(p, o, lse)
    # every key minus infinity along a query of ones
    p = Problem(1, 3, 2, 1, 64, 64, 16, [20], dtype, seed=8)
    p.q[:] = 1.0
    p.k[:] = 0.0
    p.k[..., 0] = -math.inf
    p.v[:] = 3.0
    p.gpu()
    o, lse, _ = run(api, handle, p)
    assert not o.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("t", [4, 40])
def test_graph_on_other_streams_lengths_change(api, handle, t):
    """Two captured passes with a workspace each, replayed at once; the cache grows between replays."""
    sets = []
    for seed in (1, 2):
        p = Problem(6, t, 8, 2, 128, 128, 16, [400, 300, 200, 100, 50, 0], BF16, seed=seed).gpu()
        spare = torch.randn(p.k.shape, generator=torch.Generator().manual_seed(9)).to(BF16)
        p.k, p.v = torch.where(torch.isnan(p.k), spare, p.k), torch.where(torch.isnan(p.v), spare, p.v)
        p.gpu()
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            o, lse, keep = run(api, handle, p)
        sets.append((p, stream, graph, o, lse, keep))
    for lengths in ([400, 300, 200, 100, 50, 0], [1, 40, 199, 77, 60, 3], [0, 0, 0, 0, 0, 0]):
        torch.cuda.synchronize()
        for p, stream, graph, o, lse, keep in sets:
            p.lengths = lengths
            p.clengths.copy_(torch.tensor(lengths, dtype=torch.int32))
            o.fill_(math.nan)
        torch.cuda.synchronize()
        for _ in range(2):
            for p, stream, graph, o, lse, keep in sets:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for p, stream, graph, o, lse, keep in sets:
            # pages that this length does not reach are -1 in no table here, so all of it can be read
            compare(p, o, lse)


@pytest.mark.parametrize("dtype,t", [(BF16, 5), (F16, 33), (F32, 5)])
def test_offsets_beyond_32_bits(api, handle, dtype, t):
    """A pool of more than 2^32 bytes with the used pages at its end."""
    d, page, hk = 128, 16, 2
    elements = (1 << 33) // torch.finfo(dtype).bits + (1 << 22)          # just above 2^30 bytes' worth more than 4 GiB in bytes
    pages = (elements * 4) // (page * hk * d)
    p = Problem(1, t, 8, hk, d, d, page, [200], dtype, seed=3).gpu()
    k = torch.empty(pages, page, hk, d, dtype=dtype, device="cuda")
    v = torch.empty_like(k)
    n = p.ck.shape[0]
    k[-n:], v[-n:] = p.ck, p.cv
    assert (pages - n) * page * hk * d * k.element_size() > 1 << 32
    small_k, small_v, table = p.ck, p.cv, p.ctable
    p.ck, p.cv, p.ctable = k, v, torch.where(table >= 0, table + (pages - n), table).to(torch.int32)
    o, lse, _ = run(api, handle, p)
    p.ck, p.cv = small_k, small_v
    compare(p, o, lse)


def test_tree_masks(api, handle):
    masks, depth = api.tree_masks([-1, 0, 0, 2, -1, -2] + [4] * 30)
    assert depth[:7] == [0, 1, 1, 2, 0, -1, 1] and masks[3] == [0b1101, 0] and masks[5] == [0, 0] and masks[31][0] == -(1 << 31) + 16
    assert masks[35] == [16, 1 << 3]
