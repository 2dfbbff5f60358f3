"""Cache pages on the GPU against a step-by-step Python model: whole numbers and page contents have to be equal."""
import random

import pytest
import torch

import helpers
from decoder_reference import PagesState

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def info(api, handle, t):
    return api.TensorInfo(handle, api.dtype_code(t.dtype), t.shape, t.stride())


class Machine:
    """The same state on the GPU and in the model; every step runs on both and compares all of it."""

    def __init__(self, api, handle, N, M, P, S, pools=None, table_t=False, refs_offset=0):
        self.api, self.N, self.M, self.P, self.S = api, N, M, P, S
        self.table = torch.full((M, N), -1, dtype=torch.int32, device="cuda").T if table_t else torch.full((N, M), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(N, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(P + refs_offset, dtype=torch.int32, device="cuda")[refs_offset:]
        self.pools = pools if pools is not None else [torch.randint(-30000, 30000, (P, S, 2, 8), dtype=torch.int32, device="cuda").to(torch.bfloat16)]
        self.model_pools = [p.cpu().clone() for p in self.pools]
        self.model = PagesState(self.table.tolist(), [0] * N, [0] * P, S)
        self.op = api.Pages(handle, [info(api, handle, p) for p in self.pools][:4], info(api, handle, self.table), S)
        self.ws = torch.full((self.op.workspace_size(),), 0x5a, dtype=torch.uint8, device="cuda")
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")

    @property
    def stream(self):
        return torch.cuda.current_stream().cuda_stream

    def pointers(self):
        return [p.data_ptr() for p in self.pools]

    def state(self):
        return self.table.data_ptr(), self.lengths.data_ptr(), self.refs.data_ptr()

    def ints(self, values):
        return torch.tensor(list(values) or [0], dtype=torch.int32, device="cuda")

    def move(self, moves):
        for pool in self.model_pools:
            old = pool.clone()
            for a, b in moves:
                pool[b] = old[a]

    def same(self):
        torch.cuda.synchronize()
        assert self.table.tolist() == self.model.table
        assert self.lengths.tolist() == self.model.lengths
        assert self.refs.tolist() == self.model.refs
        for a, b in zip(self.pools, self.model_pools):
            assert torch.equal(a.cpu(), b)

    def extend(self, new, most, bare=False):
        slots = torch.full((self.N, most), -77, dtype=torch.int32, device="cuda")
        n = self.ints(new)
        self.op.extend(self.stream, n.data_ptr(), *self.state(), slots.data_ptr(), most, [] if bare else self.pointers(),
                       workspace=self.ws.data_ptr(), workspace_bytes=self.ws.numel(), flags=self.flags.data_ptr())
        want, moves = self.model.extend(list(new), most)
        if not bare:
            self.move(moves)
        self.same()
        assert slots.tolist() == want
        return moves

    def fork(self, src, dst):
        a, b = self.ints(src), self.ints(dst)
        self.op.fork(self.stream, a.data_ptr(), b.data_ptr(), len(src), *self.state(), flags=self.flags.data_ptr())
        self.model.fork(src, dst)
        self.same()

    def free(self, sequences):
        a = self.ints(sequences)
        self.op.free(self.stream, a.data_ptr(), len(sequences), *self.state(), flags=self.flags.data_ptr())
        self.model.free(sequences)
        self.same()

    def compact(self):
        self.op.compact(self.stream, self.table.data_ptr(), self.refs.data_ptr(), self.pointers(), workspace=self.ws.data_ptr(),
                        workspace_bytes=self.ws.numel(), flags=self.flags.data_ptr())
        moves = self.model.compact()
        self.move(moves)
        self.same()
        return moves


@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (4, 5, 9, 3), (7, 8, 30, 16), (33, 6, 90, 1), (70, 20, 900, 8), (5, 40, 150, 7)])
def test_random_life(api, handle, shape):
    """Steps of a scheduler in random order, until long after the pool has run out for the first time."""
    N, M, P, S = shape
    rng = random.Random(sum(shape))
    m = Machine(api, handle, N, M, P, S, table_t=N == 7, refs_offset=N % 3)
    copies = moves = 0
    for step in range(30):
        live = [s for s in range(N) if m.model.lengths[s] > 0]
        empty = [s for s in range(N) if m.model.lengths[s] == 0]
        what = rng.choice(["extend", "extend", "extend", "fork", "free", "compact"])
        if what == "extend":
            most = rng.choice([1, 1, 3, 2 * S + 1])
            copies += len(m.extend([rng.choice([0, 1, most, rng.randint(0, most)]) for _ in range(N)], most))
        elif what == "fork" and live and empty:
            k = rng.randint(1, len(empty))
            m.fork([rng.choice(live) for _ in range(k)], rng.sample(empty, k))
        elif what == "free" and live:
            m.free(rng.sample(live, rng.randint(1, max(1, len(live) // 2))))
        elif what == "compact":
            moves += len(m.compact())
    assert m.flags.item() & ~(api.FLAG_POOL_EXHAUSTED | api.FLAG_BAD_LENGTH) == 0
    if N >= 7:
        assert moves > 0 and (copies > 0 or S == 1)        # pages of one token are never partly filled


def test_large_pool(api, handle):
    """More pages and sequences than one CTA covers in a step; the pool share is no multiple of anything."""
    N, M, P, S = 9001, 6, 30011, 4
    rng = random.Random(5)
    pool = torch.arange(P, dtype=torch.int32, device="cuda").view(P, 1).repeat(1, 4)
    m = Machine(api, handle, N, M, P, S, pools=[pool])
    m.extend([rng.randint(0, 15) for _ in range(N)], 15)
    live = [s for s in range(N) if m.model.lengths[s] > 0]
    m.free(rng.sample(live, len(live) // 2))
    empty = [s for s in range(N) if m.model.lengths[s] == 0]
    live = [s for s in range(N) if m.model.lengths[s] > 0]
    m.fork([rng.choice(live) for _ in range(2000)], rng.sample(empty, 2000))
    assert len(m.extend([1] * N, 1)) > 500
    assert len(m.compact()) > 1000
    m.extend([9] * N, 9)                       # does not fit: a prefix gets its pages
    assert m.flags.item() & api.FLAG_POOL_EXHAUSTED


def test_prompt_in_one_call(api, handle):
    """A prompt of thousands of tokens at once, an exactly full row, an exactly full pool."""
    m = Machine(api, handle, 3, 260, 530, 16)
    m.extend([4000, 4160, 0], 4160)
    m.extend([0, 0, 160], 160)
    assert m.flags.item() == 0 and m.model.refs.count(0) == 530 - 250 - 260 - 10
    m.extend([160, 0, 0], 160)
    assert m.model.refs.count(0) == 0 and m.flags.item() == 0
    m.extend([0, 0, 1], 1)
    assert m.flags.item() == api.FLAG_POOL_EXHAUSTED
    m.flags.zero_()
    m.extend([1, 1, 0], 1)
    assert m.flags.item() == api.FLAG_BAD_LENGTH


def test_copy_on_write_sharing(api, handle):
    """Two and three sharers of a partly filled page; a full last page is never copied."""
    m = Machine(api, handle, 6, 4, 24, 8)
    m.extend([11, 8, 0, 0, 0, 0], 11)
    m.fork([0, 0, 1], [2, 3, 4])
    assert len(m.extend([1, 1, 0, 1, 1, 0], 1)) == 2       # sequences 0 and 3 copy, 2 keeps the page, 1 and 4 open new ones
    assert len(m.extend([0, 0, 1, 0, 0, 0], 1)) == 0       # the last sharer is alone
    m.fork([2], [5])
    assert len(m.extend([0, 0, 1, 0, 0, 1], 1)) == 2       # both sides copy at once; the old page falls free
    m.compact()


def test_bad_input_is_reported_and_skipped(api, handle):
    m = Machine(api, handle, 4, 3, 10, 4)
    m.extend([5, 3, 0, 0], 5)
    m.fork([0, 9, 0, -1, 2], [1, 2, 7, 3, 2])              # 1 is not empty, 9, 7 and -1 do not exist, 2 -> 2
    assert m.flags.item() == api.FLAG_BAD_SEQUENCE
    m.flags.zero_()
    m.free([17, -3])
    assert m.flags.item() == api.FLAG_BAD_SEQUENCE
    m.flags.zero_()
    m.extend([-1, 1, 6, 0], 5)
    assert m.flags.item() == api.FLAG_BAD_LENGTH
    m.flags.zero_()
    m.table[0, 1] = 99                                     # the partly filled last page of sequence 0
    m.model.table[0][1] = 99
    m.extend([1, 1, 1, 0], 1)
    assert m.flags.item() == api.FLAG_BAD_PAGE
    m.flags.zero_()
    m.free([0, 0])                                         # twice in one list: once
    assert m.flags.item() == api.FLAG_BAD_PAGE


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.float64, torch.complex64, torch.complex128, torch.int32])
def test_copy_layouts(api, handle, dtype):
    """Contents of any type and layout; bytes outside the destination pages stay."""
    g = torch.Generator()
    g.manual_seed(3)
    P = 11

    def fill(*shape):
        x = torch.randint(-1000, 1000, shape, generator=g)
        return (torch.complex(x.double(), -2.0 * x.double()) if dtype.is_complex else x).to(dtype).cuda()

    wide = fill(P, 6, 4, 20)
    shifted = fill(P * 24 + 1)
    layouts = [
        fill(P, 16, 2, 64),                          # one block
        fill(P, 3, 5, 7),                            # odd block
        wide[:, 1:4, :, 3:16],                       # holes everywhere
        fill(2, P, 8, 8).transpose(0, 1),            # pages of two layers
        fill(4, 6, P).permute(2, 1, 0),              # the page is the fastest mode
        shifted[1:].view(P, 24),                     # off 16-byte alignment
        fill(P),                                     # a page of one element
        fill(5000, P, 9).transpose(0, 1),
    ]
    pairs = torch.tensor([[0, 5], [3, 1], [-1, 2], [4, -9], [10, 9], [0, 7]], dtype=torch.int32)
    bad = torch.tensor([[0, 11], [2 ** 31 - 1, 0]], dtype=torch.int32)
    table = api.TensorInfo(handle, api.I32, (1, 1))
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    for t in layouts:
        whole = t._base if t._base is not None else t
        before = whole.cpu().clone()
        want = t.cpu().clone()
        for a, b in pairs.tolist():
            if a >= 0 and b >= 0:
                want[b] = t[a].cpu()
        op = api.Pages(handle, info(api, handle, t), table, 1)
        cp = torch.cat((pairs, bad)).cuda()
        flags.zero_()
        op.copy(torch.cuda.current_stream().cuda_stream, cp.data_ptr(), len(cp), [t.data_ptr()], flags=flags.data_ptr())
        torch.cuda.synchronize()
        assert torch.equal(t.cpu(), want)
        assert flags.item() == api.FLAG_BAD_PAGE
        t[[5, 1, 9, 7]] = before.as_strided(t.shape, t.stride(), t.storage_offset())[[5, 1, 9, 7]].cuda()
        assert torch.equal(whole.cpu(), before)


def test_copy_many_tensors_of_several_layouts(api, handle):
    """Keys and values of different head sizes and types, more tensors than one launch takes."""
    P, layers = 5, 100
    g = torch.Generator()
    g.manual_seed(4)
    tensors, want = [], []
    for _ in range(layers):
        for t in (torch.randn(P, 4, 3, 16, generator=g).to(torch.bfloat16), torch.randn(P, 4, 3, 10, generator=g)[..., :7],
                  torch.randn(P, 2, generator=g).double()):
            want.append(t.clone())
            want[-1][3] = t[0]
            tensors.append(t.cuda() if t.is_contiguous() else torch.zeros(P, 4, 3, 10, device="cuda")[..., :7].copy_(t))
    op = api.Pages(handle, [info(api, handle, t) for t in tensors[:3]], api.TensorInfo(handle, api.I32, (1, 1)), 4)
    pairs = torch.tensor([[0, 3]], dtype=torch.int32, device="cuda")
    op.copy(torch.cuda.current_stream().cuda_stream, pairs.data_ptr(), 1, [t.data_ptr() for t in tensors])
    torch.cuda.synchronize()
    for t, w in zip(tensors, want):
        assert torch.equal(t.cpu(), w)


def test_copy_beyond_32_bits(api, handle):
    flat = torch.zeros(2 * 1_200_000_000 + 64, dtype=torch.bfloat16, device="cuda")
    t = torch.as_strided(flat, (3, 64), (1_200_000_000, 1))
    t[0] = torch.arange(64, device="cuda")
    op = api.Pages(handle, info(api, handle, t), api.TensorInfo(handle, api.I32, (1, 1)), 1)
    pairs = torch.tensor([[0, 2]], dtype=torch.int32, device="cuda")
    op.copy(torch.cuda.current_stream().cuda_stream, pairs.data_ptr(), 1, [t.data_ptr()])
    torch.cuda.synchronize()
    assert torch.equal(t[2].cpu(), torch.arange(64).to(torch.bfloat16)) and (t[1] == 0).all()


def test_state_without_tensors_and_graph(api, handle):
    """Only the state changes when no tensors are given; a captured extend serves step after step."""
    m = Machine(api, handle, 4, 8, 20, 4)
    m.extend([3, 5, 0, 2], 5, bare=True)
    m.fork([0], [2])
    m.extend([1, 0, 1, 0], 1, bare=True)
    new = torch.ones(4, dtype=torch.int32, device="cuda")
    slots = torch.empty(4, 1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.op.extend(torch.cuda.current_stream().cuda_stream, new.data_ptr(), *m.state(), slots.data_ptr(), 1, m.pointers(),
                    workspace=m.ws.data_ptr(), workspace_bytes=m.ws.numel())
    for _ in range(6):
        graph.replay()
        want, moves = m.model.extend([1] * 4, 1)
        m.move(moves)
        m.same()
        assert slots.tolist() == want
