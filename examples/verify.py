"""A decoder layer in 16 bits that verifies trees of drafted tokens, made of the library's operations alone.

Each step takes up to T drafted tokens per sequence, a tree of them:

    AddNorm           residual stream + the block before, root-mean-square norm, result in 8 bits with a scale per token
    Linear4           4-bit weights: queries, keys and values of all drafts
    Rotary            rotation by the drafts' positions (length + depth in the tree); keys and values into their pages
    TreeAttention     every draft sees the cached tokens, itself and what it continues
    Linear4           the output projection
    AddNorm, Linear4  the feed-forward block: norm in 8 bits, gated half (activation and product included)
    Linear4           its second half

The host reads nothing back inside a step: it is captured into a CUDA graph once.  When a path of the tree is accepted, its keys and
values are written once more, to the places behind the cached tokens in a row (Rotary, with the other drafts' slots negative).
At the end the outputs along accepted paths are compared with a plain recomputation of the layer that rounds where the layer stores.

    python examples/verify.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07827_b200 import api  # noqa: E402

SEQUENCES, DRAFTS, WIDTH, HEADS, KEY_HEADS, HEAD, INNER = 4, 12, 256, 8, 2, 64, 512
PAGE, CAPACITY, GROUP = 16, 160, 64
EPS = 1e-6
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
ROWS = HEADS + 2 * KEY_HEADS


class Weights:
    """Codes, scales and zeros of a matrix [rows, k], and the numbers they stand for."""

    def __init__(self, g, rows, k):
        self.rows, self.k = rows, k
        self.codes = torch.randint(0, 256, (rows, k // 2), generator=g, dtype=torch.uint8)
        self.scales = ((0.5 + torch.rand(rows, k // GROUP, generator=g)) / (4.6 * k ** 0.5)).to(BF16)
        self.zeros = torch.randint(6, 10, (rows, k // GROUP), generator=g, dtype=torch.uint8)
        code = torch.stack((self.codes & 15, self.codes >> 4), -1).view(rows, k).double()
        spread = lambda v: v.double().repeat_interleave(GROUP, 1)  # noqa: E731
        self.numbers = (code - spread(self.zeros)) * spread(self.scales)


class Layer:
    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.w_qkv, self.w_out = Weights(g, ROWS * HEAD, WIDTH), Weights(g, WIDTH, HEADS * HEAD)
        self.w_up, self.w_down = Weights(g, 2 * INNER, WIDTH), Weights(g, WIDTH, INNER)
        self.norm_1, self.norm_2 = ((1 + 0.2 * torch.randn(WIDTH, generator=g)).to(BF16).cuda() for _ in range(2))
        self.freq, self.mult = api.rotary_frequencies(HEAD)

        n, t = SEQUENCES, SEQUENCES * DRAFTS
        i32 = dict(dtype=torch.int32, device="cuda")
        wide = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.lengths, self.positions, self.slots = torch.zeros(n, **i32), torch.zeros(t, **i32), torch.full((t,), -1, **i32)
        self.masks = torch.zeros(n, DRAFTS, 1, **i32)
        self.flags = torch.zeros(1, **i32)
        # the cache: all pages a sequence may need are taken at the start, and with them the slot of every position
        columns = CAPACITY // PAGE
        self.table, held, refs = torch.full((n, columns), -1, **i32), torch.zeros(n, **i32), torch.zeros(n * columns, **i32)
        self.keys = wide(n * columns, PAGE, KEY_HEADS, HEAD)
        self.values = torch.zeros_like(self.keys)
        self.places = torch.empty(n, CAPACITY, **i32)
        # activations: what comes in (the block before and the residual stream), and every stored result
        self.x, self.stream = wide(t, WIDTH), wide(t, WIDTH)
        self.h1, self.h2 = wide(t, WIDTH), wide(t, WIDTH)
        self.n1, self.n2 = wide(t, WIDTH, dtype=E4M3), wide(t, WIDTH, dtype=E4M3)
        self.s1, self.s2 = wide(t, 1, dtype=torch.float32), wide(t, 1, dtype=torch.float32)
        self.qkv, self.q = wide(t, ROWS, HEAD), wide(t, HEADS, HEAD)
        self.o, self.a = wide(t, HEADS, HEAD), wide(t, WIDTH)
        self.f, self.y = wide(t, INNER), wide(t, WIDTH)

        h = self.handle = api.Handle()
        info = lambda x: api.TensorInfo(h, api.dtype_code(x.dtype), x.shape, x.stride())  # noqa: E731
        flat = lambda x: x.view(t, -1)  # noqa: E731
        weights = dict(scale_type=api.BF16, group=GROUP, zeros=True)
        self.add_1 = api.AddNorm(h, info(self.x), info(self.n1), R=info(self.stream), H=info(self.h1), S=info(self.s1), eps=EPS)
        self.add_2 = api.AddNorm(h, info(self.a), info(self.n2), R=info(self.h1), H=info(self.h2), S=info(self.s2), eps=EPS)
        self.project = api.Linear4(h, info(self.n1), info(flat(self.qkv)), XS=info(self.s1), **weights)
        self.out = api.Linear4(h, info(flat(self.o)), info(self.a), **weights)
        self.up = api.Linear4(h, info(self.n2), info(self.f), XS=info(self.s2), activation="silu", **weights)
        self.down = api.Linear4(h, info(self.f), info(self.y), **weights)
        self.parts = torch.split(self.qkv, [HEADS, KEY_HEADS, KEY_HEADS], 1)
        self.rotary = api.Rotary(h, self.freq, info(self.parts[0]), info(self.q), info(self.parts[1]), info(self.keys), info(self.parts[2]),
                                 info(self.values), multiplier=self.mult)
        tree = lambda x: x.view(n, DRAFTS, HEADS, HEAD)  # noqa: E731
        self.attention = api.TreeAttention(h, info(tree(self.q)), info(self.keys), info(self.values), info(self.table), info(self.masks), info(tree(self.o)))
        self.pages = api.Pages(h, info(self.keys), info(self.table), PAGE)
        self.work = {op: torch.empty(max(op.workspace_size(), 1), dtype=torch.uint8, device="cuda")
                     for op in (self.project, self.out, self.up, self.down, self.attention, self.pages)}

        now = torch.cuda.current_stream().cuda_stream
        self.packed = {}
        for op, w in ((self.project, self.w_qkv), (self.out, self.w_out), (self.up, self.w_up), (self.down, self.w_down)):
            self.packed[op] = torch.empty(op.packed_size(), dtype=torch.uint8, device="cuda")
            c, s, z = w.codes.cuda(), w.scales.cuda(), w.zeros.cuda()
            op.pack(now, c.data_ptr(), s.data_ptr(), z.data_ptr(), self.packed[op].data_ptr())
            torch.cuda.synchronize()
        every = torch.full((n,), CAPACITY, **i32)
        self.pages.extend(now, every.data_ptr(), self.table.data_ptr(), held.data_ptr(), refs.data_ptr(),
                          self.places.data_ptr(), CAPACITY, [self.keys.data_ptr(), self.values.data_ptr()], flags=self.flags.data_ptr(), **self._ws(self.pages))
        torch.cuda.synchronize()

    def _ws(self, op):
        return dict(workspace=self.work[op].data_ptr(), workspace_bytes=self.work[op].numel())

    def _linear(self, op, s, x, y, xs=None):
        op.execute(s, self.packed[op].data_ptr(), x.data_ptr(), y.data_ptr(), XS=xs.data_ptr() if xs is not None else 0, **self._ws(op))

    def place(self, s):
        """Queries rotated, keys and values of the drafts with a slot into the cache."""
        q, k, v = (p.data_ptr() for p in self.parts)
        self.rotary.execute(s, self.positions.data_ptr(), 0, 0, q, self.q.data_ptr(), k, self.keys.data_ptr(), v, self.values.data_ptr(),
                            slots=self.slots.data_ptr(), flags=self.flags.data_ptr())

    def step(self):
        """One pass: reads x, stream, masks, lengths, positions, slots; writes h2 + y (the stream and the block for the next layer)."""
        s = torch.cuda.current_stream().cuda_stream
        self.add_1.execute(s, self.x.data_ptr(), self.norm_1.data_ptr(), self.n1.data_ptr(), R=self.stream.data_ptr(), H=self.h1.data_ptr(), S=self.s1.data_ptr())
        self._linear(self.project, s, self.n1, self.qkv, self.s1)
        self.place(s)
        self.attention.execute(s, self.q.data_ptr(), self.keys.data_ptr(), self.values.data_ptr(), self.table.data_ptr(), self.lengths.data_ptr(),
                               self.masks.data_ptr(), self.o.data_ptr(), flags=self.flags.data_ptr(), **self._ws(self.attention))
        self._linear(self.out, s, self.o, self.a)
        self.add_2.execute(s, self.a.data_ptr(), self.norm_2.data_ptr(), self.n2.data_ptr(), R=self.h1.data_ptr(), H=self.h2.data_ptr(), S=self.s2.data_ptr())
        self._linear(self.up, s, self.n2, self.f, self.s2)
        self._linear(self.down, s, self.f, self.y)

    def plain(self, x, stream):
        """(h2, y) of a sequence's tokens [t, WIDTH], in 64 bits, rounded where the layer stores."""
        kept = lambda v: v.to(torch.float32).to(BF16).double()  # noqa: E731

        def norm(h, w):
            y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS) * w.double().cpu()
            s = (y.abs().amax(-1, keepdim=True) / 448).clamp(min=2.0 ** -126)
            return (y / s).float().to(E4M3).double() * s

        h1 = x.double() + stream.double()
        qkv = kept(norm(h1, self.norm_1) @ self.w_qkv.numbers.T).view(-1, ROWS, HEAD)
        q, k, v = torch.split(qkv, [HEADS, KEY_HEADS, KEY_HEADS], 1)
        angle = torch.arange(len(x)).double()[:, None, None] * torch.tensor(self.freq, dtype=torch.float64)

        def turned(z):
            z = torch.complex(z[..., :HEAD // 2], z[..., HEAD // 2:]) * torch.polar(torch.full_like(angle, self.mult), angle)
            return kept(torch.cat((z.real, z.imag), -1))

        q, k = turned(q), turned(k).repeat_interleave(HEADS // KEY_HEADS, 1)
        p = torch.einsum("ihd,jhd->hij", q, k) / HEAD ** 0.5
        p = torch.softmax(p.masked_fill(~torch.ones(len(x), len(x), dtype=torch.bool).tril(), -torch.inf), -1)
        o = kept(torch.einsum("hij,jhd->ihd", p, v.repeat_interleave(HEADS // KEY_HEADS, 1)))
        a = kept(o.reshape(len(x), -1) @ self.w_out.numbers.T)
        h2 = a + kept(h1)
        z = norm(h2, self.norm_2) @ self.w_up.numbers.T
        f = kept(z[:, :INNER] * torch.sigmoid(z[:, :INNER]) * z[:, INNER:])
        return h2, kept(f @ self.w_down.numbers.T)


def main(steps=8):
    """Runs the layer for `steps` steps; returns the largest error relative to the largest output."""
    layer = Layer()
    layer.step()                                               # (every mask is empty: first use of every operation)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    g = torch.Generator().manual_seed(1)
    history = [([], []) for _ in range(SEQUENCES)]             # accepted tokens' inputs of each sequence
    worst = 0.0
    places = layer.places.cpu()
    for step in range(steps):
        # a tree per sequence: each draft continues an earlier one or the last accepted token; a few rows hold none
        parents = []
        for n in range(SEQUENCES):
            used = DRAFTS - (3 * n + step) % 5
            parents.append([int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(used)] + [-2] * (DRAFTS - used))
        masks, depth = zip(*(api.tree_masks(p) for p in parents))
        lengths = torch.tensor([len(h[0]) for h in history], dtype=torch.int32)
        depth = torch.tensor(depth)
        slots = torch.where(depth >= 0, places[torch.arange(SEQUENCES)[:, None], lengths[:, None].long() + torch.arange(DRAFTS)], -1)
        x, stream = (torch.randn(SEQUENCES * DRAFTS, WIDTH, generator=g).to(BF16) for _ in range(2))
        layer.x.copy_(x)
        layer.stream.copy_(stream)
        layer.masks.copy_(torch.tensor(masks, dtype=torch.int32))
        layer.lengths.copy_(lengths)
        layer.positions.copy_((lengths[:, None] + depth.clamp(min=0)).view(-1))
        layer.slots.copy_(slots.view(-1))
        graph.replay()
        # one path is accepted: its keys and values go where the sequence continues
        accepted = torch.full((SEQUENCES, DRAFTS), -1, dtype=torch.int32)
        h2, y = layer.h2.double().cpu().view(SEQUENCES, DRAFTS, -1), layer.y.double().cpu().view(SEQUENCES, DRAFTS, -1)
        for n in range(SEQUENCES):
            i, path = int(torch.randint(0, sum(p >= -1 for p in parents[n]), (1,), generator=g)), []
            while i >= 0:
                path.insert(0, i)
                i = parents[n][i]
            for d, i in enumerate(path):
                accepted[n, i] = places[n, int(lengths[n]) + d]
                history[n][0].append(x[n * DRAFTS + i])
                history[n][1].append(stream[n * DRAFTS + i])
            want = layer.plain(torch.stack(history[n][0]), torch.stack(history[n][1]))
            for got, exact in ((h2, want[0]), (y, want[1])):
                worst = max(worst, float((got[n, path] - exact[-len(path):]).abs().max() / exact.abs().max()))
        layer.slots.copy_(accepted.view(-1))
        layer.place(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    if layer.flags.item():
        raise RuntimeError(f"the device reported {layer.flags.item()}")
    return worst


if __name__ == "__main__":
    print("largest error relative to the largest output: %.2e" % main(int(sys.argv[1]) if len(sys.argv) > 1 else 8))
