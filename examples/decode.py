"""A decoder attention layer, token by token, made of the library's operations.

Each step takes one new token per sequence:

    Pages.extend         a place in the cache for the token (pages allocated, shared ones copied)
    Contraction          x[n,e] Wqkv[e,h,d] -> qkv[n,h,d]
    Rotary               norm and rotation of queries and keys; keys and values into their pages
    PagedAttention       one query token per sequence over its pages
    Contraction          o[n,h,d] Wo[h,d,e] -> y[n,e]

The host reads nothing back: a step is launches in stream order and is captured into a CUDA graph once.  On the way
sequences are forked, freed and the cache is compacted; at the end every output is compared with a plain
recomputation of the whole layer in 64 bits.

    python examples/decode.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07827_b200 import api  # noqa: E402

SEQUENCES, WIDTH, HEADS, KEY_HEADS, HEAD = 8, 256, 8, 2, 64
PAGE, POOL, COLUMNS = 16, 64, 16
EPS = 1e-6


class Layer:
    """Weights, cache, and the planned operations with their workspaces."""

    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
        self.wqkv = rand(WIDTH, HEADS + 2 * KEY_HEADS, HEAD) / WIDTH ** 0.5
        self.wo = rand(HEADS, HEAD, WIDTH) / (HEADS * HEAD) ** 0.5
        self.norm_q, self.norm_k = 1 + 0.1 * rand(HEAD), 1 + 0.1 * rand(HEAD)
        self.freq, self.mult = api.rotary_frequencies(HEAD, scaling="bands", factor=4.0, original_length=4096)

        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((SEQUENCES, COLUMNS), -1, **i32)
        self.lengths, self.refs = torch.zeros(SEQUENCES, **i32), torch.zeros(POOL, **i32)
        self.slots, self.positions = torch.empty(SEQUENCES, 1, **i32), torch.empty(SEQUENCES, **i32)
        self.new = torch.zeros(SEQUENCES, **i32)               # tokens each sequence takes in a step: 1 or 0
        self.keys = torch.zeros(POOL, PAGE, KEY_HEADS, HEAD, device="cuda")
        self.values = torch.zeros_like(self.keys)
        self.flags = torch.zeros(1, **i32)

        self.x = torch.zeros(SEQUENCES, WIDTH, device="cuda")
        self.qkv = torch.empty(SEQUENCES, HEADS + 2 * KEY_HEADS, HEAD, device="cuda")
        self.q = torch.empty(SEQUENCES, HEADS, HEAD, device="cuda")
        self.o, self.y = torch.empty_like(self.q), torch.empty_like(self.x)

        h = self.handle = api.Handle()
        info = lambda t: api.TensorInfo(h, api.dtype_code(t.dtype), t.shape, t.stride())  # noqa: E731
        parts = torch.split(self.qkv, [HEADS, KEY_HEADS, KEY_HEADS], 1)
        self.parts = parts
        self.project = api.Contraction(h, info(self.x), "ne", info(self.wqkv), "ehd", None, None, info(self.qkv), "nhd")
        self.back = api.Contraction(h, info(self.o), "nhd", info(self.wo), "hde", None, None, info(self.y), "ne")
        self.rotary = api.Rotary(h, self.freq, info(parts[0]), info(self.q), info(parts[1]), info(self.keys), info(parts[2]),
                                 info(self.values), norm=True, eps=EPS, multiplier=self.mult)
        self.attention = api.PagedAttention(h, info(self.q), info(self.keys), info(self.values), info(self.table), info(self.o))
        self.pages = api.Pages(h, info(self.keys), info(self.table), PAGE)
        self.work = {op: torch.empty(max(op.workspace_size(), 1), dtype=torch.uint8, device="cuda")
                     for op in (self.project, self.back, self.attention, self.pages)}

    def _ws(self, op):
        return dict(workspace=self.work[op].data_ptr(), workspace_bytes=self.work[op].numel())

    def _state(self):
        return self.table.data_ptr(), self.lengths.data_ptr(), self.refs.data_ptr()

    def step(self):
        """One token for every sequence with new == 1: reads x, writes y."""
        s, flags = torch.cuda.current_stream().cuda_stream, self.flags.data_ptr()
        cache = [self.keys.data_ptr(), self.values.data_ptr()]
        self.pages.extend(s, self.new.data_ptr(), *self._state(), self.slots.data_ptr(), 1, cache, flags=flags, **self._ws(self.pages))
        torch.sub(self.lengths, 1, out=self.positions)
        self.project.execute(s, self.x.data_ptr(), self.wqkv.data_ptr(), None, self.qkv.data_ptr(), **self._ws(self.project))
        q, k, v = (p.data_ptr() for p in self.parts)
        self.rotary.execute(s, self.positions.data_ptr(), self.norm_q.data_ptr(), self.norm_k.data_ptr(), q, self.q.data_ptr(),
                            k, cache[0], v, cache[1], slots=self.slots.data_ptr(), flags=flags)
        self.attention.execute(s, self.q.data_ptr(), *cache, self.table.data_ptr(), self.lengths.data_ptr(), self.o.data_ptr(),
                               flags=flags, **self._ws(self.attention))
        self.back.execute(s, self.o.data_ptr(), self.wo.data_ptr(), None, self.y.data_ptr(), **self._ws(self.back))

    def fork(self, src, dst):
        a, b = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst))
        self.pages.fork(torch.cuda.current_stream().cuda_stream, a.data_ptr(), b.data_ptr(), len(src), *self._state(), flags=self.flags.data_ptr())

    def free(self, sequences):
        a = torch.tensor(sequences, dtype=torch.int32, device="cuda")
        self.pages.free(torch.cuda.current_stream().cuda_stream, a.data_ptr(), len(sequences), *self._state(), flags=self.flags.data_ptr())

    def compact(self):
        self.pages.compact(torch.cuda.current_stream().cuda_stream, self.table.data_ptr(), self.refs.data_ptr(),
                           [self.keys.data_ptr(), self.values.data_ptr()], flags=self.flags.data_ptr(), **self._ws(self.pages))

    def plain(self, tokens):
        """The layer's output for the last of a sequence's tokens [t, WIDTH], in 64 bits."""
        qkv = torch.einsum("te,ehd->thd", tokens.double().cpu(), self.wqkv.double().cpu())
        q, k, v = torch.split(qkv, [HEADS, KEY_HEADS, KEY_HEADS], 1)
        angle = torch.arange(len(tokens)).double()[:, None, None] * torch.tensor(self.freq, dtype=torch.float64)

        def turned(x, w):
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double().cpu()
            z = torch.complex(x[..., :HEAD // 2], x[..., HEAD // 2:]) * torch.polar(torch.full_like(angle, self.mult), angle)
            return torch.cat((z.real, z.imag), -1)

        q, k = turned(q, self.norm_q)[-1], turned(k, self.norm_k).repeat_interleave(HEADS // KEY_HEADS, 1)
        p = torch.softmax(torch.einsum("hd,thd->ht", q, k) / HEAD ** 0.5, -1)
        o = torch.einsum("ht,thd->hd", p, v.repeat_interleave(HEADS // KEY_HEADS, 1))
        return torch.einsum("hd,hde->e", o, self.wo.double().cpu())


def main(steps=60):
    """Runs the layer for `steps` steps; returns the largest error relative to the largest output."""
    layer = Layer()
    layer.step()                                               # (no sequence is running: first use of every operation)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    g = torch.Generator().manual_seed(1)
    history = [[] for _ in range(SEQUENCES)]
    running = [0, 1, 2]
    worst = 0.0
    for t in range(steps):
        if t == 20:                                            # two more answers to the first two prompts
            layer.fork([0, 0, 1], [3, 4, 5])
            history[3], history[4], history[5] = list(history[0]), list(history[0]), list(history[1])
            running += [3, 4, 5]
        if t == 33:                                            # two answers end, a new request takes a free row
            layer.free([0, 2])
            history[0], history[2] = [], []
            running = [1, 3, 4, 5, 6]
        if t == 45:
            layer.compact()
        x = torch.randn(SEQUENCES, WIDTH, generator=g)
        layer.x.copy_(x)
        layer.new.copy_(torch.tensor([int(n in running) for n in range(SEQUENCES)], dtype=torch.int32))
        graph.replay()
        for n in running:
            history[n].append(x[n])
        if t % 7 == 0 or t in (20, 21, 33, 34, 45, 46, steps - 1):
            y = layer.y.double().cpu()
            for n in running:
                want = layer.plain(torch.stack(history[n]))
                worst = max(worst, float((y[n] - want).abs().max() / want.abs().max()))
    torch.cuda.synchronize()
    if layer.flags.item():
        raise RuntimeError(f"the device reported {layer.flags.item()}")
    if layer.lengths.tolist() != [len(h) for h in history]:
        raise RuntimeError("lengths differ from what was fed")
    return worst


if __name__ == "__main__":
    print("largest error relative to the largest output: %.2e" % main(int(sys.argv[1]) if len(sys.argv) > 1 else 60))
