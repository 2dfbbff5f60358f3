"""Plain 64-bit implementations of the decoder operators (loops and numpy / torch double, on the CPU) and the
error bounds that the tests hold the kernels to.

Bounds.  u is the unit roundoff of the storage type (2^-8 bf16, 2^-11 f16, 2^-24 fp32) and e = 2^-24.  A value computed in fp32 through a chain of n roundings and rounded once to its type is
off by at most u |y| + n e S, with S the sum of the moduli of the terms; n is stated where it is used.
"""
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# f16 subnormals: half the spacing below 2^-14
FLOOR = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
E32 = 2.0 ** -24


def rotary_forward(x, w, pos, freq, mult, interleaved, norm, eps):
    """x [T, H, D] in its storage type; returns float64 [T, H, D]."""
    x = x.double()
    if norm:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w.double()
    pairs = len(freq)
    if pairs == 0:
        return x
    angle = pos.double()[:, None, None] * torch.tensor(freq, dtype=torch.float64)
    c, s = torch.cos(angle) * mult, torch.sin(angle) * mult
    i = torch.arange(pairs)
    a_at, b_at = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    a, b = x[..., a_at], x[..., b_at]
    y = x.clone()
    y[..., a_at] = a * c - b * s
    y[..., b_at] = b * c + a * s
    return y


def rotary_backward(x, w, pos, freq, mult, interleaved, norm, eps, dy):
    """Formula of the gradients (float64): dx, dw."""
    dm = rotary_forward(dy, None, pos, [-f for f in freq], mult, interleaved, False, eps)
    if not norm:
        return dm, None
    xd = x.double()
    r = 1.0 / torch.sqrt((xd * xd).mean(-1, keepdim=True) + eps)
    n = xd * r
    g = dm * w.double() if w is not None else dm
    return r * (g - n * (g * n).mean(-1, keepdim=True)), (dm * n).sum((0, 1))


def attention(q, k, v, table, lengths, scale, window, pages_ok=None):
    """q [N, Hq, D], k / v [P, S, Hk, *], lengths as given; returns float64 o [N, Hq, Dv], lse [N, Hq], and per
    (sequence, head) the scale of the error bound: sum p|v| [N, Hq, Dv], max_j scale sum_d |q k|, max |s|, tokens."""
    N, Hq, D = q.shape
    P, S, Hk, _ = k.shape
    Dv = v.shape[-1]
    group = Hq // Hk
    o = torch.zeros(N, Hq, Dv, dtype=torch.float64)
    lse = torch.full((N, Hq), float("-inf"), dtype=torch.float64)
    size = torch.zeros(N, Hq, Dv, dtype=torch.float64)
    moduli, top, count = torch.zeros(N, Hq), torch.zeros(N, Hq), torch.zeros(N, Hq)
    for n in range(N):
        length = max(0, min(int(lengths[n]), table.shape[1] * S))
        low = max(0, length - window) if window else 0
        tokens = [(int(table[n, j // S]), j % S) for j in range(low, length)]
        tokens = [(p, r) for p, r in tokens if 0 <= p < P]
        if not tokens:
            continue
        pg, rw = torch.tensor([t[0] for t in tokens]), torch.tensor([t[1] for t in tokens])
        for h in range(Hq):
            kk, vv, qq = k[pg, rw, h // group].double(), v[pg, rw, h // group].double(), q[n, h].double()
            s = kk @ qq * scale
            p = torch.softmax(s, 0)
            o[n, h], lse[n, h] = p @ vv, torch.logsumexp(s, 0)
            size[n, h] = p @ vv.abs()
            moduli[n, h] = (kk.abs() @ qq.abs()).max() * abs(scale)
            top[n, h], count[n, h] = s.abs().max(), len(tokens)
    return o, lse, size, moduli, top, count


def attention_bounds(o, lse, size, moduli, top, count, dim, dtype):
    """Largest errors allowed (see test_gpu_paged_attention.py)."""
    split = {torch.float32: 2.0 ** -20, torch.float16: 2.0 ** -20, torch.bfloat16: 2.0 ** -15}[dtype]
    score = (2 * dim + 8) * E32 * moduli + 4 * E32 * top + 8 * E32
    if dtype == torch.float32:
        score = score + 2.0 ** -20 * moduli
    chain = 4 * (count / 16 + 64) * E32
    rel = 2 * score + split + chain
    return (UNIT[dtype] * o.abs() + rel[..., None].double() * size + FLOOR[dtype] + 1e-300,
            score.double() + 4 * E32 * lse.abs().nan_to_num(0, 0, 0) + chain.double())


class PagesState:
    """The bookkeeping of cache pages, one step at a time (plain Python)."""

    def __init__(self, table, lengths, refs, page_tokens):
        self.table = [list(map(int, r)) for r in table]
        self.lengths, self.refs, self.S = list(map(int, lengths)), list(map(int, refs)), page_tokens
        self.columns, self.P = len(self.table[0]), len(self.refs)

    def free(self, sequences):
        for s in sequences:
            if not 0 <= s < len(self.table):
                continue
            for j, p in enumerate(self.table[s]):
                if 0 <= p < self.P:
                    self.refs[p] -= 1
                self.table[s][j] = -1
            self.lengths[s] = 0

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            if not (0 <= a < len(self.table) and 0 <= b < len(self.table)) or a == b or self.lengths[b] != 0:
                continue
            self.table[b], self.lengths[b] = list(self.table[a]), self.lengths[a]
            for p in self.table[a]:
                if p >= 0:
                    self.refs[p] += 1

    def extend(self, new, most):
        """Returns (slots, copies)."""
        S, room = self.S, self.columns * self.S
        empty = [p for p in range(self.P) if self.refs[p] == 0]
        refs_before = list(self.refs)
        slots, copies, at, stopped = [], [], 0, False
        for s, add in enumerate(new):
            length = self.lengths[s]
            row = [-1] * most
            slots.append(row)
            if add <= 0 or length < 0 or add > most or length + add > room:
                continue
            held = -(-length // S)
            partial = length % S != 0
            last = self.table[s][held - 1] if partial else -1
            if partial and not 0 <= last < self.P:
                continue
            copy = partial and refs_before[last] > 1
            need = -(-(length + add) // S) - held + int(copy)
            if stopped or at + need > len(empty):
                stopped = True
                continue
            if copy:
                fresh = empty[at]
                at += 1
                copies.append((last, fresh))
                self.refs[last] -= 1
                self.refs[fresh] = 1
                self.table[s][held - 1] = fresh
            for j in range(held, -(-(length + add) // S)):
                self.table[s][j] = empty[at]
                self.refs[empty[at]] = 1
                at += 1
            for i in range(add):
                t = length + i
                row[i] = self.table[s][t // S] * S + t % S
            self.lengths[s] = length + add
        return slots, copies

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] <= 0]
        late = [p for p in range(live, self.P) if self.refs[p] > 0]
        to = dict(zip(late, holes))
        for row in self.table:
            for j, p in enumerate(row):
                row[j] = to.get(p, p)
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        return list(to.items())
