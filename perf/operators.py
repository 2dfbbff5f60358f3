"""The decoder operators on real work: what a serving step and a training step ask of them.

Four kinds of case:

  attention  one new token per sequence over a paged key-value cache
  append     head norm and rotary positions of a step's queries and keys, keys and values written into
             their cache pages in the same pass (serving: decode steps and prefill)
  train      head norm and rotary positions of queries and keys with the backward pass (inputs' and
             norm weights' gradients)
  pages      the cache's pages: a scheduler step (free, fork, extend with copy on write) or a compaction

`own = False` computes a case with elementary torch operations in 32 bits, rounded once at the end;
`own = True` makes the calls a user makes of the library.  `exact` is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
_handle = None


def _library():
    """The binding and one handle for the process, as a program keeps them."""
    global _handle
    from paper_2601_07827_b200 import api
    if _handle is None:
        _handle = api.Handle()
    return api, _handle


def _info(api, handle, t):
    return api.TensorInfo(handle, api.dtype_code(t.dtype), t.shape, t.stride())


# ---- the cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # one user waiting for the next token: nothing but latency
        dict(name="attention one request", kind="attention", n=1, hq=32, hk=8, d=128, dv=128, page=16, shortest=1500,
             longest=1500, empty=0, window=0, heads_first=False, dtype="bf16"),
        # a server's ordinary decode step: requests of very different ages, one slot idle
        dict(name="attention batch", kind="attention", n=64, hq=32, hk=8, d=128, dv=128, page=16, shortest=64,
             longest=8192, empty=1, window=0, heads_first=False, dtype="bf16"),
        # a few users with whole books in their contexts: 4.3 GB of cache in one pass
        dict(name="attention long", kind="attention", n=8, hq=64, hk=8, d=128, dv=128, page=64, shortest=131072,
             longest=131072, empty=0, window=0, heads_first=True, dtype="f16"),
        # a small 32-bit model with a sliding window, odd group, head and page sizes
        dict(name="attention window f32", kind="attention", n=24, hq=20, hk=4, d=80, dv=72, page=24, shortest=10,
             longest=4100, empty=1, window=1000, heads_first=False, dtype="f32"),
        # decode step of 128 requests: one token each, every token into a page of its own
        dict(name="append decode", kind="append", t=128, hq=32, hk=8, d=128, rot=128, interleaved=False, norm=True,
             page=16, run=1, scaling="none", dtype="bf16"),
        # prefill of 16 ki prompt tokens, half of each head rotated, context stretched by bands
        dict(name="append prefill", kind="append", t=16384, hq=64, hk=8, d=128, rot=64, interleaved=True, norm=False,
             page=64, run=4096, scaling="bands", dtype="f16"),
        # one training step's layer: 16 ki tokens, 40 heads, forward and backward
        dict(name="train large", kind="train", t=16384, hq=32, hk=8, d=128, rot=128, interleaved=False, norm=True,
             scaling="none", dtype="bf16"),
        # a small 32-bit model with odd sizes
        dict(name="train odd f32", kind="train", t=777, hq=6, hk=2, d=80, rot=36, interleaved=True, norm=True,
             scaling="linear", dtype="f32"),
        # a scheduler's turn between two decode steps: 8 requests end, 8 answers fork, all take one token
        dict(name="pages step", kind="pages", do="step", n=64, page=16, pool=4096, longest=900, frees=8, forks=8,
             new=1, tensors=8, hk=8, d=64, dtype="bf16"),
        # the same for a large fleet with a big pool and several tokens a turn (speculation)
        dict(name="pages step fleet", kind="pages", do="step", n=1000, page=16, pool=200000, longest=5000, frees=60,
             forks=50, new=5, tensors=2, hk=1, d=64, dtype="bf16"),
        # a half-full pool is squeezed together before part of it is given back
        dict(name="pages compact", kind="pages", do="compact", n=128, page=32, pool=16384, longest=4096, frees=0,
             forks=0, new=1, tensors=2, hk=8, d=128, dtype="bf16"),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def _draw_attention(rng):
    hk = rng.choice([1, 2, 3, 4, 5, 8])
    d = rng.choice([32, 64, 72, 80, 96, 128, 128, 160, 192, 256])
    dv = rng.choice([d, d, d, max(32, d - 64)])
    longest = _spread(rng, 1, 131072)
    # the padded cache of a drawn case is at most a quarter of the largest listed one's
    n = _spread(rng, 1, max(1, min(300, 268435456 // (longest * hk * max(d, dv)))))
    window = rng.choice([0, 0, 0, _spread(rng, 1, max(1, longest))])
    return dict(kind="attention", n=n, hq=hk * rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]), hk=hk, d=d, dv=dv,
                page=rng.choice([8, 16, 16, 24, 32, 64, 128]), shortest=_spread(rng, 1, longest), longest=longest,
                empty=rng.choice([0, 0, 1]) if n > 1 else 0, window=window, heads_first=rng.random() < 0.5,
                dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))


def _draw_heads(rng, most):
    hk = rng.choice([1, 2, 4, 5, 8])
    hq = hk * rng.choice([1, 2, 3, 4, 7, 8])
    d = rng.choice([32, 64, 72, 80, 96, 128, 128, 160, 256])
    t = _spread(rng, 1, max(1, min(20000, most // ((hq + 2 * hk) * d))))
    return dict(t=t, hq=hq, hk=hk, d=d, rot=rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)]),
                interleaved=rng.random() < 0.5, norm=rng.random() < 0.7,
                scaling=rng.choice(["none", "linear", "bands"]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))


def draw(rng):
    kind = rng.choice(["attention", "attention", "append", "train", "pages"])
    if kind == "attention":
        return _draw_attention(rng)
    if kind == "append":
        return dict(kind="append", **_draw_heads(rng, 16384 * 80 * 128), page=rng.choice([8, 16, 24, 64]),
                    run=rng.choice([1, 1, _spread(rng, 2, 5000)]))
    if kind == "train":
        c = dict(kind="train", **_draw_heads(rng, 16384 * 48 * 128))
        return c
    do = rng.choice(["step", "compact"])
    n = _spread(rng, 4, 1000)
    page = rng.choice([8, 16, 24, 64])
    longest = _spread(rng, page, 6000)
    hk, d = rng.choice([1, 2, 3, 8]), rng.choice([64, 72, 128])
    dtype = rng.choice(["bf16", "f16", "f32"])
    held = sum(-(-x // page) for x in _lengths(n, 1, longest, 0)) + 2 * n
    pool = int(held * rng.uniform(1.1, 2.5)) + 8
    # at most 1 GB a tensor
    while pool * page * hk * d * BYTES[dtype] > (1 << 30):
        n, longest = max(4, n // 2), max(page, longest // 2)
        held = sum(-(-x // page) for x in _lengths(n, 1, longest, 0)) + 2 * n
        pool = int(held * rng.uniform(1.1, 2.5)) + 8
    frees = rng.randint(0, n // 4) if do == "step" else 0
    return dict(kind="pages", do=do, n=n, page=page, pool=pool, longest=longest, frees=frees,
                forks=rng.randint(0, frees), new=rng.choice([1, 1, 3, 8]), tensors=rng.choice([1, 2, 4]), hk=hk, d=d,
                dtype=dtype)


def _lengths(n, shortest, longest, empty):
    """n lengths, even over their logarithm from shortest to longest, the first `empty` of them zero."""
    f = [shortest * (longest / shortest) ** ((i + 0.5) / n) for i in range(n)]
    return [0 if i < empty else max(1, min(longest, int(round(x)))) for i, x in enumerate(f)]


def _frequencies(rot, scaling):
    """Radians per position of each rotated pair, and the multiplier: base 10000, or stretched eightfold for
    long contexts: all pairs alike (linear), or by bands of wavelength (fast pairs as they are, slow ones
    stretched, a ramp between) with attention sharpened."""
    freq = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [f / 8.0 for f in freq], 1.0
    if scaling == "bands":
        out = []
        for f in freq:
            turns = 8192 * f / (2 * math.pi)           # turns within the context trained on
            keep = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
            out.append(f * keep + f / 8.0 * (1.0 - keep))
        return out, 0.1 * math.log(8.0) + 1.0
    return freq, 1.0


# ---- inputs -------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(TYPES[dtype])


def _pool(g, pages, page, heads, d, dtype, heads_first=False):
    """Cache pages [pages, page, heads, d]; heads_first: laid out head by head inside a page."""
    if heads_first:
        return _normal(g, (pages, heads, page, d), dtype).transpose(1, 2)
    return _normal(g, (pages, page, heads, d), dtype)


def _tables(g, lengths, page, pool, columns):
    """Page tables of the sequences: pages drawn at random from the pool, -1 beyond the length."""
    held = (lengths + page - 1) // page
    taken = torch.arange(columns, device="cuda")[None, :] < held[:, None]
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    rank = (torch.cumsum(taken.reshape(-1), 0) - 1).clamp(min=0)
    return torch.where(taken, order[rank].reshape(taken.shape), -1).to(torch.int32)


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case, "seed": seed}
    {"attention": _prepare_attention, "append": _prepare_append, "train": _prepare_train, "pages": _prepare_pages}[case["kind"]](case, g, s)
    if own:
        _plan(case, s)
    return s


def _prepare_attention(c, g, s):
    lens = torch.tensor(_lengths(c["n"], c["shortest"], c["longest"], c["empty"]), device="cuda", dtype=torch.int64)
    lens = lens[torch.randperm(c["n"], generator=g, device="cuda")]
    columns = -(-c["longest"] // c["page"])
    total = sum(-(-x // c["page"]) for x in _lengths(c["n"], c["shortest"], c["longest"], c["empty"]))
    pool = total + total // 16 + 2
    s["columns"] = columns
    s["table"] = _tables(g, lens, c["page"], pool, columns)
    s["lengths"] = lens.to(torch.int32)
    s["q"] = _normal(g, (c["n"], c["hq"], c["d"]), c["dtype"], 1.5)
    s["k"] = _pool(g, pool, c["page"], c["hk"], c["d"], c["dtype"], c["heads_first"])
    s["v"] = _pool(g, pool, c["page"], c["hk"], c["dv"], c["dtype"], c["heads_first"])
    s["o"] = torch.empty((c["n"], c["hq"], c["dv"]), dtype=TYPES[c["dtype"]], device="cuda")
    s["lse"] = torch.empty((c["n"], c["hq"]), dtype=torch.float32, device="cuda")


def _prepare_heads(c, g, s, kinds):
    """A projection's packed output [tokens, all heads, d] and its parts, norm weights, positions."""
    t, hq, hk, d = c["t"], c["hq"], c["hk"], c["d"]
    packed = _normal(g, (t, hq + (kinds - 1) * hk, d), c["dtype"])
    s["packed"] = packed
    s["xq"], s["xk"] = packed[:, :hq], packed[:, hq:hq + hk]
    if kinds == 3:
        s["xv"] = packed[:, hq + hk:]
    s["wq"] = _normal(g, (d,), c["dtype"], 0.1).add_(1.0)
    s["wk"] = _normal(g, (d,), c["dtype"], 0.1).add_(1.0)
    s["freq"], s["mult"] = _frequencies(c["rot"], c["scaling"])
    # turns per position; the product with a position keeps its fraction in 64 bits (32 bits would lose
    # the angle itself at long positions), everything after it is in 32 bits
    s["turns"] = torch.tensor(s["freq"], dtype=torch.float64, device="cuda") / (2 * math.pi)


def _prepare_append(c, g, s):
    _prepare_heads(c, g, s, 3)
    t, page, run = c["t"], c["page"], c["run"]
    # runs of consecutive tokens: each run is one sequence's, in pages of its own, at a position of its own
    runs = -(-t // run)
    per = -(-run // page)
    pool = runs * per + runs * per // 16 + 2
    start = torch.randint(0, 100000, (runs,), generator=g, device="cuda")
    token = torch.arange(t, device="cuda")
    which, at = token // run, token % run
    s["pos"] = (start[which] + at).to(torch.int32)
    pages = torch.randperm(pool, generator=g, device="cuda")[:runs * per].reshape(runs, per)
    s["slots"] = (pages[which, at // page] * page + at % page).to(torch.int32)
    s["kpool"] = _pool(g, pool, page, c["hk"], c["d"], c["dtype"])
    s["vpool"] = _pool(g, pool, page, c["hk"], c["d"], c["dtype"])
    s["yq"] = torch.empty((t, c["hq"], c["d"]), dtype=TYPES[c["dtype"]], device="cuda")


def _prepare_train(c, g, s):
    _prepare_heads(c, g, s, 2)
    t, hq, hk, d = c["t"], c["hq"], c["hk"], c["d"]
    s["pos"] = ((torch.arange(t, device="cuda") + torch.randint(0, 4000, (1,), generator=g, device="cuda")) % 8192).to(torch.int32)
    s["dyq"], s["dyk"] = _normal(g, (t, hq, d), c["dtype"]), _normal(g, (t, hk, d), c["dtype"])
    like = dict(dtype=TYPES[c["dtype"]], device="cuda")
    s["yq"], s["yk"] = torch.empty((t, hq, d), **like), torch.empty((t, hk, d), **like)
    s["dpacked"] = torch.empty((t, hq + hk, d), **like)
    s["dxq"], s["dxk"] = s["dpacked"][:, :hq], s["dpacked"][:, hq:]
    s["dwq"], s["dwk"] = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")


def _prepare_pages(c, g, s):
    n, page, pool = c["n"], c["page"], c["pool"]
    lens = torch.tensor(_lengths(n, 1, c["longest"], 0), device="cuda", dtype=torch.int64)
    lens = lens[torch.randperm(n, generator=g, device="cuda")]
    columns = -(-(c["longest"] + c["new"]) // page)
    table = _tables(g, lens, page, pool, columns)
    refs = torch.zeros(pool, dtype=torch.int32, device="cuda")
    refs.index_add_(0, table.clamp(min=0).reshape(-1), (table >= 0).to(torch.int32).reshape(-1))
    # the state is one buffer so that a pass can begin from the same state again with one copy
    s["before"] = torch.cat([table.reshape(-1), lens.to(torch.int32), refs])
    s["state"] = s["before"].clone()
    a, b = n * columns, n * columns + n
    s["table"], s["lengths"], s["refs"] = s["state"][:a].view(n, columns), s["state"][a:b], s["state"][b:]
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    s["frees"], s["dst"] = order[:c["frees"]].contiguous(), order[:c["forks"]].contiguous()
    s["src"] = order[c["frees"]:c["frees"] + c["forks"]].contiguous()
    s["new"] = torch.full((n,), c["new"], dtype=torch.int32, device="cuda")
    s["slots"] = torch.empty((n, c["new"]), dtype=torch.int32, device="cuda")
    s["pools"] = [_pool(g, pool, page, c["hk"], c["d"], c["dtype"]) for _ in range(c["tensors"])]


def _plan(c, s):
    """The library's operation objects and workspaces: made once, kept by the program."""
    api, h = _library()
    info = lambda t: _info(api, h, t)  # noqa: E731
    s["stream"] = torch.cuda.current_stream().cuda_stream
    if c["kind"] == "attention":
        op = api.PagedAttention(h, info(s["q"]), info(s["k"]), info(s["v"]), info(s["table"]), info(s["o"]),
                                scale=1.0 / math.sqrt(c["d"]), window=c["window"])
    elif c["kind"] == "append":
        op = api.Rotary(h, s["freq"], info(s["xq"]), info(s["yq"]), info(s["xk"]), info(s["kpool"]), info(s["xv"]),
                        info(s["vpool"]), interleaved=c["interleaved"], norm=c["norm"], eps=EPS, multiplier=s["mult"])
    elif c["kind"] == "train":
        op = api.Rotary(h, s["freq"], info(s["xq"]), info(s["yq"]), info(s["xk"]), info(s["yk"]),
                        interleaved=c["interleaved"], norm=c["norm"], eps=EPS, multiplier=s["mult"])
    else:
        op = api.Pages(h, info(s["pools"][0]), info(s["table"]), c["page"])
    s["op"] = op
    s["bytes"] = op.workspace_size()
    s["workspace"] = torch.empty(max(s["bytes"], 1), dtype=torch.uint8, device="cuda")


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    return {"attention": _attention, "append": _append, "train": _train, "pages": _pages}[state["case"]["kind"]](state["case"], state)


def _attention(c, s):
    if own:
        s["op"].execute(s["stream"], s["q"].data_ptr(), s["k"].data_ptr(), s["v"].data_ptr(), s["table"].data_ptr(),
                        s["lengths"].data_ptr(), s["o"].data_ptr(), lse=s["lse"].data_ptr(),
                        workspace=s["workspace"].data_ptr(), workspace_bytes=s["bytes"])
        return {"o": s["o"], "lse": s["lse"]}
    n, hk, group, page = c["n"], c["hk"], c["hq"] // c["hk"], c["page"]
    rows = s["table"].clamp(min=0).to(torch.int64)
    k = s["k"][rows].float().reshape(n, -1, hk, c["d"])
    v = s["v"][rows].float().reshape(n, -1, hk, c["dv"])
    q = s["q"].float().reshape(n, hk, group, c["d"]) * (1.0 / math.sqrt(c["d"]))
    at = torch.arange(s["columns"] * page, device="cuda")[None, :]
    length = s["lengths"].to(torch.int64)[:, None]
    seen = at < length
    if c["window"]:
        seen = seen & (at >= length - c["window"])
    scores = torch.einsum("nhgd,nthd->nhgt", q, k)
    scores = torch.where(seen[:, None, None, :], scores, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    o = torch.einsum("nhgt,nthd->nhgd", p, v) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return {"o": o.reshape(n, c["hq"], c["dv"]).to(TYPES[c["dtype"]]), "lse": lse.reshape(n, c["hq"])}


def _angles(s):
    """Cosines and sines [tokens, 1, pairs] of a step's positions."""
    turns = torch.remainder(s["pos"].double()[:, None] * s["turns"][None, :], 1.0).float()[:, None, :]
    return torch.cos(2 * math.pi * turns) * s["mult"], torch.sin(2 * math.pi * turns) * s["mult"]


def _rotated(x, cos, sin, rot, interleaved):
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., rot:]), -1) if rot < x.shape[-1] else y


def _normed(x, w, norm):
    """(normalised times weight, normalised, 1 / rms) in 32 bits."""
    x = x.float()
    if not norm:
        return x, x, None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r * w.float(), x * r, r


def _append(c, s):
    if own:
        weights = (s["wq"].data_ptr(), s["wk"].data_ptr()) if c["norm"] else (0, 0)
        s["op"].execute(s["stream"], s["pos"].data_ptr(), weights[0], weights[1], s["xq"].data_ptr(), s["yq"].data_ptr(),
                        s["xk"].data_ptr(), s["kpool"].data_ptr(), s["xv"].data_ptr(), s["vpool"].data_ptr(),
                        slots=s["slots"].data_ptr())
        return {"q": s["yq"], "k": s["kpool"], "v": s["vpool"]}
    cos, sin = _angles(s)
    kind, slots = TYPES[c["dtype"]], s["slots"].to(torch.int64)
    q = _rotated(_normed(s["xq"], s["wq"], c["norm"])[0], cos, sin, c["rot"], c["interleaved"]).to(kind)
    k = _rotated(_normed(s["xk"], s["wk"], c["norm"])[0], cos, sin, c["rot"], c["interleaved"]).to(kind)
    s["kpool"].view(-1, c["hk"], c["d"])[slots] = k
    s["vpool"].view(-1, c["hk"], c["d"])[slots] = s["xv"]
    return {"q": q, "k": s["kpool"], "v": s["vpool"]}


def _backward(x, w, dy, cos, sin, c):
    """Gradients of the input and of the norm's weight (32 bits)."""
    dm = _rotated(dy.float(), cos, -sin, c["rot"], c["interleaved"])   # the transposed rotation
    if not c["norm"]:
        return dm.to(x.dtype), torch.zeros(c["d"], device="cuda")
    _, n, r = _normed(x, w, True)
    g = dm * w.float()
    dx = r * (g - n * (g * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), (dm * n).sum((0, 1))


def _train(c, s):
    if own:
        at = {k: s[k].data_ptr() for k in ("pos", "wq", "wk", "xq", "xk", "yq", "yk", "dyq", "dyk", "dxq", "dxk", "dwq", "dwk")}
        if not c["norm"]:
            at["wq"] = at["wk"] = at["dwq"] = at["dwk"] = 0
        s["op"].execute(s["stream"], at["pos"], at["wq"], at["wk"], at["xq"], at["yq"], at["xk"], at["yk"])
        s["op"].backward(s["stream"], at["pos"], at["wq"], at["wk"], at["xq"], at["dyq"], at["dxq"], at["xk"], at["dyk"],
                         at["dxk"], dWq=at["dwq"], dWk=at["dwk"], workspace=s["workspace"].data_ptr(), workspace_bytes=s["bytes"])
        return {"yq": s["yq"], "yk": s["yk"], "dx": s["dpacked"], "dwq": s["dwq"], "dwk": s["dwk"]}
    cos, sin = _angles(s)
    kind = TYPES[c["dtype"]]
    yq = _rotated(_normed(s["xq"], s["wq"], c["norm"])[0], cos, sin, c["rot"], c["interleaved"]).to(kind)
    yk = _rotated(_normed(s["xk"], s["wk"], c["norm"])[0], cos, sin, c["rot"], c["interleaved"]).to(kind)
    dxq, dwq = _backward(s["xq"], s["wq"], s["dyq"], cos, sin, c)
    dxk, dwk = _backward(s["xk"], s["wk"], s["dyk"], cos, sin, c)
    return {"yq": yq, "yk": yk, "dx": torch.cat((dxq, dxk), 1), "dwq": dwq, "dwk": dwk}


def _pages(c, s):
    s["state"].copy_(s["before"])
    out = {"table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "pools": s["pools"]}
    if c["do"] == "step":
        out["slots"] = s["slots"]
    if own:
        op, stream = s["op"], s["stream"]
        table, lengths, refs = s["table"].data_ptr(), s["lengths"].data_ptr(), s["refs"].data_ptr()
        pools = [x.data_ptr() for x in s["pools"]]
        work = dict(workspace=s["workspace"].data_ptr(), workspace_bytes=s["bytes"])
        if c["do"] == "compact":
            op.compact(stream, table, refs, pools, **work)
            return out
        if c["frees"]:
            op.free(stream, s["frees"].data_ptr(), c["frees"], table, lengths, refs)
        if c["forks"]:
            op.fork(stream, s["src"].data_ptr(), s["dst"].data_ptr(), c["forks"], table, lengths, refs)
        op.extend(stream, s["new"].data_ptr(), table, lengths, refs, s["slots"].data_ptr(), c["new"], pools, **work)
        return out
    table, lengths, refs, pools = s["table"], s["lengths"], s["refs"], s["pools"]
    if c["do"] == "compact":
        ids = torch.arange(c["pool"], device="cuda")
        live = refs > 0
        count = live.sum()
        src, dst = ids[live & (ids >= count)], ids[~live & (ids < count)]
        to = ids.to(torch.int32)
        to[src] = dst.to(torch.int32)
        table.copy_(torch.where(table >= 0, to[table.clamp(min=0)], table))
        refs[dst] = refs[src]
        refs[src] = 0
        s["pools"] = [p.index_copy_(0, dst, p[src]) for p in pools]
        return out
    if c["frees"]:
        gone = table[s["frees"]]
        refs.index_add_(0, gone.clamp(min=0).reshape(-1), -(gone >= 0).to(torch.int32).reshape(-1))
        table[s["frees"]] = -1
        lengths[s["frees"]] = 0
    if c["forks"]:
        rows = table[s["src"]]
        refs.index_add_(0, rows.clamp(min=0).reshape(-1), (rows >= 0).to(torch.int32).reshape(-1))
        table[s["dst"]] = rows
        lengths[s["dst"]] = lengths[s["src"]]
    _extend(c, s, table, lengths, refs, pools)
    return out


def _extend(c, s, table, lengths, refs, pools):
    page, columns, new = c["page"], table.shape[1], s["new"].to(torch.int64)
    length = lengths.to(torch.int64)
    fits = (new > 0) & (length + new <= columns * page)
    first, after = (length + page - 1) // page, (length + new + page - 1) // page
    last = table.gather(1, (first - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0).to(torch.int64)
    shared = fits & (length % page != 0) & (refs[last] > 1)
    need = torch.where(fits, after - first + shared, 0)
    upto = torch.cumsum(need, 0)
    free = refs == 0
    granted = fits & (upto <= free.sum())
    rank = torch.cumsum(free, 0) - 1
    ids = torch.arange(c["pool"], device="cuda")
    order = torch.zeros(c["pool"] + 1, dtype=torch.int64, device="cuda").scatter_(0, torch.where(free, rank, c["pool"]), ids)
    begin = upto - need
    copied = (shared & granted)
    refs.add_((free & (rank < torch.where(granted, need, 0).sum())).to(torch.int32))
    refs.index_add_(0, last, -copied.to(torch.int32))
    column = torch.arange(columns, device="cuda")[None, :]
    fresh = granted[:, None] & (column >= first[:, None]) & (column < after[:, None])
    at = torch.where(fresh, begin[:, None] + copied[:, None] + column - first[:, None], 0)
    swap = copied[:, None] & (column == first[:, None] - 1)
    own_page = order[begin.clamp(max=c["pool"])]
    table.copy_(torch.where(fresh, order[at.clamp(0, c["pool"])], torch.where(swap, own_page[:, None], table.to(torch.int64))))
    src, dst = last[copied], own_page[copied]
    s["pools"] = [p.index_copy_(0, dst, p[src]) for p in pools]
    token = torch.arange(c["new"], device="cuda")[None, :]
    place = length[:, None] + token
    into = table.gather(1, (place // page).clamp(max=columns - 1)).to(torch.int64)
    s["slots"].copy_(torch.where(granted[:, None] & (token < new[:, None]), into * page + place % page, -1))
    lengths.add_(torch.where(granted, new, 0).to(torch.int32))


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "attention":
        size, lens = BYTES[c["dtype"]], _lengths(c["n"], c["shortest"], c["longest"], c["empty"])
        seen = sum(min(x, c["window"]) if c["window"] else x for x in lens)
        pages = sum(-(-x // c["page"]) for x in lens)
        cache = seen * c["hk"] * (c["d"] + c["dv"]) * size
        return {"bytes": cache + c["n"] * c["hq"] * ((c["d"] + c["dv"]) * size + 4) + 4 * (pages + c["n"]),
                "flops": 2 * seen * c["hq"] * (c["d"] + c["dv"])}
    if c["kind"] == "append":
        values = c["t"] * (c["hq"] + 2 * c["hk"]) * c["d"]
        return {"bytes": 2 * values * BYTES[c["dtype"]] + 8 * c["t"], "flops": values * (7 if c["norm"] else 3)}
    if c["kind"] == "train":
        values = c["t"] * (c["hq"] + c["hk"]) * c["d"]
        # forward: x read, y written; backward: dy read, dx written, x read again only where there is a norm
        return {"bytes": values * BYTES[c["dtype"]] * (5 if c["norm"] else 4) + 4 * c["t"], "flops": values * (19 if c["norm"] else 6)}
    block = c["page"] * c["hk"] * c["d"] * BYTES[c["dtype"]] * c["tensors"]
    held = sum(-(-x // c["page"]) for x in _lengths(c["n"], 1, c["longest"], 0))
    if c["do"] == "compact":
        moved = held * (c["pool"] - held) / c["pool"]     # expected: live pages beyond the live count
        return {"bytes": 2 * moved * block + 4 * (c["pool"] + 2 * held), "flops": c["pool"]}
    shared = 2 * c["forks"] * (c["page"] - 1) / c["page"]  # expected: both sides of a fork copy their last page
    rows = held / c["n"]
    return {"bytes": 2 * shared * block + 4 * (c["pool"] + rows * (c["frees"] * 2 + c["forks"] * 3) + c["n"] * (4 + c["new"])),
            "flops": c["pool"]}


# ---- the definition in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    g = _generator(seed)
    s = {"case": case, "seed": seed}
    if case["kind"] == "attention":
        _prepare_attention(case, g, s)
        return _exact_attention(case, s)
    if case["kind"] == "append":
        _prepare_append(case, g, s)
        return _exact_append(case, s)
    if case["kind"] == "train":
        _prepare_train(case, g, s)
        return _exact_train(case, s)
    _prepare_pages(case, g, s)
    return _exact_pages(case, s)


def _exact_attention(c, s):
    o = torch.zeros((c["n"], c["hq"], c["dv"]), dtype=torch.float64, device="cuda")
    lse = torch.full((c["n"], c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    group = c["hq"] // c["hk"]
    for i, length in enumerate(s["lengths"].tolist()):
        low = max(0, length - c["window"]) if c["window"] else 0
        if length <= low:
            continue
        at = torch.arange(low, length, device="cuda")
        pages, inside = s["table"][i, at // c["page"]].long(), at % c["page"]
        for h in range(c["hk"]):
            k, v = s["k"][pages, inside, h].double(), s["v"][pages, inside, h].double()
            x = s["q"][i, h * group:(h + 1) * group].double() @ k.T / math.sqrt(c["d"])
            o[i, h * group:(h + 1) * group] = torch.softmax(x, -1) @ v
            lse[i, h * group:(h + 1) * group] = torch.logsumexp(x, -1)
    return {"o": o, "lse": lse}


def _exact_heads(c, s, x, w):
    """Norm and rotation of [tokens, heads, d] in 64 bits, as complex products."""
    x = x.double()
    if c["norm"]:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * w.double()
    half = c["rot"] // 2
    angle = s["pos"].double()[:, None, None] * torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    first = torch.arange(half, device="cuda") * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else half)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(angle, s["mult"]), angle)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(c, s):
    k, v = s["kpool"].double(), s["vpool"].double()
    slots = s["slots"].long()
    k[slots // c["page"], slots % c["page"]] = _exact_heads(c, s, s["xk"], s["wk"])
    v[slots // c["page"], slots % c["page"]] = s["xv"].double()
    return {"q": _exact_heads(c, s, s["xq"], s["wq"]), "k": k, "v": v}


def _exact_train(c, s):
    out, dx = {}, []
    for y, x, w, dy, dw in (("yq", "xq", "wq", "dyq", "dwq"), ("yk", "xk", "wk", "dyk", "dwk")):
        a, b = s[x].double().requires_grad_(), s[w].double().requires_grad_()
        z = _exact_heads(c, s, a, b)
        z.backward(s[dy].double())
        out[y] = z.detach()
        out[dw] = b.grad if b.grad is not None else torch.zeros(c["d"], dtype=torch.float64, device="cuda")
        dx.append(a.grad)
    out["dx"] = torch.cat(dx, 1)
    return out


def _exact_pages(c, s):
    """The pools after the step; whole numbers are compared by themselves."""
    table, lengths, refs = (s[x].cpu().numpy().copy() for x in ("table", "lengths", "refs"))
    moves = []
    if c["do"] == "compact":
        count = int((refs > 0).sum())
        holes = [p for p in range(count) if refs[p] == 0]
        late = [p for p in range(count, c["pool"]) if refs[p] > 0]
        moves = list(zip(late, holes))
    else:
        for f in s["frees"].tolist():
            for p in table[f][table[f] >= 0]:
                refs[p] -= 1
            table[f], lengths[f] = -1, 0
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            table[b], lengths[b] = table[a], lengths[a]
            for p in table[a][table[a] >= 0]:
                refs[p] += 1
        empty = [int(p) for p in np.flatnonzero(refs == 0)]
        at = 0
        for i in range(c["n"]):
            length, to = int(lengths[i]), int(lengths[i]) + c["new"]
            if to > table.shape[1] * c["page"]:
                continue
            held = -(-length // c["page"])
            own_last = length % c["page"] != 0 and refs[table[i][held - 1]] > 1
            need = -(-to // c["page"]) - held + int(own_last)
            if at + need > len(empty):
                break
            if own_last:
                moves.append((int(table[i][held - 1]), empty[at]))
            at += need
    pools = []
    for p in s["pools"]:
        q = p.double() if p.numel() <= (1 << 30) else None
        if q is not None and moves:
            src, dst = (torch.tensor([m[k] for m in moves], device="cuda") for k in (0, 1))
            q[dst] = p[src].double()
        pools.append(q)
    return {"pools": pools}
