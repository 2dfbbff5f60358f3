"""The rest of a decoder layer on real work: what stands around the rotary positions and the paged cache.

Three kinds of case:

  norm     the residual's addition and the root-mean-square norm after it: serving (the norm's result in 8 bits
           with scales, or in the model's type) and training (forward and backward)
  linear   products with 4-bit weights and group scales for the few tokens of a decode step, plain or as the gated
           half of a feed-forward block (activation and product included)
  tree     attention of a tree of drafted tokens of each sequence over its paged key-value cache

`own = False` computes a case with elementary torch operations in 32 bits, rounded once at the end;
`own = True` makes the calls a user makes of the library.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-5
_handle = None


def _library():
    """The binding and one handle for the process, as a program keeps them."""
    global _handle
    from paper_2601_07827_b200 import api
    if _handle is None:
        _handle = api.Handle()
    return api, _handle


# ---- the cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # the norm between two projections of a decode step of 16 tokens, result in 8 bits for the next product
        dict(name="norm decode 8 bit", kind="norm", t=16, d=4096, dtype="bf16", stream="bf16", out="e4m3", group=0,
             backward=False),
        # prefill of a large model: residual stream kept in 32 bits, scales for groups of 128
        dict(name="norm prefill 8 bit", kind="norm", t=8192, d=8192, dtype="bf16", stream="f32", out="e4m3", group=128,
             backward=False),
        # one training step's layer: 16 ki tokens, forward and backward
        dict(name="norm train", kind="norm", t=16384, d=4096, dtype="bf16", stream="bf16", out="bf16", group=0,
             backward=True),
        # a small 32-bit model with odd sizes
        dict(name="norm train odd f32", kind="norm", t=777, d=1001, dtype="f32", stream="f32", out="f32", group=0,
             backward=True),
        # one user's token through the queries', keys' and values' projection
        dict(name="linear one token", kind="linear", t=1, k=4096, n=6144, dtype="f16", out="f16", scales="f16", group=128,
             xgroup=0, zeros=False, act="none"),
        # the gated half of a feed-forward block for a decode step of 8 tokens
        dict(name="linear gated decode", kind="linear", t=8, k=4096, n=14336, dtype="bf16", out="bf16", scales="bf16",
             group=64, xgroup=0, zeros=True, act="silu"),
        # the same for a large model and the drafts of a few requests, input in 8 bits as the norm left it
        dict(name="linear gated drafts 8 bit", kind="linear", t=32, k=8192, n=28672, dtype="e4m3", out="bf16", scales="f16",
             group=128, xgroup=0, zeros=False, act="silu"),
        # a small 32-bit model with odd sizes
        dict(name="linear odd f32", kind="linear", t=5, k=1001, n=777, dtype="f32", out="f32", scales="f32", group=32,
             xgroup=0, zeros=True, act="none"),
        # one user: 16 drafted tokens after 1500 cached ones
        dict(name="tree one request", kind="tree", n=1, t=16, hq=32, hk=8, d=128, dv=128, page=16, shortest=1500,
             longest=1500, unused=0, window=0, dtype="bf16"),
        # a server's ordinary verification step: requests of very different ages, trees of up to 32 drafts
        dict(name="tree batch", kind="tree", n=32, t=32, hq=32, hk=8, d=128, dv=128, page=16, shortest=64, longest=8192,
             unused=7, window=0, dtype="bf16"),
        # long documents with large trees: a gigabyte of cache
        dict(name="tree long", kind="tree", n=4, t=64, hq=64, hk=8, d=128, dv=128, page=64, shortest=65536, longest=65536,
             unused=0, window=0, dtype="f16"),
        # a small 32-bit model with odd head sizes and a sliding window
        dict(name="tree window f32", kind="tree", n=12, t=7, hq=20, hk=4, d=80, dv=72, page=24, shortest=10, longest=4100,
             unused=2, window=1000, dtype="f32"),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    kind = rng.choice(["norm", "linear", "tree"])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        stream = rng.choice([dtype, dtype, "f32"])
        out = rng.choice([dtype, "e4m3"])
        d = rng.choice([_spread(rng, 64, 8192), 32 * _spread(rng, 2, 256), rng.choice([2048, 4096, 5120, 8192])])
        t = _spread(rng, 1, min(20000, 8192 * 4096 // d))
        return dict(kind="norm", t=t, d=d, dtype=dtype, stream=stream, out=out,
                    group=rng.choice([0, 32, 64, 128]) if out == "e4m3" else 0, backward=out != "e4m3" and rng.random() < 0.7)
    if kind == "linear":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32", "e4m3"])
        act = rng.choice(["none", "none", "silu", "gelu"])
        k = rng.choice([_spread(rng, 64, 8192), 64 * _spread(rng, 2, 128)])
        n = rng.choice([_spread(rng, 16, 28672), 16 * _spread(rng, 2, 1792)])
        group = rng.choice([0, 32, 64, 128, 128])
        return dict(kind="linear", t=rng.choice([1, _spread(rng, 1, 32), rng.randint(1, 32)]), k=k, n=n, dtype=dtype,
                    out=rng.choice(["bf16", "f16"]) if dtype == "e4m3" else dtype, scales=rng.choice(["f16", "bf16", "f32"]),
                    group=group, xgroup=rng.choice([0, 128]) if dtype == "e4m3" else 0, zeros=rng.random() < 0.5, act=act)
    hk = rng.choice([1, 2, 3, 4, 8])
    hq = hk * rng.choice([1, 2, 4, 4, 7, 8])
    d = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256])
    dv = rng.choice([d, d, d, max(32, d - 64)])
    t = rng.choice([_spread(rng, 1, 64), rng.randint(2, 64)])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    longest = _spread(rng, 16, 65536)
    # rows times tokens at most a quarter of the largest listed case's, the cache at most half of its
    most = min(134217728 // (longest * hk * max(d, dv)), 268435456 // (longest * hq * t))
    n = _spread(rng, 1, max(1, min(200, most)))
    while n * longest * hq * t > 268435456:
        t, longest = max(1, t // 2), max(16, longest // 2)
    window = rng.choice([0, 0, 0, t + _spread(rng, 1, longest)])
    return dict(kind="tree", n=n, t=t, hq=hq, hk=hk, d=d, dv=dv, page=rng.choice([8, 16, 16, 24, 32, 64, 128]),
                shortest=_spread(rng, 1, longest), longest=longest, unused=rng.randint(0, t // 3), window=window, dtype=dtype)


def _lengths(n, shortest, longest):
    """n lengths, even over their logarithm from shortest to longest."""
    f = [shortest * (longest / shortest) ** ((i + 0.5) / n) for i in range(n)]
    return [max(1, min(longest, int(round(x)))) for x in f]


# ---- inputs -------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(TYPES[dtype])


def _empty(shape, dtype):
    return torch.empty(shape, dtype=TYPES[dtype], device="cuda")


def _pieces(extent, group):
    """How many groups an extent has (group 0: one)."""
    return -(-extent // group) if group else 1


def prepare(case, seed):
    s = {"case": case}
    {"norm": _prepare_norm, "linear": _prepare_linear, "tree": _prepare_tree}[case["kind"]](case, _generator(seed), s)
    if own:
        {"norm": _plan_norm, "linear": _plan_linear, "tree": _plan_tree}[case["kind"]](case, s)
        s["stream"] = torch.cuda.current_stream().cuda_stream
    return s


def _prepare_norm(c, g, s):
    t, d = c["t"], c["d"]
    # a block's output and the residual stream it is added to; a few channels of the stream are large
    s["x"] = _normal(g, (t, d), c["dtype"])
    stream = torch.randn((t, d), generator=g, device="cuda")
    stream[:, ::97] *= 20.0
    s["r"] = stream.to(TYPES[c["stream"]])
    s["w"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(TYPES[c["dtype"]])
    if c["backward"]:
        s["dy"] = _normal(g, (t, d), c["dtype"])
        s["dh"] = _normal(g, (t, d), c["stream"])


def _prepare_linear(c, g, s):
    t, k = c["t"], c["k"]
    rows = c["n"] * (1 if c["act"] == "none" else 2)
    s["codes"] = torch.randint(0, 256, (rows, (k + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
    groups = _pieces(k, c["group"])
    s["scales"] = ((0.5 + torch.rand((rows, groups), generator=g, device="cuda")) / (4.6 * math.sqrt(k))).to(TYPES[c["scales"]])
    s["zeros"] = torch.randint(5, 11, (rows, groups), generator=g, device="cuda", dtype=torch.uint8) if c["zeros"] else None
    x = torch.randn((t, k), generator=g, device="cuda") * 1.5
    if c["dtype"] == "e4m3":
        # as a norm leaves it: every group's largest value is 448 times its scale
        size = c["xgroup"] or k
        padded = torch.zeros((t, _pieces(k, c["xgroup"]) * size), device="cuda")
        padded[:, :k] = x
        padded = padded.view(t, -1, size)
        s["xs"] = padded.abs().amax(-1).clamp(min=1e-30) / 448.0
        s["x"] = (padded / s["xs"][..., None]).view(t, -1)[:, :k].contiguous().to(torch.float8_e4m3fn)
    else:
        s["x"], s["xs"] = x.to(TYPES[c["dtype"]]), None


def _prepare_tree(c, g, s):
    n, t, page, hk = c["n"], c["t"], c["page"], c["hk"]
    counted = _lengths(n, c["shortest"], c["longest"])
    lens = torch.tensor(counted, device="cuda", dtype=torch.int64)[torch.randperm(n, generator=g, device="cuda")]
    columns = -(-(c["longest"] + t) // page)
    held = (lens + t + page - 1) // page
    pool = sum(-(-(x + t) // page) for x in counted)
    pool += pool // 16 + 2
    # page tables: pages drawn at random from the pool, -1 behind the last
    taken = torch.arange(columns, device="cuda")[None, :] < held[:, None]
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    rank = (torch.cumsum(taken.reshape(-1), 0) - 1).clamp(min=0)
    s["table"] = torch.where(taken, order[rank].reshape(taken.shape), -1).to(torch.int32)
    s["lengths"], s["columns"] = lens.to(torch.int32), columns
    # trees: every draft continues an earlier one or the last cached token; the last `unused` rows of every
    # second sequence hold no draft
    parent = (torch.rand((n, t), generator=g, device="cuda") * (torch.arange(t, device="cuda") + 1)).long() - 1
    sees = torch.zeros((n, t, t), dtype=torch.bool, device="cuda")
    sequence = torch.arange(n, device="cuda")
    for i in range(t):
        before = sees[sequence, parent[:, i].clamp(min=0)] & (parent[:, i] >= 0)[:, None]
        before[:, i] = True
        sees[:, i] = before
    if c["unused"]:
        sees[::2, t - c["unused"]:] = False
    words = -(-t // 32)
    bits = torch.zeros((n, t, words * 32), dtype=torch.int64, device="cuda")
    bits[:, :, :t] = sees
    packed = (bits.view(n, t, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    s["masks"] = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)
    s["q"] = _normal(g, (n, t, c["hq"], c["d"]), c["dtype"], 1.5)
    s["k"] = _normal(g, (pool, page, hk, c["d"]), c["dtype"])
    s["v"] = _normal(g, (pool, page, hk, c["dv"]), c["dtype"])


# ---- operation objects, workspaces and outputs: made once, kept by the program --------------------------

def _info(t):
    api, h = _library()
    return api.TensorInfo(h, api.dtype_code(t.dtype), t.shape, t.stride())


def _workspace(s):
    s["bytes"] = s["op"].workspace_size()
    s["workspace"] = torch.empty(max(s["bytes"], 1), dtype=torch.uint8, device="cuda")


def _plan_norm(c, s):
    api, h = _library()
    t, d = c["t"], c["d"]
    s["h"], s["y"] = _empty((t, d), c["stream"]), _empty((t, d), c["out"])
    s["s"] = _empty((t, _pieces(d, c["group"])), "f32") if c["out"] == "e4m3" else None
    if c["backward"]:
        s["dx"], s["dw"] = _empty((t, d), c["dtype"]), _empty((d,), "f32")
        s["dr"] = _empty((t, d), c["stream"]) if c["stream"] != c["dtype"] else None
    s["op"] = api.AddNorm(h, _info(s["x"]), _info(s["y"]), R=_info(s["r"]), H=_info(s["h"]),
                          S=_info(s["s"]) if s["s"] is not None else None, group=c["group"], eps=EPS)
    _workspace(s)


def _plan_linear(c, s):
    api, h = _library()
    s["y"] = _empty((c["t"], c["n"]), c["out"])
    s["op"] = api.Linear4(h, _info(s["x"]), _info(s["y"]), scale_type=api.dtype_code(s["scales"].dtype), group=c["group"],
                          zeros=c["zeros"], activation=c["act"], XS=_info(s["xs"]) if s["xs"] is not None else None,
                          x_group=c["xgroup"])
    s["packed"] = torch.empty(s["op"].packed_size(), dtype=torch.uint8, device="cuda")
    s["op"].pack(torch.cuda.current_stream().cuda_stream, s["codes"].data_ptr(), s["scales"].data_ptr(),
                 s["zeros"].data_ptr() if c["zeros"] else 0, s["packed"].data_ptr())
    _workspace(s)


def _plan_tree(c, s):
    api, h = _library()
    s["o"] = _empty((c["n"], c["t"], c["hq"], c["dv"]), c["dtype"])
    s["lse"] = _empty((c["n"], c["t"], c["hq"]), "f32")
    s["op"] = api.TreeAttention(h, _info(s["q"]), _info(s["k"]), _info(s["v"]), _info(s["table"]), _info(s["masks"]),
                                _info(s["o"]), scale=1.0 / math.sqrt(c["d"]), window=c["window"])
    _workspace(s)


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    return {"norm": _norm, "linear": _linear, "tree": _tree}[state["case"]["kind"]](state["case"], state)


def _norm(c, s):
    if own:
        op, stream = s["op"], s["stream"]
        op.execute(stream, s["x"].data_ptr(), s["w"].data_ptr(), s["y"].data_ptr(), R=s["r"].data_ptr(), H=s["h"].data_ptr(),
                   S=s["s"].data_ptr() if s["s"] is not None else 0)
        out = {"h": s["h"], "y": s["y"]}
        if s["s"] is not None:
            out["s"] = s["s"]
        if c["backward"]:
            op.backward(stream, s["h"].data_ptr(), s["w"].data_ptr(), s["dy"].data_ptr(), dH=s["dh"].data_ptr(),
                        dX=s["dx"].data_ptr(), dR=s["dr"].data_ptr() if s["dr"] is not None else 0, dW=s["dw"].data_ptr(),
                        workspace=s["workspace"].data_ptr(), workspace_bytes=s["bytes"])
            out["dx"], out["dw"] = s["dx"], s["dw"]
            if s["dr"] is not None:
                out["dr"] = s["dr"]
        return out
    h, w = s["x"].float() + s["r"].float(), s["w"].float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * w
    out = {"h": h.to(TYPES[c["stream"]])}
    if c["out"] == "e4m3":
        size, t, d = c["group"] or c["d"], c["t"], c["d"]
        blocks = torch.nn.functional.pad(y, (0, -d % size)).view(t, -1, size)
        scale = (blocks.abs().amax(-1) / 448.0).clamp(min=2.0 ** -126)
        out["y"] = (blocks / scale[..., None]).view(t, -1)[:, :d].to(TYPES["e4m3"])
        out["s"] = scale
        return out
    out["y"] = y.to(TYPES[c["out"]])
    if c["backward"]:
        h = out["h"].float()                     # what the forward pass kept
        r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
        dy, n = s["dy"].float(), h * r
        g = dy * w
        total = s["dh"].float() + r * (g - n * (g * n).mean(-1, keepdim=True))
        out["dx"], out["dw"] = total.to(TYPES[c["dtype"]]), (dy * n).sum(0)
        if c["stream"] != c["dtype"]:
            out["dr"] = total.to(TYPES[c["stream"]])
    return out


def _activation(x, act):
    if act == "silu":
        return x / (1.0 + torch.exp(-x))
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _weights(c, s, kind, rows):
    """The given rows' weights (code - zero) * scale."""
    codes, k = s["codes"][rows], c["k"]
    code = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1)[:, :k].to(kind)
    size = c["group"] or k
    spread = lambda v: v[rows].to(kind).repeat_interleave(size, 1)[:, :k]  # noqa: E731
    return (code - (spread(s["zeros"]) if c["zeros"] else 8)) * spread(s["scales"])


def _linear(c, s):
    if own:
        s["op"].execute(s["stream"], s["packed"].data_ptr(), s["x"].data_ptr(), s["y"].data_ptr(),
                        XS=s["xs"].data_ptr() if s["xs"] is not None else 0, workspace=s["workspace"].data_ptr(),
                        workspace_bytes=s["bytes"])
        return s["y"]
    x = s["x"].float()
    if s["xs"] is not None:
        x = x * s["xs"].repeat_interleave(c["xgroup"] or c["k"], 1)[:, :c["k"]]
    z = x @ _weights(c, s, torch.float32, slice(None)).T
    if c["act"] != "none":
        z = _activation(z[:, :c["n"]], c["act"]) * z[:, c["n"]:]
    return z.to(TYPES[c["out"]])


def _tree(c, s):
    if own:
        s["op"].execute(s["stream"], s["q"].data_ptr(), s["k"].data_ptr(), s["v"].data_ptr(), s["table"].data_ptr(),
                        s["lengths"].data_ptr(), s["masks"].data_ptr(), s["o"].data_ptr(), lse=s["lse"].data_ptr(),
                        workspace=s["workspace"].data_ptr(), workspace_bytes=s["bytes"])
        return {"o": s["o"], "lse": s["lse"]}
    n, t, hk, group = c["n"], c["t"], c["hk"], c["hq"] // c["hk"]
    rows = s["table"].clamp(min=0).to(torch.int64)
    k = s["k"][rows].float().reshape(n, -1, hk, c["d"])
    v = s["v"][rows].float().reshape(n, -1, hk, c["dv"])
    q = s["q"].float().reshape(n, t, hk, group, c["d"]) * (1.0 / math.sqrt(c["d"]))
    at = torch.arange(s["columns"] * c["page"], device="cuda")[None, None, :]
    length = s["lengths"].to(torch.int64)[:, None, None]
    bits = (s["masks"].to(torch.int64)[..., None] >> torch.arange(32, device="cuda")) & 1
    bits = bits.reshape(n, t, -1)[:, :, :t]
    count = bits.sum(-1, keepdim=True)
    draft = (at - length).clamp(0, t - 1).expand(n, t, -1)
    seen = torch.where(at < length, count > 0, (at < length + t) & (bits.gather(2, draft) > 0))
    if c["window"]:
        seen = seen & ((at >= length + count - c["window"]) | (at >= length))
    seen = seen[:, None, None]
    scores = torch.einsum("nthgd,nshd->nhgts", q, k)
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    o = torch.einsum("nhgts,nshd->nhgtd", p, v) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)[..., 0]
    return {"o": o.permute(0, 3, 1, 2, 4).reshape(n, t, c["hq"], c["dv"]).to(TYPES[c["dtype"]]),
            "lse": lse.permute(0, 3, 1, 2).reshape(n, t, c["hq"])}


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "norm":
        values = c["t"] * c["d"]
        x, stream, out = BYTES[c["dtype"]], BYTES[c["stream"]], BYTES[c["out"]]
        nbytes = values * (x + 2 * stream + out) + c["d"] * x
        if c["out"] == "e4m3":
            nbytes += 4 * c["t"] * _pieces(c["d"], c["group"])
        if c["backward"]:
            # the kept sum, the result's and the stream's gradients read; the input's and the stream's written
            nbytes += values * (2 * stream + 2 * x + (stream if stream != x else 0)) + 4 * c["d"]
        return {"bytes": nbytes, "flops": values * (20 if c["backward"] else 6)}
    if c["kind"] == "linear":
        rows, groups = c["n"] * (1 if c["act"] == "none" else 2), _pieces(c["k"], c["group"])
        weights = rows * ((c["k"] + 1) // 2 + groups * (BYTES[c["scales"]] + int(c["zeros"])))
        scales = 4 * c["t"] * _pieces(c["k"], c["xgroup"]) if c["dtype"] == "e4m3" else 0
        return {"bytes": weights + c["t"] * (c["k"] * BYTES[c["dtype"]] + c["n"] * BYTES[c["out"]]) + scales,
                "flops": 2 * c["t"] * rows * c["k"]}
    size, lens = BYTES[c["dtype"]], _lengths(c["n"], c["shortest"], c["longest"])
    read = seen = 0
    depth = 1.0 + math.log(c["t"])                       # a random tree's usual depth: drafts that a row sees
    for i, x in enumerate(lens):
        rows = c["t"] - (c["unused"] if i % 2 == 0 else 0)
        cached = min(x, c["window"]) if c["window"] else x
        read += cached + c["t"]
        seen += rows * (cached + depth)
    heads = c["n"] * c["t"] * c["hq"]
    return {"bytes": int(read * c["hk"] * (c["d"] + c["dv"]) * size + heads * ((c["d"] + c["dv"]) * size + 4)
                         + 4 * c["n"] * c["t"] * -(-c["t"] // 32) + 4 * (read // c["page"] + c["n"])),
            "flops": int(2 * seen * c["hq"] * (c["d"] + c["dv"]))}


# ---- the definition in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    s = {"case": case}
    g = _generator(seed)
    if case["kind"] == "norm":
        _prepare_norm(case, g, s)
        return _exact_norm(case, s)
    if case["kind"] == "linear":
        _prepare_linear(case, g, s)
        return _exact_linear(case, s)
    _prepare_tree(case, g, s)
    return _exact_tree(case, s)


def _exact_norm(c, s):
    w, h = s["w"].double(), s["x"].double() + s["r"].double()
    y = h / (h.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt() * w
    out = {"h": h, "y": y}
    if c["out"] == "e4m3":
        size = c["group"] or c["d"]
        out["s"] = torch.stack([p.abs().amax(-1) for p in y.split(size, 1)], 1) / 448.0
        out["y"] = torch.cat([p / out["s"][:, i:i + 1] for i, p in enumerate(y.split(size, 1))], 1)
    if c["backward"]:
        # the backward pass is that of the norm of the kept sum, which the stream's type holds
        kept, w = h.to(TYPES[c["stream"]]).double().requires_grad_(), w.requires_grad_()
        z = kept / (kept.pow(2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt() * w
        dh, out["dw"] = torch.autograd.grad(z, (kept, w), s["dy"].double())
        out["dx"] = dh + s["dh"].double()
        if c["stream"] != c["dtype"]:
            out["dr"] = out["dx"]
    return out


def _exact_linear(c, s):
    t, k, rows = c["t"], c["k"], s["codes"].shape[0]
    x = s["x"].double()
    if s["xs"] is not None:
        x = x * s["xs"].double()[:, torch.arange(k, device="cuda") // (c["xgroup"] or k)]
    z = torch.empty((t, rows), dtype=torch.float64, device="cuda")
    at = torch.arange(k, device="cuda")
    for a in range(0, rows, 4096):
        b = min(rows, a + 4096)
        code = (s["codes"][a:b, at // 2].int() >> (4 * (at % 2))) & 15
        which = at // (c["group"] or k)
        zero = s["zeros"][a:b, which].double() if c["zeros"] else 8.0
        z[:, a:b] = x @ ((code.double() - zero) * s["scales"][a:b, which].double()).T
    if c["act"] == "none":
        return z
    g, u = z[:, :c["n"]], z[:, c["n"]:]
    if c["act"] == "silu":
        return g * torch.sigmoid(g) * u
    return torch.nn.functional.gelu(g, approximate="tanh") * u


def _exact_tree(c, s):
    n, t, hq, hk = c["n"], c["t"], c["hq"], c["hk"]
    o = torch.zeros((n, t, hq, c["dv"]), dtype=torch.float64, device="cuda")
    lse = torch.full((n, t, hq), -math.inf, dtype=torch.float64, device="cuda")
    group = hq // hk
    masks = s["masks"].cpu().tolist()
    for i, length in enumerate(s["lengths"].tolist()):
        bits = [[(masks[i][r][j // 32] >> (j % 32)) & 1 for j in range(t)] for r in range(t)]
        used = [r for r in range(t) if any(bits[r])]
        if not used:
            continue
        low = [max(0, length + sum(bits[r]) - c["window"]) if c["window"] else 0 for r in used]
        first = min(low + [length])
        at = torch.arange(first, length + t, device="cuda")
        pages, inside = s["table"][i, at // c["page"]].long(), at % c["page"]
        cached = at[None, :] >= torch.tensor(low, device="cuda")[:, None]
        cached[:, length - first:] = torch.tensor([bits[r] for r in used], dtype=torch.bool, device="cuda")
        for h in range(hk):
            k, v = s["k"][pages, inside, h].double(), s["v"][pages, inside, h].double()
            for j in range(h * group, (h + 1) * group):
                x = s["q"][i, used, j].double() @ k.T / math.sqrt(c["d"])
                x = x.masked_fill(~cached, -math.inf)
                o[i, used, j] = torch.softmax(x, -1) @ v
                lse[i, used, j] = torch.logsumexp(x, -1)
    return {"o": o, "lse": lse}
