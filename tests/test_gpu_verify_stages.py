"""The layer of examples/verify.py stage by stage: what each operation stored, from what the operations before it stored, within the bounds of a single
rounding (so that a code that falls to the other side of a border in one stage does not widen the bounds of the next)."""
import importlib.util
import os

import pytest
import torch

from conftest import ROOT
from decoder_reference import E32, UNIT, attention_bounds, rotary_forward
from layer_reference import NORM_CHAIN, check, check_e4m3, linear4, mask_words, norm_forward, random_trees, tree_attention

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("verify_example", os.path.join(ROOT, "examples", "verify.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("seed", [1, 2])
def test_stages(example, seed):
    e, layer = example, example.Layer(seed)
    g = torch.Generator().manual_seed(seed)
    n, t = e.SEQUENCES, e.DRAFTS
    lengths = [0, 7, 64, e.CAPACITY - t]
    sees = random_trees(n, t, seed, unused=3)
    places = layer.places.cpu()
    layer.keys.copy_(torch.randn(layer.keys.shape, generator=g).to(BF16))
    layer.values.copy_(torch.randn(layer.values.shape, generator=g).to(BF16))
    depth = sees.sum(-1) - 1
    slots = torch.stack([places[i, x:x + t] for i, x in enumerate(lengths)])
    positions = torch.tensor(lengths)[:, None] + depth.clamp(min=0)
    layer.x.copy_(torch.randn(layer.x.shape, generator=g).to(BF16))
    layer.stream.copy_((3 * torch.randn(layer.x.shape, generator=g)).to(BF16))
    layer.masks.copy_(mask_words(sees))
    layer.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    layer.positions.copy_(positions.view(-1).to(torch.int32))
    layer.slots.copy_(torch.where(depth >= 0, slots, -1).view(-1).to(torch.int32))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        layer.step()
    graph.replay()
    torch.cuda.synchronize()
    assert layer.flags.item() == 0

    def norm(x, r, w, h, codes, scales):
        eh, ey = norm_forward(x.cpu(), w.cpu(), r.cpu(), e.EPS)
        check(h, eh, (UNIT[BF16] + E32) * eh.abs())
        check_e4m3(codes, scales, ey, 0, NORM_CHAIN)

    def product(x, xs, weights, kind, y):
        want, bound = linear4(x.cpu(), xs.cpu() if xs is not None else None, 0, weights.numbers, kind, BF16)
        check(y, want, bound)

    norm(layer.x, layer.stream, layer.norm_1, layer.h1, layer.n1, layer.s1)
    product(layer.n1, layer.s1, layer.w_qkv, "none", layer.qkv.view(n * t, -1))
    q, k, v = (p.cpu() for p in layer.parts)
    at = positions.view(-1)
    # a rotation: two products, a sum, and angles of 2^-22 of a radian
    turned = lambda z: rotary_forward(z, None, at, layer.freq, layer.mult, False, False, 0.0)  # noqa: E731
    bound = lambda want, z: UNIT[BF16] * want.abs() + 8 * E32 * z.double().abs().amax(-1, keepdim=True) * 2  # noqa: E731
    check(layer.q, turned(q), bound(turned(q), q))
    held = (depth >= 0).view(-1)
    where = slots.view(-1)[held].long()
    kept = layer.keys.cpu().view(-1, e.KEY_HEADS, e.HEAD)[where]
    check(kept, turned(k)[held], bound(turned(k), k)[held])
    assert torch.equal(layer.values.cpu().view(-1, e.KEY_HEADS, e.HEAD)[where], v[held])
    want = tree_attention(layer.q.view(n, t, e.HEADS, e.HEAD), layer.keys, layer.values, layer.table.cpu(), lengths, sees, e.HEAD ** -0.5, 0)
    check(layer.o.view(n, t, e.HEADS, e.HEAD), want[0], attention_bounds(*want, e.HEAD, BF16)[0])
    product(layer.o.view(n * t, -1), None, layer.w_out, "none", layer.a)
    norm(layer.a, layer.h1, layer.norm_2, layer.h2, layer.n2, layer.s2)
    product(layer.n2, layer.s2, layer.w_up, "silu", layer.f)
    product(layer.f, None, layer.w_down, "none", layer.y)
