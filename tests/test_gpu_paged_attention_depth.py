"""Caches so large that every warp takes dozens of tiles: its ring of buffers goes round many times, maxima move again and
again inside a warp, a warp holds many items (a sequence's key head) or a small part of one.

All sizes of head and group that the kernel has a form for.  Bounds: those of the small shapes (decoder_reference), and
for fp32, where they are wide, the norm of the error over all outputs against that of a plain fp32 evaluation of the
same data: products in three parts and sums rounded to nearest are as good as fp32 products and sums, so 1.5 times its
error and 2^-24 of the outputs' norm are allowed.  (Without the low parts the error is 100 times larger, see
test_decoder_bounds_cpu.py.)"""
import math
import random

import pytest
import torch

import helpers
from attention_on_gpu import cache, definition, run, tiles, warps
from decoder_reference import attention_bounds

pytestmark = pytest.mark.gpu

HEADS = [
    # D, Dv, Hq, Hk: head sizes up to 64, 96, 128 and 256, up to 8 heads to a key head and more
    (64, 64, 32, 8),
    (48, 40, 96, 8),
    (80, 72, 40, 8),
    (96, 96, 96, 6),
    (128, 128, 32, 8),
    (128, 104, 72, 8),
    (256, 160, 24, 8),
    (192, 256, 40, 4),
]
LENGTHS = {
    # items of many tiles, cut between warps and CTAs; the same seen through a window; items of a few tiles
    "long": (48, 300, 6000, 24, 0),
    "window": (64, 1, 5000, 16, 2477),
    "short": (1100, 0, 160, 7, 0),
}


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", list(LENGTHS))
@pytest.mark.parametrize("heads", HEADS)
def test_many_tiles_to_a_warp(api, handle, heads, kind, dtype):
    D, Dv, Hq, Hk = heads
    N, shortest, longest, S, window = LENGTHS[kind]
    rng = random.Random(11)
    lengths = [rng.randint(shortest, longest) for _ in range(N)]
    assert tiles(lengths, window, Hk) > 12 * warps()              # the ring has at most six stages
    x = cache(5, N, Hq, Hk, D, Dv, S, lengths, dtype, window)
    scale = 1 / math.sqrt(D)
    want = definition(*x, scale, window)
    o, lse, flags = run(api, handle, *x, scale, window)
    bo, bl = attention_bounds(*want, D, dtype)
    assert flags == 0
    assert ((o.double() - want[0]).abs() <= bo).all()
    empty = torch.isinf(want[1])
    assert torch.equal(lse == -math.inf, empty)
    assert ((lse.double() - want[1]).abs() <= bl)[~empty].all()
    if dtype == torch.float32:
        before = torch.backends.cuda.matmul.allow_tf32
        torch.backends.cuda.matmul.allow_tf32 = False
        plain = definition(*x, scale, window, dtype=torch.float32)
        torch.backends.cuda.matmul.allow_tf32 = before
        for got, other, ref in ((o, plain[0], want[0]), (lse, plain[1], want[1])):
            there = torch.isfinite(ref)
            size = ref[there].norm()
            error, theirs = ((y.double() - ref)[there].norm() / size for y in (got, other))
            assert error <= 1.5 * theirs + 2.0 ** -24, (float(error), float(theirs))
    again, lse_again, _ = run(api, handle, *x, scale, window)
    assert torch.equal(o.view(torch.uint8), again.view(torch.uint8)) and torch.equal(lse.view(torch.int32), lse_again.view(torch.int32))
