"""What the bounds of the tree attention's tests can see: mistakes planted in an emulation of the 16-bit kernels' numbers, on the CPU."""
import math

import pytest
import torch

from decoder_reference import attention_bounds
from layer_reference import random_trees, tree_attention

TOKENS = 128


def emulated(q, k, v, lengths, sees, parts=2, late=False, window=0, edge=0):
    """The tcgen05 kernel's steps for one sequence after the other (page n holds sequence n): tiles of 128 tokens, probabilities in `parts` 16-bit
    parts, sums in fp32.  late: a tile's probabilities are taken against the maximum of the next tile; edge: the window moved by so many."""
    n, t, hq, d = q.shape
    hk, dtype, factor = k.shape[2], q.dtype, 1024.0 if q.dtype == torch.float16 else 1.0
    o = torch.zeros(n, t, hq, v.shape[-1])
    for s in range(n):
        end = lengths[s] + t
        at = torch.arange(end)
        drafts = sees[s].sum(-1, keepdim=True)
        visible = (at[None, :] < lengths[s]) & (drafts > 0)
        if window:
            visible &= at[None, :] >= lengths[s] + drafts - window + edge
        visible[:, lengths[s]:] = sees[s]
        for h in range(hq):
            score = (q[s, :, h].float() @ k[s, :end, h // (hq // hk)].float().T) * (d ** -0.5 / math.log(2.0))
            score = score.masked_fill(~visible, -math.inf)
            tiles = [score[:, a:a + TOKENS] for a in range(0, end, TOKENS)]
            tops = torch.stack([x.amax(-1) for x in tiles], -1).cummax(-1).values.clamp(min=-1e30)
            out, total = torch.zeros(t, v.shape[-1]), torch.zeros(t)
            for j, x in enumerate(tiles):
                scale = torch.exp2(tops[:, j - 1] - tops[:, j]) if j else torch.zeros(t)
                p = torch.exp2(x - tops[:, j, None]) * factor
                seen = torch.exp2(x - tops[:, min(j + 1, len(tiles) - 1), None]) * factor if late else p
                high = seen.to(dtype)
                low = (seen - high.float()).to(dtype).float() if parts == 2 else 0.0
                f = (high.float() + low) @ v[s, j * TOKENS:min(end, (j + 1) * TOKENS), h // (hq // hk)].float()
                out, total = out * scale[:, None] + f, total * scale + p.sum(-1)
            o[s, :, h] = torch.where(total[:, None] > 0, out / total[:, None].clamp(min=1e-30), 0.0)
    return o.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_planted_mistakes(dtype):
    n, t, hq, hk, d, window = 3, 40, 4, 2, 64, 150
    lengths = [30, 110, 300]
    g = torch.Generator().manual_seed(3)
    q = (1.5 * torch.randn(n, t, hq, d, generator=g)).to(dtype)
    k, v = (torch.randn(n, 512, hk, d, generator=g).to(dtype) for _ in range(2))
    sees = random_trees(n, t, 5, unused=7)
    table = torch.arange(n, dtype=torch.int32)[:, None]

    def beyond(got, w):
        want = tree_attention(q, k, v, table, lengths, sees, d ** -0.5, w)
        return int(((got.double() - want[0]).abs() > attention_bounds(*want, d, dtype)[0]).sum())

    for w in (0, window):
        assert beyond(emulated(q, k, v, lengths, sees, window=w), w) == 0
        assert beyond(emulated(q, k, v, lengths, sees, window=w, parts=1), w) > 0
        assert beyond(emulated(q, k, v, lengths, sees, window=w, late=True), w) > 0
    for edge in (1, -1):
        assert beyond(emulated(q, k, v, lengths, sees, window=window, edge=edge), window) > 0
