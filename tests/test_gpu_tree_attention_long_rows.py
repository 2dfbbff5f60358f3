"""Table rows of 2^31 tokens (one page over and over): the last tokens that count, and lengths beyond them."""
import math

import pytest
import torch

import helpers
from decoder_reference import attention_bounds
from layer_reference import check, info, mask_words, tree_attention
from test_gpu_tree_attention import BF16, F16, F32, now

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,t,hq", [(BF16, 20, 4), (F16, 70, 4), (BF16, 3, 2), (F32, 20, 2)])
def test_the_last_tokens_of_a_row(dtype, t, hq):
    api = helpers.api()
    handle = api.Handle()
    page, d, window, room = 1 << 24, 8, 90, (1 << 31) - 256
    g = torch.Generator(device="cuda").manual_seed(t)
    k, v = (torch.randn(1, page, 1, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.zeros(4, 128, dtype=torch.int32, device="cuda")
    # drafts that just fit, drafts of which three fit, a length beyond what counts, and the largest
    lengths = [room - t, room - 3 + (t <= 3), room + 7, (1 << 31) - 1]
    sees = torch.ones(4, t, t, dtype=torch.bool).tril()
    q = torch.randn(4, t, hq, d, generator=g, device="cuda").to(dtype)
    masks, o = mask_words(sees).cuda(), torch.full((4, t, hq, d), math.nan, dtype=dtype, device="cuda")
    lse, flags = torch.full((4, t, hq), math.nan, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    op = api.TreeAttention(handle, *(info(api, handle, x) for x in (q, k, v, table, masks, o)), window=window)
    ws = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")

    def run(counted):
        n = torch.tensor(counted, dtype=torch.int32, device="cuda")
        flags.zero_()
        op.execute(now(), q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(), n.data_ptr(), masks.data_ptr(), o.data_ptr(), lse=lse.data_ptr(),
                   workspace=ws.data_ptr(), workspace_bytes=ws.numel(), flags=flags.data_ptr())
        # the last 512 tokens that count as a cache of their own
        first = room - 512
        at = (torch.arange(first, room, device="cuda") % page)
        small = (k[:, at], v[:, at])
        want = tree_attention(q, *small, torch.zeros(4, 1, dtype=torch.int32), [min(x, room) - first for x in counted], sees, d ** -0.5, window)
        bo, bl = attention_bounds(*want, d, dtype)
        check(o, want[0], bo)
        check(lse, want[1], bl)
        return flags.item()

    assert run(lengths) == api.FLAG_BAD_LENGTH
    assert run([room - t, room - t - 1, room - t - 130, room - 400]) == 0
