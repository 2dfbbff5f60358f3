"""Bounded waits of the tree attention that run out: the kernel returns, says so in its outputs and in the flags, and the next call is right."""
import math

import pytest
import torch

import helpers
from decoder_reference import attention_bounds
from layer_reference import check, info, tree_attention
from test_gpu_tree_attention import BF16, F16, Problem, now

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_flags", [True, False])
@pytest.mark.parametrize("limit", [0, 1, 2])
@pytest.mark.parametrize("case", [(40, 8, 2, 64, 16, BF16), (40, 8, 2, 128, 20, F16), (70, 8, 2, 128, 64, BF16)], ids=["0", "1", "2"])
def test_waits_that_run_out(case, limit, with_flags):
    """With a limit of zero every wait gives up at once and no row is complete; with one or two polls that depends on timing: a row is right or NaN as a
    whole.  Many short sequences and a long one: items in one CTA and over several, queries that fill one and two blocks of 128 rows."""
    t, hq, hk, d, page, dtype = case
    api = helpers.api()
    handle = api.Handle()
    lengths = [(37 * i) % 700 for i in range(40)] + [30000]
    p = Problem(len(lengths), t, hq, hk, d, d, page, lengths, dtype, seed=t).gpu()
    o, lse = torch.zeros(len(lengths), t, hq, d, dtype=dtype, device="cuda"), torch.zeros(len(lengths), t, hq, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    op = api.TreeAttention(handle, *(info(api, handle, x) for x in (p.cq, p.ck, p.cv, p.ctable, p.cmasks, o)))
    ws = torch.full((op.workspace_size(),), 255, dtype=torch.uint8, device="cuda")
    want = tree_attention(p.cq, p.ck, p.cv, p.table, p.lengths, p.sees, d ** -0.5, 0)
    bo, bl = attention_bounds(*want, d, dtype)

    def run():
        o.fill_(7.0)
        lse.fill_(7.0)
        op.execute(now(), p.cq.data_ptr(), p.ck.data_ptr(), p.cv.data_ptr(), p.ctable.data_ptr(), p.clengths.data_ptr(), p.cmasks.data_ptr(), o.data_ptr(),
                   lse=lse.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel(), flags=flags.data_ptr() if with_flags else 0)
        torch.cuda.synchronize()

    for _ in range(3):
        op.set_attr(api.ATTR_POLL_LIMIT, limit)
        run()
        lost = torch.isnan(lse).cpu()
        assert torch.equal(torch.isnan(o).any(-1).cpu(), lost) and torch.equal(torch.isnan(o).all(-1).cpu(), lost)
        assert limit > 0 or lost.all()
        if with_flags:
            assert flags.item() == (api.FLAG_TIMEOUT if lost.any() else 0)
        check(torch.where(lost[..., None], 0.0, o.cpu()).to(dtype), torch.where(lost[..., None], 0.0, want[0]), bo)
        check(torch.where(lost, 0.0, lse.cpu()), torch.where(lost, 0.0, want[1]), bl)
        flags.zero_()
        op.set_attr(api.ATTR_POLL_LIMIT, 1 << 22)
        run()
        check(o, want[0], bo)
        check(lse, want[1], bl)
        assert flags.item() == 0
