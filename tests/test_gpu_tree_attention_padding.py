"""Padded batches: rows that hold no draft need neither pages nor room in the table, and are not reported."""
import math

import pytest
import torch

import helpers
from test_gpu_tree_attention import BF16, F16, F32, Problem, compare, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("t,hq", [(4, 8), (40, 8), (40, 24)])
def test_rows_without_a_draft_need_no_pages(t, hq, dtype):
    """Sequences with few drafts and pages for no more, one that is not in use, one whose drafts fill the table row; then the same with a draft
    that has no page, and one that has no room."""
    api = helpers.api()
    handle = api.Handle()
    page, used, lengths = 16, [2, 0, 1, 3], [30, 0, 47, 16 * 12 - 3]
    sees = torch.zeros(4, t, t, dtype=torch.bool)
    for n, u in enumerate(used):
        sees[n, :u, :u] = torch.ones(u, u, dtype=torch.bool).tril()
    p = Problem(4, t, hq, 2, 64, 64, page, lengths, dtype, seed=5, sees=sees, columns=12)
    for n, u in enumerate(used):
        p.table[n, -(-(lengths[n] + u) // page):] = -1
    p.gpu()
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    for window in (0, 60):
        o, lse, _ = run(api, handle, p, window=window, flags=flags.data_ptr())
        compare(p, o, lse, window)
        assert flags.item() == 0
        assert not o[1].any() and (lse[1] == -math.inf).all()
    # a row of sequence 2 sees draft 3, which lies on a page that is not there
    p.sees[2, 0, 3] = True
    p.gpu()
    o, lse, _ = run(api, handle, p, flags=flags.data_ptr())
    compare(p, o, lse)
    assert flags.item() == api.FLAG_BAD_PAGE
    p.sees[2, 0, 3], p.sees[3, 1, 3] = False, True       # draft 3 of sequence 3 lies behind the table row
    p.gpu()
    flags.zero_()
    o, lse, _ = run(api, handle, p, flags=flags.data_ptr())
    compare(p, o, lse)
    assert flags.item() == api.FLAG_BAD_LENGTH
