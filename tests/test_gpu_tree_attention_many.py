"""Trees of many sequences: several items to a thread block, items that begin in one and end in another, next to sequences out of use."""
import pytest
import torch

import helpers
from layer_reference import random_trees
from test_gpu_tree_attention import BF16, F16, F32, Problem, compare, run

pytestmark = pytest.mark.gpu

CASES = [
    # sequences, t, hq, hk, d, dv, page, shortest, longest, window
    (60, 33, 16, 8, 128, 128, 16, 1, 900, 0),
    (60, 40, 16, 8, 64, 64, 16, 1, 900, 300),
    (90, 64, 8, 4, 128, 64, 24, 100, 400, 0),
    (50, 128, 12, 4, 64, 64, 64, 1, 700, 0),
    (70, 50, 12, 2, 96, 128, 8, 1, 600, 129),
    (120, 17, 8, 8, 128, 128, 128, 1, 500, 0),
    (100, 5, 8, 2, 64, 64, 16, 1, 900, 0),
    (40, 20, 8, 2, 200, 256, 16, 1, 500, 64),
    (30, 9, 40, 2, 64, 64, 16, 1, 3000, 0),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_many_sequences(case, dtype):
    n, t, hq, hk, d, dv, page, shortest, longest, window = case
    lengths = [int(shortest * (longest / shortest) ** ((7 * i % n + 0.5) / n)) for i in range(n)]
    sees = random_trees(n, t, t, unused=t // 3)
    sees[5::9] = False                                   # out of use
    sees[4::9] = torch.ones(t, t, dtype=torch.bool).tril()
    p = Problem(n, t, hq, hk, d, dv, page, lengths, dtype, seed=n, sees=sees, heads_first=n % 4 == 0).gpu()
    api = helpers.api()
    handle = api.Handle()
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    o, lse, _ = run(api, handle, p, window=window, flags=flags.data_ptr())
    compare(p, o, lse, window)
    assert flags.item() == 0
    again, _, _ = run(api, handle, p, window=window, lse=False)
    assert torch.equal(o, again)
