"""Values that are not finite and that some rows of a tree do not see: they have no influence on those rows, wherever tiles begin and end."""
import math

import pytest
import torch

import helpers
from decoder_reference import attention_bounds
from layer_reference import check, tree_attention
from test_gpu_tree_attention import BF16, F16, F32, Problem, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def place(p, n, position):
    """Page and row of a position of sequence n."""
    return int(p.table[n, position // p.page]), position % p.page


def spoil(p, odd, window=0):
    """Puts the values odd = [(sequence, position, key head, first element, last, value)] into V and returns the problem's own V without them, and
    which outputs see one."""
    n, t, hq, dv = p.q.shape[0], p.t, p.q.shape[2], p.v.shape[-1]
    clean, hit = p.v.clone(), torch.zeros(n, t, hq, dv, dtype=torch.bool)
    group = hq // p.v.shape[2]
    for s, position, head, first, last, value in odd:
        page, row = place(p, s, position)
        p.v[page, row, head, first:last] = value
        drafts = p.sees[s].sum(-1)
        if position >= p.lengths[s]:
            sees = p.sees[s][:, position - p.lengths[s]]
        else:
            sees = (drafts > 0) & ((position >= p.lengths[s] + drafts - window) if window else True)
        hit[s, :, head * group:(head + 1) * group, first:last] |= sees[:, None, None]
    assert not hit.all(-1).all()
    return clean, hit


def compare(p, clean, hit, o, lse, window=0):
    scale = p.q.shape[-1] ** -0.5
    want = tree_attention(p.cq, p.ck, clean.cuda(), p.table, p.lengths, p.sees, scale, window)
    bo, bl = attention_bounds(*want, p.q.shape[-1], p.q.dtype)
    o = o.cpu()
    assert not torch.isfinite(o[hit]).any()              # rows that see one: infinities or NaN
    check(torch.where(hit, 0.0, o).to(o.dtype), torch.where(hit, 0.0, want[0]), bo)
    check(lse, want[1], bl)


ACROSS = [
    # t, hq, hk, d, page, cached tokens of every second sequence (drafts lie in two tiles of 128)
    (64, 4, 2, 64, 16, [100, 90]),
    (64, 2, 2, 128, 16, [100, 330]),
    (20, 4, 2, 128, 20, [120, 250]),
    (80, 8, 2, 64, 16, [100, 60]),
    (128, 4, 4, 128, 32, [100, 5]),
    (5, 4, 2, 64, 16, [125, 254]),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("case", ACROSS, ids=[str(i) for i in range(len(ACROSS))])
def test_draft_in_a_tile_before_the_last(api, handle, case, dtype):
    """The drafts reach into the next tile, where every row has a larger score than before (its own): the rows that do not see the odd draft of the
    first tile weigh its other tokens by the right maximum.  (As many sequences as give a CTA whole ones.)"""
    t, hq, hk, d, page, lengths = case
    lengths = lengths * 45
    p = Problem(len(lengths), t, hq, hk, d, d, page, lengths, dtype, seed=t + d)
    group = hq // hk
    for n, length in enumerate(lengths):
        border = (length // 128 + 1) * 128 - length      # first draft of the next tile
        assert 1 < border < t
        for i in range(border, t):
            where = place(p, n, length + i)
            for h in range(hk):
                q = p.q[n, i, h * group].double()
                # a score of about 6: one and a half above the largest of the others
                p.k[where[0], where[1], h] = (q * (6.0 * d ** 0.5 / (q * q).sum())).to(dtype)
    odd = []
    for n, length in enumerate(lengths):
        p.sees[n, :, 1] = False                          # draft 1 is nobody's, row 1 holds none
        p.sees[n, 1] = False
        odd += [(n, length + 1, 0, 0, d, math.nan), (n, length, hk - 1, 0, d // 2 + 3, math.inf), (n, length, 0, d - 5, d, -math.inf)]
    clean, hit = spoil(p, odd)
    p.gpu()
    o, lse, _ = run(api, handle, p)
    compare(p, clean, hit, o, lse)


EDGE = [
    # t, hq, hk, d, page, cached tokens of every second sequence, window (its edge lies in tiles without drafts)
    (48, 4, 2, 64, 16, [400, 389], 140),
    (64, 8, 2, 128, 16, [400, 700], 160),
    (33, 3, 3, 128, 20, [300, 1111], 100),
    (80, 8, 2, 64, 64, [1000, 530], 300),
    (4, 8, 2, 64, 16, [400, 389], 140),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("case", EDGE, ids=[str(i) for i in range(len(EDGE))])
def test_cached_tokens_at_the_windows_edge(api, handle, case, chain, dtype):
    """Rows that see more drafts begin later in the cache.  A chain: tokens that only its first rows see.  Rows that see every draft: tokens
    at the edge that nobody sees."""
    t, hq, hk, d, page, lengths, window = case
    lengths = lengths * 20
    sees = torch.ones(len(lengths), t, t, dtype=torch.bool)
    p = Problem(len(lengths), t, hq, hk, d, d, page, lengths, dtype, seed=t + d, sees=sees.tril() if chain else sees)
    odd = []
    for n, length in enumerate(lengths):
        first = length + 1 - window                      # what a row that sees one draft begins with
        odd += [(n, first, 0, 0, d, math.nan), (n, first + 2, hk - 1, 3, d // 2, math.inf), (n, first + min(t, 6) - 2, 0, d // 2, d, -math.inf)]
    clean, hit = spoil(p, odd, window)
    assert hit.any() == chain
    p.gpu()
    o, lse, _ = run(api, handle, p, window=window)
    compare(p, clean, hit, o, lse, window)
