"""Pools larger than a CTA's threads cover in one round (8 CTAs of 1024 threads with four pages each: 32768 pages), against the
step-by-step Python model: just below that size, just above it, and several rounds."""
import random

import pytest
import torch

import helpers
from test_gpu_pages import Machine

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.fixture(scope="module")
def handle(api):
    return api.Handle()


def occupied(api, handle, P, N, S, share, seed, refs_offset=0):
    """A machine whose pool is in use to `share`, its pages spread over all of it: rows of scattered pages, full ones."""
    rng = random.Random(seed)
    each = int(P * share) // N
    pool = torch.arange(P, dtype=torch.int32, device="cuda").view(P, 1).repeat(1, 4)
    m = Machine(api, handle, N, each + 12, P, S, pools=[pool], refs_offset=refs_offset)
    pages = rng.sample(range(P), each * N)
    for n in range(N):
        row = pages[n * each:(n + 1) * each]
        m.model.table[n][:each] = row
        m.model.lengths[n] = each * S
        for p in row:
            m.model.refs[p] = 1
    m.table.copy_(torch.tensor(m.model.table, dtype=torch.int32))
    m.lengths.copy_(torch.tensor(m.model.lengths, dtype=torch.int32))
    m.refs.copy_(torch.tensor(m.model.refs, dtype=torch.int32))
    m.same()
    return m, rng


@pytest.mark.parametrize("P", [32768, 32769, 32771, 36001, 140011, 300007])
@pytest.mark.parametrize("share", [0.03, 0.5, 0.98])
def test_pools_of_several_rounds(api, handle, P, share):
    N, S = 60, 4
    m, rng = occupied(api, handle, P, N, S, share, P, refs_offset=P % 3)
    m.extend([rng.randint(0, 3) for _ in range(N)], 3)                 # few pages: the first rounds have them
    m.free(rng.sample(range(N), 7))
    empty = [n for n in range(N) if m.model.lengths[n] == 0]
    full = [n for n in range(N) if m.model.lengths[n] > 0]
    m.fork(rng.sample(full, 4), empty[:4])
    m.extend([1] * N, 1)                                               # shared last pages are copied
    most = 9 * S
    m.extend([rng.randint(0, most) for _ in range(N)], most)
    assert len(m.compact()) > 0
    m.extend([rng.randint(0, S) for _ in range(N)], S)
    m.free(rng.sample(range(N), 20))
    assert len(m.compact()) > 0
    assert m.flags.item() & ~(api.FLAG_POOL_EXHAUSTED | api.FLAG_BAD_LENGTH) == 0


@pytest.mark.parametrize("P", [32767, 32769, 140011])
def test_last_free_pages_of_a_large_pool(api, handle, P):
    """A pool that runs out within a call, and one that is used to the last page."""
    N, S = 11, 4
    m, rng = occupied(api, handle, P, N, S, 0.9, 2 * P)
    left = m.model.refs.count(0)
    used = 0
    while left >= N:
        n = min(12, left // N)
        if any(m.model.lengths[s] + n * S > m.model.columns * S for s in range(N)):
            break
        m.extend([n * S] * N, n * S)
        left -= n * N
        used += n
    assert used > 0
    # a wide call against what is left: a prefix of the sequences gets pages
    extra = Machine(api, handle, 4, P, P, S, pools=m.pools)
    extra.table[0].copy_(torch.arange(P, dtype=torch.int32))
    extra.table[0, P - 3000:] = -1
    extra.lengths[0] = (P - 3000) * S
    extra.refs[:P - 3000] = 1
    extra.model.table[0][:P - 3000] = list(range(P - 3000))
    extra.model.lengths[0] = (P - 3000) * S
    extra.model.refs[:P - 3000] = [1] * (P - 3000)
    extra.extend([0, 2000 * S, 1001 * S, 0], 2000 * S)
    assert extra.flags.item() == api.FLAG_POOL_EXHAUSTED
    extra.extend([0, 0, 1000 * S, 0], 1000 * S)
    assert extra.model.refs.count(0) == 0
    extra.extend([0, 0, 0, 1], 1)
    extra.free([0])
    assert len(extra.compact()) == 3000
    assert extra.flags.item() == api.FLAG_POOL_EXHAUSTED
