"""Block tables from any place of the free list, in it and far outside (MI355X)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu

MOST = (1 << 63) - 1


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


@pytest.mark.parametrize("R", [1, 5, 1500])
@pytest.mark.parametrize("n_free", [0, 1, 4, 900])
@pytest.mark.parametrize("first", [MOST, MOST - 1, MOST - 2000, 1 << 62, 1 << 32, 905, 900, 899, 4, 1, -1, -MOST - 1])
def test_first_outside_the_free_list(P, R, n_free, first):
    """No entry outside the list is read or given: behind its end, near the largest number, negative
    (which counts as 0). The list lies between other blocks, which would show."""
    page = 16
    new, past = (np.arange(R) * 7) % 40, (np.arange(R) * 5) % 33
    off = np.zeros(R + 1, dtype=np.int64)
    off[1:] = np.cumsum(new)
    held = -(-past // page)
    table = np.full((R, 6), -7, dtype=np.int32)
    for r in range(R):
        table[r, :held[r]] = 5000 + np.arange(held[r])
    around = torch.full((2000 + n_free + 2000,), 77777, dtype=torch.int32, device="cuda")
    around[2000:2000 + n_free] = torch.arange(n_free, device="cuda") + 100
    free = around[2000:2000 + n_free]
    want = ref.tables(off, past, held, table, page, free.cpu().numpy(), max(first, 0))
    cache = P.PagedCache(1, 1, 64, 0, block_tokens=page)
    dev = lambda x, t: torch.from_numpy(x.astype(t)).cuda()  # noqa: E731
    t = dev(table, np.int32)
    slots, pos, after, nxt = cache.tables(dev(off, np.int64), dev(past, np.int32), t, free, int(off[-1]),
                                          held=dev(held, np.int32),
                                          first=torch.tensor([first], dtype=torch.int64, device="cuda"))
    for got, w in zip((t, slots, pos, after), want):
        assert np.array_equal(got.cpu().numpy(), w.reshape(got.shape))
    assert int(nxt) == want[4]
