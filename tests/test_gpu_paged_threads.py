"""Host threads that call attention at once on one cache (MI355X)."""
from __future__ import annotations

import threading

import pytest
import torch

from test_gpu_paged import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


@pytest.mark.parametrize("reqs", [[(1, 6000), (1, 5000)], [(70, 2600)]])
@pytest.mark.parametrize("shared", [True, False])
def test_threads_on_one_cache(P, reqs, shared):
    """Four threads, each with queries of its own, on one stream or on one each: as one after another."""
    c = Case(P, "bf16", 2, 4, 128, 16, reqs, seed=24)
    off, ctx, table = c.off.cuda(), c.ctx.cuda(), c.table.cuda()
    qs = [torch.randn(c.q.shape, device="cuda").bfloat16() for _ in range(4)]
    wants = [c.cache.attend(0, q, off, ctx, table) for q in qs]
    torch.cuda.synchronize()
    streams = [None if shared else torch.cuda.Stream() for _ in qs]
    outs, start = [[] for _ in qs], threading.Barrier(len(qs))

    def work(i):
        start.wait()
        for _ in range(50):
            outs[i].append(c.cache.attend(0, qs[i], off, ctx, table, stream=streams[i]))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(qs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for got, want in zip(outs, wants):
        assert len(got) == 50 and all(torch.equal(o, want) for o in got)
