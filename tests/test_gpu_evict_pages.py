"""Eviction to other pages as a program runs it: planes past 32 bits, streams, graphs (MI355X). What moves is compared
with the same eviction of a small cache, or of a copy."""
from __future__ import annotations

import pytest
import torch

from test_gpu_weights import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows_of(cache, slots):
    return [x.clone() for x in cache.read(0, slots)]


# latent rows, 16 bits and 4 bits: planes of 4.8, 4.6 and 2.6 GB
BIG = [("bf16", None, 512, 260000), ("bf16", 8, 128, 140000), ("mxfp4", 8, 128, 300000)]


@pytest.mark.parametrize("kind,heads,dim,far", BIG)
@pytest.mark.parametrize("swap", [False, True])
def test_planes_past_32_bits(P, kind, heads, dim, far, swap):
    """Pages at both ends of a plane, and what is kept to others at both ends: the same bytes as in a small cache."""
    used, page = 90, 16
    small = make(P, kind, heads, dim, used, page, 3)
    big = P.LatentCache(1, dim, 64, far, kind=kind) if heads is None else P.PagedCache(1, heads, dim, far, kind=kind)
    where = torch.arange(used)
    where[swap::2] = far - 1 - where[swap::2]
    slots = torch.arange(used * page, device="cuda")
    big_slots = (where[:, None] * page + torch.arange(page)).view(-1).cuda()
    # the same bytes, block by block
    a, b = (c.data.view(2, n, -1) for c, n in ((small, used), (big, far)))
    for plane in range(2):
        b[plane, where.cuda()] = a[plane]
    order = torch.randperm(used, generator=torch.Generator().manual_seed(1))
    table, to = order[:60].view(2, 30), order[60:].view(2, 15)
    to = torch.cat((to, torch.full((2, 15), -1)), 1)
    big_table, big_to = where[table], torch.where(to >= 0, where[to.clamp(min=0)], to)
    w = small.weights().uniform_(generator=torch.Generator(device="cuda").manual_seed(4))
    big_w = big.weights()
    big_w[0, where.cuda()] = w[0]
    length, keep = i32([471, 302]), i32([200, 77])
    got = small.evict(w, length, table.int().cuda(), keep, 200, recent=16, to=to.int().cuda())
    big_got = big.evict(big_w, length, big_table.int().cuda(), keep, 200, recent=16, to=big_to.int().cuda())
    assert got.tolist() == big_got.tolist() == [200, 77]
    assert torch.equal(big_w[0, where.cuda()], w[0])
    for plane in range(2):
        assert torch.equal(b[plane, where.cuda()], a[plane])
    for x, y in zip(rows_of(small, slots), rows_of(big, big_slots)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


SHAPES = [("bf16", None, 512), ("fp16", 2, 64), ("mxfp4", 2, 128)]


class Case:
    def __init__(self, P, kind, heads, dim):
        self.blocks = 150
        self.cache = make(P, kind, heads, dim, self.blocks, 16, 5, layers=2)
        g = torch.Generator(device="cuda").manual_seed(6)
        self.weights = self.cache.weights().uniform_(generator=g)
        order = torch.randperm(self.blocks, device="cuda", generator=g, dtype=torch.int32)
        self.table, self.to = order[:100].view(2, 50), order[100:150].view(2, 25)
        self.to = torch.cat((self.to, torch.full_like(self.to, -1)), 1)
        self.length, self.keep = i32([790, 333]), i32([395, 40])
        self.data, self.start = self.cache.data.clone(), self.weights.clone()
        torch.cuda.synchronize()

    def again(self):
        self.cache.data.copy_(self.data)
        self.weights.copy_(self.start)

    def evict(self, **kw):
        return self.cache.evict(self.weights, self.length, self.table, self.keep, 400, recent=9, to=self.to, **kw)


@pytest.mark.parametrize("kind,heads,dim", SHAPES)
@pytest.mark.parametrize("raw", [False, True])
def test_on_another_stream(P, kind, heads, dim, raw):
    c = Case(P, kind, heads, dim)
    want = c.evict()
    data, weights = c.cache.data.clone(), c.weights.clone()
    assert not torch.equal(data, c.data)
    c.again()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = c.evict(stream=s.cuda_stream if raw else s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(c.weights, weights) and torch.equal(c.cache.data, data)


@pytest.mark.parametrize("kind,heads,dim", SHAPES)
def test_in_a_graph(P, kind, heads, dim):
    """Captured as the first call of its cache, replayed on other lengths and weights, with eager work between."""
    c, d = Case(P, kind, heads, dim), Case(P, kind, heads, dim)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.evict()
    g = torch.Generator(device="cuda").manual_seed(7)
    for length, keep in ([790, 333], [395, 40]), ([800, 1], [400, 1]), ([16, 700], [0, 399]), ([790, 333], [395, 40]):
        for x in (c, d):
            x.again()
        c.weights.uniform_(generator=g)
        d.weights.copy_(c.weights)
        for x in (c, d):
            x.length.copy_(i32(length))
            x.keep.copy_(i32(keep))
        graph.replay()
        torch.cuda.synchronize()
        want = d.evict()
        assert got.tolist() == want.tolist() == [min(a, b) for a, b in zip(length, keep)]
        assert torch.equal(c.weights, d.weights) and torch.equal(c.cache.data, d.cache.data)
