"""4-bit slabs written by another program, byte by byte as the header lays them out (MI355X)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


@pytest.mark.parametrize("heads,dim,page", [(1, 64, 1), (3, 64, 7), (2, 128, 16), (1, 128, 33), (8, 128, 16)])
def test_slabs_of_another_program(P, heads, dim, page):
    """Read back, and attended to by few rows and by many, as the values that they stand for."""
    blocks = 5
    rng = np.random.default_rng(page)
    codes = rng.integers(0, 16, (2, blocks, heads, page, dim)).astype(np.uint8)
    power = rng.integers(124, 128, (2, blocks, heads, page, dim // 32)).astype(np.uint8)
    slabs = [ref.pack_slab(codes[i, b], power[i, b], page) for i in range(2) for b in range(blocks)]
    data = torch.from_numpy(np.concatenate(slabs)).cuda()
    cache = P.PagedCache(1, heads, dim, blocks, page, "mxfp4", data=data)
    k, v = (torch.from_numpy(ref.values_of(codes[i], power[i])) for i in range(2))  # [block, head, slot, dim]
    slots = torch.arange(blocks * page, device="cuda")
    for got, x in zip(cache.read(0, slots), (k, v)):
        assert torch.equal(got.double().cpu(), x.transpose(1, 2).reshape(blocks * page, heads, dim))
    table = torch.tensor([[4, 1, 3, 0, 2]], dtype=torch.int32)
    for n in (1, 4 * page):
        past = 5 * page - n
        q = torch.randn((n, 4 * heads, dim), generator=torch.Generator().manual_seed(n)).bfloat16()
        off, ctx = torch.tensor([0, n]), torch.tensor([past], dtype=torch.int32)
        out, lse = cache.attend(0, q.cuda(), off.cuda(), ctx.cuda(), table.cuda(), lse=True)
        o, l, mean, reach = ref.attention(q.double(), lambda b: k[b], lambda b: v[b], off, ctx, table, page, blocks,
                                          dim ** -0.5)
        near_o, near_l = ref.bounds(o, mean, reach, dim, False)
        assert bool(((out.double().cpu() - o).abs() <= near_o).all())
        assert bool(((lse.double().cpu() - l).abs() <= near_l).all())
