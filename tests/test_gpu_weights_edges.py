"""Weighing where a call's rows are more than its requests have (MI355X)."""
from __future__ import annotations

import pytest
import torch

import latent_ref as ref
from test_gpu_weights import check_weigh, key_values, make, weigh_ref

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 2, 128, 4), ("fp16", 1, 64, 1), ("mxfp4", 2, 128, 4), ("bf16", None, 512, 16)]


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


@pytest.mark.parametrize("kind,heads,dim,group", KINDS)
@pytest.mark.parametrize("new,past", [([40], [-38]), ([40], [-40]), ([70], [-3]), ([5], [-2]), ([5, 70, 1], [-2, -69, 0]),
                                      ([600, 2], [-590, 300])])
def test_tokens_before_the_first_position(P, kind, heads, dim, group, new, past):
    """Contexts below zero: a request's first tokens see nothing, and what is left of it may be one tile of rows, of
    one request alone, too."""
    check_weigh(P, kind, heads, dim, 16, group, new, past, seed=3)


@pytest.mark.parametrize("kind,heads,dim,group", KINDS)
@pytest.mark.parametrize("begin,new,past", [(0, 1, 50), (0, 2, 300), (3, 1, 0), (0, 45, 9)])
def test_one_request_of_a_padded_batch(P, kind, heads, dim, group, begin, new, past):
    """Rows before and behind a batch's only request belong to none."""
    page, n = 16, 96
    _, context, table, blocks = ref.batch(4, [new], [past], page)
    offsets = torch.tensor([begin, begin + new])
    cache = make(P, kind, heads, dim, blocks, page, 4)
    kv_heads, size = heads or 1, dim if heads else dim + 64
    g = torch.Generator().manual_seed(5)
    q = torch.randn((n, kv_heads * group, size), generator=g).to(cache.dtype)
    lse = 3 + torch.rand((n, kv_heads * group), generator=g)
    before = torch.rand((blocks, kv_heads, page), generator=g)
    d, scale = q.cuda(), size ** -0.5
    got = cache.weigh(0, before.cuda(), *((d,) if heads else (d[..., :dim], d[..., dim:])), lse.cuda(), offsets.cuda(),
                      context.cuda(), table.cuda(), scale=scale)
    want, tol = weigh_ref(before, q, lse, key_values(cache, P, kind, heads, dim, blocks, page), offsets, context, context,
                          table, page, scale)
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol + want.abs() * 2.0 ** -23).all()), float((off / (tol + 1e-30)).max())
