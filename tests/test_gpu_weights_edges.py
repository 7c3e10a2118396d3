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


@pytest.mark.parametrize("kind,heads,dim,group", [("bf16", 2, 128, 4), ("fp16", 1, 64, 32), ("mxfp4", 2, 128, 8),
                                                  ("mxfp4", 1, 64, 1), ("bf16", None, 512, 16), ("fp16", None, 256, 33)])
@pytest.mark.parametrize("new,past", [([1, 1, 3], [300, 0, 777]), ([300], [0]), ([450], [37]), ([260, 1, 90, 515], [0, 500, 129, 255]),
                                      ([40, 9], [-30, -3])])
def test_no_weight_is_lost(P, kind, heads, dim, group, new, past):
    """Keys and queries of -1, 0 and 1, and a scale that is a power of two: scores are exact. What a request's rows give
    to its keys then sums to the number of those that see any, and each key's weight is that of 64 bits but
    for what the exponentials and the sums of this attention and this weighing are off by. In powers of two: a
    product's rounding half a step below 2^6, 2^-19, the same for a maximum and a logarithm of that size, three
    roundings of half that for the log sums and their difference from a score, together 9 * 2^-20, which is
    2^-17.5 of a weight; 2^-22 for an exponential and its rounding, twice; and 2^-24 for each term of a sum: of all
    keys for the log sum, and here of 64 rows, sums of these and shares, fewer than 256."""
    page = 16
    offsets, context, table, blocks = ref.batch(6, new, past, page)
    cache = make(P, kind, heads, dim, blocks, page, 6)
    kv_heads, size = heads or 1, dim if heads else dim + 64
    g = torch.Generator().manual_seed(7)
    k = torch.randint(-1, 2, (blocks * page, kv_heads, size), generator=g).to(cache.dtype)
    n = int(offsets[-1])
    q = torch.randint(-1, 2, (n, kv_heads * group, size), generator=g).to(cache.dtype)
    slots, d, scale = torch.arange(blocks * page, device="cuda"), q.cuda(), 2.0 ** -3 if heads else 2.0 ** -4
    batch = (offsets.cuda(), context.cuda(), table.cuda())
    if heads:
        cache.append(0, k.cuda(), torch.zeros_like(k).cuda(), slots)
        args = (d,)
    else:
        cache.append(0, k[:, 0, :dim].cuda(), k[:, 0, dim:].cuda(), slots)
        args = (d[..., :dim], d[..., dim:])
    _, lse = cache.attend(0, *args, *batch, scale=scale, lse=True)
    got = cache.weigh(0, torch.full((blocks, kv_heads, page), 5.0, device="cuda"), *args, lse, *batch, scale=scale,
                      weighed=torch.zeros(len(new), dtype=torch.int32, device="cuda")).cpu().double()
    sees = (lse > -torch.inf).cpu()
    keys = k.view(blocks, page, kv_heads, size).double()
    for r in range(len(new)):
        a, b = int(offsets[r]), int(offsets[r + 1])
        pos, block, slot = ref.keys_of(r, offsets, context, table, page, blocks)
        rows = sees[a:b].view(b - a, kv_heads, group).sum((0, 2))
        assert rows.tolist() == [group * min(b - a, max(0, int(context[r]) + b - a))] * kv_heads
        tol = (len(pos) + 256) * 2.0 ** -24 + 2.0 ** -17.5 + 2.0 ** -21
        sums = got[block, :, slot].sum(0)
        assert bool(((sums - rows).abs() <= rows * tol).all()), (sums, rows)
        for h in range(kv_heads):
            s = torch.matmul(q[a:b, h * group:(h + 1) * group].double(), keys[block, slot, h].T) * scale
            s = s.masked_fill((pos > int(context[r]) + torch.arange(b - a)[:, None])[:, None], -torch.inf)
            w = torch.softmax(s, -1).nan_to_num(0.0).sum((0, 1))
            off = (got[block, h, slot] - w).abs()
            assert bool((off <= w * tol).all()), float((off / w).max() / tol)
