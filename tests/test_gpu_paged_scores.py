"""Attention where scores, or sums of values, are as large as their types allow (MI355X)."""
from __future__ import annotations

import math

import pytest
import torch

from test_gpu_paged import DTYPE

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


SIZES = [2.0 ** 21, 2.0 ** 25, 1.5e9, 2.0 ** 60, 3.3e38]  # the last two are past fp16's products


@pytest.mark.parametrize("kind,size", [(k, x) for x in SIZES for k in ("bf16", "fp16", "mxfp4")
                                       if k != "fp16" or x < 2e9])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,past", [(1, 40), (1, 3000), (90, 10), (40, 2100)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_far_from_zero(P, kind, dim, n, past, size, sign):
    """Scores of `size` in powers of two, where a float's steps are larger than the differences that
    matter to an exponential. Only a key's first dimension is not zero, so that a score is one exact
    product, and those that are not equal are hundreds apart: a row's output is the mean of the
    values of its largest score's keys, its logarithm that score."""
    page, scale = 16, 0.95
    size /= 1.3706  # scale in powers of two
    g = torch.Generator().manual_seed(n + past)
    rows = -(-(past + n) // page) * page
    top = min(math.sqrt(size), 2.0 ** 15)  # of a key; the query has the rest
    k, v = torch.zeros((rows, 1, dim)), torch.randn((rows, 1, dim), generator=g)
    k[:, 0, 0] = -sign * (0.93 + 0.05 * torch.rand(rows, generator=g)) * top
    q = torch.zeros((n, 4, dim))
    q[..., 0] = -size / top * torch.tensor([0.5, 0.71, 0.9, 1.0])
    q = q.to(DTYPE[kind])
    cache = P.PagedCache(1, 1, dim, rows // page, page, kind)
    slots = torch.arange(rows, device="cuda")
    cache.append(0, k.to(DTYPE[kind]).cuda(), v.to(DTYPE[kind]).cuda(), slots)
    k, v = (x.double().cpu() for x in cache.read(0, slots))
    out, lse = cache.attend(0, q.cuda(), torch.tensor([0, n], device="cuda"),
                            torch.tensor([past], dtype=torch.int32, device="cuda"),
                            torch.arange(rows // page, dtype=torch.int32, device="cuda")[None], scale=scale, lse=True)
    score = q.double()[..., :1] * k[:, 0, 0] * scale
    hidden = torch.arange(rows) > past + torch.arange(n)[:, None, None]
    score = score.masked_fill(hidden, -math.inf)
    most = score.amax(-1, keepdim=True)
    tied = (score == most).double()
    want = tied @ v[:, 0] / tied.sum(-1, keepdim=True)
    mean = tied @ v[:, 0].abs() / tied.sum(-1, keepdim=True)
    # weights and the output are rounded to the type (their sums in 32 bits by far less); the score
    # to a float at its scaling, and again where it leaves as a logarithm
    u = 2.0 ** -11 if kind == "fp16" else 2.0 ** -8
    assert bool(((out.double().cpu() - want).abs() <= (u + 2.0 ** -16) * mean + u * want.abs() + 2.0 ** -24).all())
    near = most[..., 0] + tied.sum(-1).log()
    assert bool(((lse.double().cpu() - near).abs() <= 2.0 ** -21 * near.abs()).all())


def test_sums_of_the_largest_values(P):
    """2^28 keys, whose values' sum leaves a float unless weights are small: each sixteenth of them
    begins with a page of scores 2^8 below the rest. All values are alike, and so is the output."""
    page, dim, n = 64, 64, 40
    pages = 1 << 22
    cache = P.PagedCache(1, 1, dim, 2, page, "bf16")
    k = torch.zeros((2 * page, 1, dim), dtype=torch.bfloat16, device="cuda")
    k[:page, 0, 0] = 8.0
    value = 1.5 * 2.0 ** 127
    cache.append(0, k, torch.full_like(k, value), torch.arange(2 * page, device="cuda"))
    table = torch.zeros((1, pages), dtype=torch.int32, device="cuda")
    table[0, torch.arange(16) * (pages // 16)] = 1
    q = torch.zeros((n, 1, dim), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    out, lse = cache.attend(0, q, torch.tensor([0, n], device="cuda"),
                            torch.tensor([pages * page - n], dtype=torch.int32, device="cuda"), table,
                            scale=0.6931472, lse=True)
    # the sum of 2^20 equal steps of a part in 32 bits, then the output's rounding
    assert bool(((out.double() / value - 1).abs() <= 2.0 ** -4 + 2.0 ** -8).all())
    want = math.log((pages - 16.0) * page * 2.0 ** 8 + 16.0 * page)
    assert bool(((lse.double() - want).abs() <= 2.0 ** -4).all())
