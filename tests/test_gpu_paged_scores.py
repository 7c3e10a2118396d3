"""Attention where scores are as large as their types allow (MI355X)."""
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


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,past", [(1, 40), (1, 3000), (90, 10), (40, 2100)])
@pytest.mark.parametrize("size", [2.0 ** 21, 2.0 ** 25, 1.5e9, 2.0 ** 60, 3.3e38])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_far_from_zero(P, kind, dim, n, past, size, sign):
    """Scores of `size` in powers of two, where a float's steps are larger than the differences that
    matter to an exponential. Only a key's first dimension is not zero, so that a score is one exact
    product, and those that are not equal are hundreds apart: a row's output is the mean of the
    values of its largest score's keys, its logarithm that score."""
    if kind == "fp16" and size > 2e9:
        pytest.skip("past the products of fp16 values")
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
