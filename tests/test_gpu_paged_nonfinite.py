"""Attention over keys and values that are not finite, where a row's keys are cut into parts (MI355X).

A score that is NaN, and a value that is not finite, count wherever a row sees them: which part
of its keys they fall into, and how little that part weighs beside the others, changes nothing.
"""
from __future__ import annotations

import pytest
import torch

from test_gpu_paged import DTYPE

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


def attend(P, kind, dim, n, past, edit, seed=0, group=4, width=None):
    """One request, n tokens behind `past` keys of one head; `edit` changes (q, k, v) first. Returns
    the output and the logarithms of the sums."""
    page = 16
    blocks = -(-(past + n) // page)
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((n, group, dim), generator=g)
    k, v = (torch.randn((blocks * page, 1, dim), generator=g) for _ in range(2))
    edit(q, k, v)
    cache = P.PagedCache(1, 1, dim, blocks, page, kind)
    k, v = (x.to(DTYPE[kind]).cuda() for x in (k, v))
    cache.append(0, k, v, torch.arange(blocks * page, device="cuda"))
    table = torch.full((1, width or blocks), -1, dtype=torch.int32)
    table[0, :blocks] = torch.arange(blocks)
    out, lse = cache.attend(0, q.to(DTYPE[kind]).cuda(), torch.tensor([0, n], device="cuda"),
                            torch.tensor([past], dtype=torch.int32, device="cuda"), table.cuda(), lse=True)
    return out.float().cpu(), lse.cpu()


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("past", [100, 2048, 8192])
def test_nan_key_of_the_newest_token(P, kind, dim, past):
    """The only key of its part, or one of a request done whole."""
    def edit(q, k, v):
        k[past] = NAN
    out, lse = attend(P, kind, dim, 1, past, edit)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
@pytest.mark.parametrize("at", [0, 5, 20])
def test_nan_keys_of_a_whole_part(P, kind, at):
    """All keys of a step, hence of a share's part: the first, one in between, the last."""
    step = 256 if kind == "mxfp4" else 128
    past = 21 * step - 1

    def edit(q, k, v):
        k[at * step:(at + 1) * step] = NAN
    out, lse = attend(P, kind, 128, 1, past, edit)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
@pytest.mark.parametrize("dim", [64, 128])
def test_nan_keys_of_a_prompt_s_part(P, kind, dim):
    """All keys of the second of three parts: 34 steps of 64 keys, of which it has 11."""
    def edit(q, k, v):
        k[704:1408] = NAN
    out, lse = attend(P, kind, dim, 40, 2100, edit)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("keys", [(0, 128), (704, 1408), (1000, 1001), (2000, 2048)])
def test_values_of_keys_that_weigh_nothing(P, kind, n, bad, keys):
    """Values that are not finite behind scores 300 below the others: as seen as any."""
    def edit(q, k, v):
        q[..., 0], k[..., 0] = 32.0, 0.0
        k[keys[0]:keys[1], 0, 0] = -75.0
        v[keys[0]:keys[1], 0, 3] = bad
    out, lse = attend(P, kind, 64, n, 2100, edit)
    clean, lse0 = attend(P, kind, 64, n, 2100, lambda q, k, v: (edit(q, k, v), v.nan_to_num_(0.0, 0.0, 0.0)))
    assert not bool(torch.isfinite(out[..., 3]).any())
    keep = [d for d in range(64) if d != 3]
    assert torch.equal(out[..., keep], clean[..., keep]) and torch.equal(lse, lse0)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("past", [300, 2100])
def test_parts_without_keys_count_nothing(P, n, past):
    """A table far wider than the request, whose parts may then have no keys."""
    out, lse = attend(P, "bf16", 64, n, past, lambda q, k, v: None, width=4000)
    near, lse0 = attend(P, "bf16", 64, n, past, lambda q, k, v: None)
    # the same values in another order of sums: a step of bf16 apart at most, 2^-8 of a value below 4
    assert bool(torch.isfinite(out).all())
    assert bool(((out - near).abs() <= 2.0 ** -6).all()) and bool(((lse - lse0).abs() <= 2.0 ** -16).all())
