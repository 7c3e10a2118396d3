"""Latent attention where a batch is not what it should be, or only partly there (MI355X)."""
from __future__ import annotations

import math

import pytest
import torch

from test_gpu_latent_serving import Batch, i64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


MOST, LEAST = 2 ** 63 - 1, -2 ** 63


@pytest.mark.parametrize("heads", [2, 40, 65])
@pytest.mark.parametrize("bad,none", [
    ([0, 500, 208], [0, 1]), ([0, -5, 208], [0, 1]), ([0, 1 << 40, 208], [0, 1]), ([7, 185, 100], [1]), ([0, 185, 209], [1]),
    ([185, 185, 208], [0]), ([0, MOST, LEAST], [0, 1]), ([LEAST, MOST, MOST], [0, 1]), ([LEAST, 0, 208], [0]),
    ([MOST, LEAST, 208], [0, 1]), ([0, 0, MOST], [0, 1])])
def test_key_offsets_that_do_not_rise(P, heads, bad, none):
    """Requests whose key offsets do not rise within 0 .. n_keys, or name no key, have none: zeros, and the logarithm of
    nothing. (All kernels: tiles of 32 tokens, of 128 by eight waves and by four.)"""
    b = Batch(P, [140, 3], [45, 20], heads=heads, seed=3)
    assert b.n_keys == 208
    clean, sums = b.expanded(lse=True)
    b.key_offsets = i64(bad)
    got, lse = b.expanded(lse=True)
    rows = (slice(0, 140), slice(140, 143))
    for r in range(2):
        if r in none:
            assert not bool(got[rows[r]].any()) and bool((lse[rows[r]] == -math.inf).all())
    if bad == [7, 185, 100]:  # 178 keys from the seventh place on: all that the first 128 tokens see
        assert torch.equal(got[:128], clean[:128]) and torch.equal(lse[:128], sums[:128])
    if bad == [0, 185, 209]:
        assert torch.equal(got[:140], clean[:140]) and torch.equal(lse[:140], sums[:140])
    if bad == [185, 185, 208]:
        assert torch.equal(got[140:], clean[140:]) and torch.equal(lse[140:], sums[140:])
    if bad == [LEAST, 0, 208]:  # the second request's keys are 208 now: the 23 that it sees begin where its pages do
        assert torch.equal(got[140:], clean[140:]) and torch.equal(lse[140:], sums[140:])
