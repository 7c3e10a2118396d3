"""Latent attention where a batch is not what it should be, or only partly there (MI355X)."""
from __future__ import annotations

import math

import pytest
import torch

from test_gpu_latent import check, check_expanded
from test_gpu_latent_serving import Batch, i32, i64
from test_gpu_weights import evict_ref

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


@pytest.mark.parametrize("kind,latent,heads,new,past", [
    ("bf16", 512, 16, [5], [-2]), ("fp16", 256, 2, [5, 1], [-2, 40]), ("bf16", 256, 64, [5, 3, 40], [-2, 0, -39]),
    ("fp16", 512, 128, [2, 70, 1], [-1, -5, 300]), ("bf16", 512, 16, [1, 1, 1], [-1, 129, 0])])
def test_absorbed_tokens_before_the_first_position(P, kind, latent, heads, new, past):
    """Contexts below zero: a request's first tokens see nothing, the others the keys from position 0 on."""
    check(P, kind, latent, 16, heads, new, past, seed=heads)


@pytest.mark.parametrize("kind,latent,heads,new,past", [
    ("bf16", 512, 3, [5], [-2]), ("fp16", 256, 4, [40, 3], [-39, 20]), ("bf16", 256, 33, [200, 2, 33], [-70, 0, -33]),
    ("fp16", 512, 65, [300, 1], [-5, 64])])
def test_expanded_tokens_before_the_first_position(P, kind, latent, heads, new, past):
    """The same in tiles of 32 tokens, and of 128 by eight waves and by four."""
    check_expanded(P, kind, latent, 16, heads, new, past, seed=heads)


@pytest.mark.parametrize("heads", [2, 40, 65])
def test_contexts_at_the_ends_of_their_type(P, heads):
    """Far below zero a request sees nothing; far past its pages all that they hold. Eviction gives each the tokens that it
    keeps, and moves nothing of the others."""
    b = Batch(P, [140, 2, 3], [0, 60, 20], heads=heads, seed=9)
    args = (b.args[0], i32([-2 ** 31, 2 ** 31 - 1, -5]), b.args[2])
    out, lse = b.expanded(args=args, lse=True)
    for rows in (slice(0, 140), slice(142, 145)):
        assert not bool(out[rows].any()) and bool((lse[rows] == -math.inf).all())
    want, sums = b.expanded(args=(b.args[0], i32([0, 100, 0]), b.args[2]), lse=True)
    assert torch.equal(out[140:142], want[140:142]) and torch.equal(lse[140:142], sums[140:142])
    weights = b.cache.weights().uniform_(generator=torch.Generator(device="cuda").manual_seed(4))
    before, rows, table = weights.clone(), b.rows.clone(), b.host[2]
    after = b.cache.evict(weights, args[1], args[2], i32([4, 9, 2 ** 31 - 1]), 9)
    assert after.tolist() == [0, 9, 0]
    # the second request's tokens: all slots of its pages, and none where it has no page
    t = torch.arange(table.shape[1] * 16)
    block, slot = table[1].long()[t // 16], t % 16
    w = [float(before[0, x, 0, y]) if x >= 0 else -math.inf for x, y in zip(block.tolist(), slot.tolist())]
    stay = torch.tensor(evict_ref(w, len(w), 9, 0))
    want_rows, want_weights = rows.clone(), before.clone()
    for i, s in enumerate(stay.tolist()):
        want_rows[block[i], slot[i]] = rows[block[s], slot[s]]
        want_weights[0, block[i], 0, slot[i]] = before[0, block[s], 0, slot[s]]
    assert torch.equal(b.rows, want_rows) and torch.equal(weights, want_weights)
