"""Latent caches' operators in 64 bits, plain and slow (what the tests compare with)."""
from __future__ import annotations

import math

import torch

from paged_ref import bounds  # noqa: F401  (sums of `dim` products and 16-bit weights, as there)


def keys_of(r, offsets, context, table, page, cache_blocks):
    """Request r's keys: their positions, blocks and slots, those that are there."""
    new, past = int(offsets[r + 1] - offsets[r]), int(context[r])
    end = max(0, min(past + new, table.shape[1] * page))
    pos = torch.arange(end)
    block = table[r].long()[pos // page] if end else pos
    there = (block >= 0) & (block < cache_blocks)
    return pos[there], block[there], (pos % page)[there]


def attention(q, rows, offsets, context, table, page, scale, k_of=None, v_of=None):
    """q [n, heads, dim] float64 (CPU); rows [blocks, page, dim] float64. k_of(rows, h) and v_of(rows, h) give
    a head's keys and values (None: the rows themselves, their first dim - 64 values). Returns out, lse
    and, for bounds, mean = sum w |v| / sum w and reach = max |q| . |k| * scale over the seen keys."""
    n, heads, _ = q.shape
    k_of = k_of or (lambda x, h: x)
    v_of = v_of or (lambda x, h: x[:, :-64])
    size = v_of(rows[0, :1], 0).shape[-1]
    out = torch.zeros((n, heads, size), dtype=torch.float64)
    mean = torch.zeros_like(out)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64)
    reach = torch.zeros((n, heads), dtype=torch.float64)
    for r in range(len(offsets) - 1):
        a, b, past = int(offsets[r]), int(offsets[r + 1]), int(context[r])
        pos, block, slot = keys_of(r, offsets, context, table, page, rows.shape[0])
        if b <= a or not len(pos):
            continue
        x = rows[block, slot]
        for h in range(heads):
            k, v = k_of(x, h), v_of(x, h)
            for i in range(a, b):
                seen = pos <= past + i - a
                if not bool(seen.any()):
                    continue
                kk, vv = k[seen], v[seen]
                s = (kk @ q[i, h]) * scale
                if bool((s == -math.inf).all()):
                    continue
                top = s.max()
                w = torch.exp(s - top)
                out[i, h] = w @ vv / w.sum()
                mean[i, h] = w @ vv.abs() / w.sum()
                lse[i, h] = top + torch.log(w.sum())
                reach[i, h] = ((kk.abs() @ q[i, h].abs()) * scale).max()
    return out, lse, mean, reach


def batch(seed, new, past, page, spare=3, hole=False):
    """Offsets, context and a page table for requests of `new` tokens behind `past`, and how many blocks the
    cache has. hole: an entry of the longest request is -1, another past the cache."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-(a + b) // page) for a, b in zip(new, past)]
    blocks = sum(need) + spare
    ids = torch.randperm(blocks, generator=g, dtype=torch.int32)
    table = torch.full((len(new), max(1, max(need)) + 1), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    if hole:
        r = max(range(len(new)), key=lambda i: need[i])
        table[r, need[r] // 2] = -1
        table[r, 0] = blocks + 5
    offsets = torch.zeros(len(new) + 1, dtype=torch.int64)
    offsets[1:] = torch.tensor(new).cumsum(0)
    return offsets, torch.tensor(past, dtype=torch.int32), table, blocks
