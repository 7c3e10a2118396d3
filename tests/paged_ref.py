"""The paged cache's operators in 64 bits, plain and slow (what the tests compare with)."""
from __future__ import annotations

import math

import numpy as np
import torch

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
GROUP = 32


def tables(offsets, context, held, table, page, free, first=0):
    """Request by request, block by block. Returns (table, slots, positions, held, next)."""
    shape = np.shape(table)
    table = [list(map(int, row)) for row in table]
    n = int(offsets[-1])
    slots, positions = [-1] * n, [0] * n
    after, at = [], first
    for r, row in enumerate(table):
        new = int(offsets[r + 1] - offsets[r])
        need = min(-(-max(0, int(context[r]) + new) // page), len(row))
        have = int(held[r])
        got = have
        for b in range(have, need):
            if at < len(free):
                row[b] = int(free[at])
                got = b + 1
                at += 1
            else:
                row[b] = -1
        after.append(got)
        for i in range(new):
            t, pos = int(offsets[r]) + i, int(context[r]) + i
            positions[t] = pos
            if 0 <= pos < len(row) * page and row[pos // page] >= 0:
                slots[t] = row[pos // page] * page + pos % page
    return (np.array(table, dtype=np.int32).reshape(shape), np.array(slots, dtype=np.int64),
            np.array(positions, dtype=np.int32), np.array(after, dtype=np.int32), at)


def four_bits(x):
    """x [..., dim] (any float array) -> (codes 0..15 [..., dim], exponent bytes [..., dim/32])."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    codes = np.zeros(g.shape, dtype=np.uint8)
    power = np.zeros(g.shape[:-1], dtype=np.uint8)
    for i in np.ndindex(power.shape):
        most = np.abs(g[i]).max()
        if not np.isfinite(most):
            power[i] = 255
            continue
        e = -126
        while most > 7 * math.ldexp(1.0, e) and e < 125:  # 6 * 2^125 is the largest that bf16 holds
            e += 1
        power[i] = e + 127
        far = np.abs(np.abs(g[i])[:, None] / math.ldexp(1.0, e) - LEVELS)
        near = far.min(1, keepdims=True)
        tied = far == near
        even = tied & (np.arange(8) % 2 == 0)
        code = np.where(tied.sum(1) > 1, even.argmax(1), tied.argmax(1))
        codes[i] = code + 8 * np.signbit(g[i])
    return codes.reshape(x.shape), power


def values_of(codes, power):
    """The values that codes and exponent bytes stand for (255: NaN)."""
    level = np.concatenate([LEVELS, -LEVELS])[codes]
    step = np.where(power == 255, np.nan, np.exp2(power.astype(np.float64) - 127))
    return (level.reshape(*power.shape, GROUP) * step[..., None]).reshape(codes.shape)


def pack_slab(codes, power, page):
    """[heads, page, dim] codes -> the bytes of one 4-bit slab."""
    low, high = codes[..., 0::2], codes[..., 1::2]
    raw = np.concatenate([(low | (high << 4)).astype(np.uint8).ravel(), power.ravel()])
    return np.concatenate([raw, np.zeros(-len(raw) % 16, dtype=np.uint8)])


def attention(q, k_of, v_of, offsets, context, table, page, cache_blocks, scale):
    """q [n, q_heads, dim] float64; k_of(block) -> [heads, page, dim] float64. Returns out, lse and
    `mean` = sum w |v| / sum w and `reach` = max |q| . |k| * scale over the seen keys, for bounds."""
    n, q_heads, dim = q.shape
    out = torch.zeros_like(q)
    mean = torch.zeros_like(q)
    lse = torch.full((n, q_heads), -math.inf, dtype=torch.float64)
    reach = torch.zeros((n, q_heads), dtype=torch.float64)
    for r in range(len(offsets) - 1):
        a, b, past = int(offsets[r]), int(offsets[r + 1]), int(context[r])
        if b <= a:
            continue
        end = max(0, min(past + b - a, table.shape[1] * page))
        ks, vs, where = [], [], []
        for c in range(-(-end // page)):
            block = int(table[r, c])
            if 0 <= block < cache_blocks:
                m = min(page, end - c * page)
                ks.append(k_of(block)[:, :m])
                vs.append(v_of(block)[:, :m])
                where.extend(range(c * page, c * page + m))
        if not where:
            continue
        k, v, where = torch.cat(ks, 1), torch.cat(vs, 1), torch.tensor(where)
        group = q_heads // k.shape[0]
        for i in range(b - a):
            seen = where <= past + i
            if not bool(seen.any()):
                continue
            kk, vv = k[:, seen], v[:, seen]
            for h in range(q_heads):
                s = (kk[h // group] @ q[a + i, h]) * scale
                if bool((s == -math.inf).all()):
                    continue
                top = s.max()
                w = torch.exp(s - top)
                out[a + i, h] = w @ vv[h // group] / w.sum()
                mean[a + i, h] = w @ vv[h // group].abs() / w.sum()
                lse[a + i, h] = top + torch.log(w.sum())
                reach[a + i, h] = ((kk[h // group].abs() @ q[a + i, h].abs()) * scale).max()
    return out, lse, mean, reach


def bounds(out, mean, reach, dim, half):
    """How far an output in 16 bits, and its lse in 32, may be from the 64-bit ones.

    Scores: a sum of dim products in 32 bits, each product exact, is off by at most
    dim 2^-24 of the sum of magnitudes; scaling, subtraction and the exponential add a few
    2^-23 of the score. Call that d; a weight is then off by a factor of 1 + d, and rounded to 16 bits by
    1 + u. Numerator and denominator move by at most (2 d + u) mean |v|, their 32-bit sums
    by as little as the scores'. The output's own rounding adds u |out|, and the smallest
    fp16 step where it is that small."""
    u = 2.0 ** -11 if half else 2.0 ** -8
    d = reach * (dim * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -20
    tiny = 2.0 ** -24 if half else 0.0
    return ((2 * d[..., None] + u + 2.0 ** -16) * mean * 1.02 + u * out.abs() + tiny), d + 2.0 ** -20
