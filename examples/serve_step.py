"""A serving program's steps around the prefix store, on one layer's worth of model.

Requests share long passages. For each batch: the store is asked what it holds of
each request, the requests get cache blocks, the stored prefixes are loaded into the
paged cache, the remaining tokens' K and V are appended, and attention runs over
the pages: the prompts behind their prefixes, then single tokens. What was new goes
to the store, and the second batch finds it there. The model is a stand-in: random
tables give a token's q, k and v, so that a loaded prefix must give the same attention
as a computed one, which is what the program checks.

    python examples/serve_step.py [--kind bf16|fp16|mxfp4] [--requests 8] [--passage 512]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_22648_amd.ptstore import PagedCache, PrefixStore  # noqa: E402

VOCAB, PAGE = 1000, 16


class Layer:
    """q, k and v of a token, by table."""

    def __init__(self, heads: int, group: int, dim: int, dtype, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.q = torch.randn((VOCAB, heads * group, dim), device="cuda", generator=g).to(dtype)
        self.kv = torch.randn((VOCAB, 2 * heads, dim), device="cuda", generator=g).to(dtype)
        self.heads = heads

    def __call__(self, tokens):
        kv = self.kv[tokens.long()]
        return self.q[tokens.long()], kv[:, :self.heads], kv[:, self.heads:]


def batch(prompts):
    """Packed tokens and offsets of a list of prompts."""
    offsets = torch.zeros(len(prompts) + 1, dtype=torch.int64)
    offsets[1:] = torch.tensor([len(p) for p in prompts]).cumsum(0)
    return torch.cat(prompts), offsets.cuda()


def serve(store, cache, layer, prompts, steps: int):
    """Answers a batch of prompts with `steps` more tokens each; returns the attention of every
    prompt's last tokens and of every step, and how many prefix tokens came from the store."""
    R = len(prompts)
    tokens, offsets = batch(prompts)
    lengths = offsets.diff().int()
    most = int(lengths.max())
    width = -(-(most + steps) // PAGE)
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(cache.cache_blocks, device="cuda", dtype=torch.int32)

    # what the store has, at most all blocks but a prompt's last token's: that one is computed
    matched, ids = store.lookup(tokens, offsets, width)
    matched = torch.minimum(matched, (lengths - 1) // PAGE)

    # blocks for whole prompts; then the stored prefixes into them
    none = torch.zeros(R, dtype=torch.int32, device="cuda")
    _, _, held, nxt = cache.tables(offsets, none, table, free, tokens.numel())
    store.gather(ids, matched.int(), table, cache.data)

    # the tokens behind the prefixes: packed, with their own offsets
    context = (matched * PAGE).int()
    r = torch.repeat_interleave(torch.arange(R, device="cuda"), lengths)
    keep = torch.arange(tokens.numel(), device="cuda") - offsets[r] >= context[r]
    new = tokens[keep]
    new_offsets = torch.zeros_like(offsets)
    new_offsets[1:] = (lengths - context).cumsum(0)
    slots, _, held, nxt = cache.tables(new_offsets, context, table, free, new.numel(), held=held, first=nxt)
    q, k, v = layer(new)
    cache.append(0, k, v, slots)
    out = cache.attend(0, q, new_offsets, context, table)
    answers = [out[new_offsets[1:] - 1]]

    # new whole blocks go to the store
    m, ids, created = store.insert(tokens, offsets, width)
    store.scatter(ids, created, table, cache.data)

    # single tokens
    context = lengths.clone()
    ones = torch.arange(R + 1, dtype=torch.int64, device="cuda")
    for step in range(steps):
        slots, _, held, nxt = cache.tables(ones, context, table, free, R, held=held, first=nxt)
        q, k, v = layer((torch.arange(R, device="cuda") * 7 + step) % VOCAB)
        cache.append(0, k, v, slots)
        answers.append(cache.attend(0, q, ones, context, table))
        context = context + 1
    return torch.stack(answers), int(matched.sum()) * PAGE


def main(kind: str = "bf16", requests: int = 8, passage: int = 512, steps: int = 4) -> int:
    heads, group, dim = 8, 4, 128
    g = torch.Generator().manual_seed(1)
    blocks = requests * (-(-(passage + 200 + steps) // PAGE) + 1)
    cache = PagedCache(1, heads, dim, blocks, block_tokens=PAGE, kind=kind)
    layer = Layer(heads, group, dim, cache.dtype)
    passages = torch.randint(0, VOCAB, (2, passage), generator=g, dtype=torch.int32).cuda()
    prompts = [torch.cat([passages[i % 2], torch.randint(0, VOCAB, (1 + (i * 37) % 180,), generator=g,
                                                         dtype=torch.int32).cuda()]) for i in range(requests)]
    with PrefixStore(cache.shape, pool_blocks=2 * blocks) as store:
        cold, loaded = serve(store, cache, layer, prompts, steps)
        assert loaded == 0
        warm, loaded = serve(store, cache, layer, prompts, steps)
        assert loaded >= requests * (passage // PAGE) * PAGE
        # The prefixes' K and V are the same bytes, so the scores are; only the order of sums differs
        # with the number of new tokens.
        off = float((warm.float() - cold.float()).abs().max())
        assert off < 0.02, off
        torch.cuda.synchronize()
    print(f"serve_step ok: {requests} requests, {loaded} prefix tokens loaded, {kind} cache, answers within {off:.2g}")
    return loaded


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--kind", default="bf16", choices=("bf16", "fp16", "mxfp4"))
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--passage", type=int, default=512)
    a = ap.parse_args()
    main(a.kind, a.requests, a.passage)
