"""A serving program's steps with latent caches, the prefix store and a budget of tokens a request.

Requests share long passages. The store loads the prefixes that it holds into a latent cache; the
remaining tokens' rows are appended, and the prompts run in the expanded form, each head's keys and values
formed from the rows; single tokens run in the latent space, where a head's query is multiplied by
its key matrix first. Each step's queries add their attention weights to the tokens they read, and a request that
has grown past its budget keeps, in each layer, its latest tokens and those of largest weight. The model is
a stand-in of two layers: random tables give a token's rows and queries, so that the two forms must
agree, as a loaded prefix and a computed one must, which is what the program checks.

    python examples/latent_step.py [--kind bf16|fp16] [--requests 6] [--passage 512] [--budget 256]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_22648_amd.ptstore import LatentCache, PrefixStore  # noqa: E402

VOCAB, PAGE, LAYERS = 1000, 16, 2
HEADS, LATENT, ROPE = 16, 512, 64
SCALE = (128 + ROPE) ** -0.5


class Layer:
    """A token's row and queries, by table, and the matrices of the heads."""

    def __init__(self, dtype, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def table(*shape, size=1.0):
            return (torch.randn(shape, device="cuda", generator=g) * size).to(dtype)
        self.row, self.q = table(VOCAB, LATENT + ROPE), table(VOCAB, HEADS, 128 + ROPE)
        self.w_k, self.w_v = (table(HEADS, 128, LATENT, size=LATENT ** -0.5) for _ in range(2))

    def rows(self, tokens):
        row = self.row[tokens.long()]
        return row[:, :LATENT], row[:, LATENT:]

    def queries(self, tokens):
        q = self.q[tokens.long()]
        return q[..., :128], q[..., 128:]

    def absorbed(self, q_nope):
        """A head's queries times its key matrix: what meets the latent rows."""
        q = q_nope.transpose(0, 1).float() @ self.w_k.float()
        return q.transpose(0, 1).to(q_nope.dtype)

    def values(self, out):
        """A head's attention in the latent space, times its value matrix."""
        return (out.transpose(0, 1).float() @ self.w_v.float().transpose(1, 2).contiguous()).transpose(0, 1)


def summed(lengths):
    offsets = torch.zeros(len(lengths) + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = lengths.cumsum(0)
    return offsets


def serve(store, cache, layers, prompts, steps: int, budget: int):
    """Answers a batch of prompts with `steps` more tokens each. Returns every request's outputs (its prompt's last
    token, then its steps), how many tokens came from the store and how many each request has at the end."""
    R = len(prompts)
    lengths = torch.tensor([len(p) for p in prompts], device="cuda")
    tokens, offsets = torch.cat(prompts), summed(lengths)
    width = -(-(int(lengths.max()) + steps) // PAGE)
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(cache.cache_blocks, device="cuda", dtype=torch.int32)

    # stored prefixes into blocks of the whole prompts, at most up to a prompt's last token
    matched, ids = store.lookup(tokens, offsets, width)
    matched = torch.minimum(matched, (lengths.int() - 1) // PAGE).int()
    none = torch.zeros(R, dtype=torch.int32, device="cuda")
    _, _, held, nxt = cache.tables(offsets, none, table, free, tokens.numel())
    store.gather(ids, matched, table, cache.data)

    # the rest of the prompts, in the expanded form
    context = matched * PAGE
    r = torch.repeat_interleave(torch.arange(R, device="cuda"), lengths)
    new = tokens[torch.arange(tokens.numel(), device="cuda") - offsets[r] >= context[r]]
    new_offsets = summed(lengths - context)
    slots, _, held, nxt = cache.tables(new_offsets, context, table, free, new.numel(), held=held, first=nxt)
    weights, unweighed = cache.weights(), none
    last = new_offsets[1:] - 1
    answers = []
    for i, layer in enumerate(layers):
        cache.append(i, *layer.rows(new), slots)
        q_nope, q_rope = layer.queries(new)
        batch = (new_offsets, context, table)
        out, lse = cache.attend_expanded(i, q_nope, q_rope, layer.w_k, layer.w_v, *batch, offsets, tokens.numel(),
                                         lse=True)
        q_latent = layer.absorbed(q_nope)
        latent = cache.attend(i, q_latent, q_rope, *batch, SCALE)
        off = float((layer.values(latent) - out.float()).abs().max())
        assert off < 0.05, off  # the absorbed queries are rounded to 16 bits, and the latent outputs
        # a loaded prefix has no weights yet: every token's begin here
        cache.weigh(i, weights[i], q_latent, q_rope, lse, *batch, SCALE, weighed=unweighed)
        answers.append([out[last].float()])

    # new whole blocks go to the store
    m, ids, created = store.insert(tokens, offsets, width)
    store.scatter(ids, created, table, cache.data)

    # single tokens, in the latent space; requests past the budget give up tokens, and their pages
    length = lengths.int()
    ones = torch.arange(R + 1, dtype=torch.int64, device="cuda")
    keep = torch.full((R,), budget, dtype=torch.int32, device="cuda")
    for step in range(steps):
        length = cache.evict(weights, length, table, keep, budget, recent=budget // 4)
        held = torch.minimum(held, (length + PAGE - 1) // PAGE)  # (their blocks could be used again)
        token = (torch.arange(R, device="cuda") * 7 + step) % VOCAB
        slots, _, held, nxt = cache.tables(ones, length, table, free, R, held=held, first=nxt)
        for i, layer in enumerate(layers):
            cache.append(i, *layer.rows(token), slots)
            q_nope, q_rope = layer.queries(token)
            q_latent = layer.absorbed(q_nope)
            out, lse = cache.attend(i, q_latent, q_rope, ones, length, table, SCALE, lse=True)
            cache.weigh(i, weights[i], q_latent, q_rope, lse, ones, length, table, SCALE)
            answers[i].append(layer.values(out))
        length = length + 1
    return torch.stack([torch.stack(a) for a in answers]), int(matched.sum()) * PAGE, length


def main(kind: str = "bf16", requests: int = 6, passage: int = 512, budget: int = 256, steps: int = 4) -> int:
    g = torch.Generator().manual_seed(1)
    blocks = requests * (-(-(passage + 200 + steps) // PAGE) + 1 + steps)
    cache = LatentCache(LAYERS, LATENT, ROPE, blocks, block_tokens=PAGE, kind=kind)
    layers = [Layer(cache.dtype, seed) for seed in range(LAYERS)]
    passages = torch.randint(0, VOCAB, (2, passage), generator=g, dtype=torch.int32).cuda()
    prompts = [torch.cat([passages[i % 2], torch.randint(0, VOCAB, (1 + (i * 37) % 180,), generator=g,
                                                         dtype=torch.int32).cuda()]) for i in range(requests)]
    with PrefixStore(cache.shape, pool_blocks=2 * blocks) as store:
        cold, loaded, length = serve(store, cache, layers, prompts, steps, 10 * passage)
        assert loaded == 0
        warm, loaded, _ = serve(store, cache, layers, prompts, steps, 10 * passage)
        assert loaded >= requests * (passage // PAGE) * PAGE
        # the prefixes' rows are the same bytes: only the order of sums differs with the number of new tokens
        off = float((warm - cold).abs().max())
        assert off < 0.02, off
        _, _, short = serve(store, cache, layers, prompts, steps, budget)
        want = length - steps
        for _ in range(steps):
            want = want.clamp(max=budget) + 1
        assert torch.equal(short, want), (short, want)
        torch.cuda.synchronize()
    print(f"latent_step ok: {requests} requests, {loaded} prefix tokens loaded, {kind} cache, answers within {off:.2g}, "
          f"{int(length.sum())} tokens, {int(short.sum())} with a budget of {budget}")
    return loaded


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--kind", default="bf16", choices=("bf16", "fp16"))
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--passage", type=int, default=512)
    ap.add_argument("--budget", type=int, default=256)
    a = ap.parse_args()
    main(a.kind, a.requests, a.passage, a.budget)
