"""Latent caches, attention weights and eviction as a program runs them: streams, graphs, threads, padded and
malformed batches, planes past 32 bits, scores past an exponential's range, all in turn (MI355X)."""
from __future__ import annotations

import importlib.util
import math
import os
import threading

import pytest
import torch

import latent_ref as ref
from test_gpu_latent import check
from test_gpu_weights import evict_ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SCALE = 576 ** -0.5


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def i64(x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


class Batch:
    """Requests on a latent cache of one layer, their queries in both forms and their weights."""

    def __init__(self, P, new, past, heads=16, latent=512, page=16, seed=0, kind="bf16", spare=3):
        offsets, context, table, self.blocks = ref.batch(seed, new, past, page, spare=spare)
        self.host = (offsets, context, table)
        self.cache = P.LatentCache(1, latent, 64, self.blocks, block_tokens=page, kind=kind)
        dtype = self.cache.dtype
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.cache.data.view(dtype).normal_(generator=g)
        self.rows = self.cache.data.view(dtype).view(-1, self.blocks, page, latent + 64)[0]
        n = int(offsets[-1])

        def random(*shape, size=1.0):
            return (torch.randn(shape, device="cuda", generator=g) * size).to(dtype)
        self.q, self.qn = random(n, heads, latent + 64), random(n, heads, 192)
        self.w = random(heads, 256, latent, size=latent ** -0.5)
        self.latent, self.page = latent, page
        self.args = (offsets.cuda(), context.cuda(), table.cuda())
        keys = [a + b for a, b in zip(new, past)]
        self.n_keys = sum(keys)
        self.key_offsets = i64([sum(keys[:i]) for i in range(len(keys) + 1)])
        self.weights = self.cache.weights()

    def attend(self, args=None, q=None, cache=None, **kw):
        q = self.q if q is None else q
        return (cache or self.cache).attend(0, q[..., :self.latent], q[..., self.latent:], *(args or self.args),
                                            scale=SCALE, **kw)

    def expanded(self, args=None, q=None, **kw):
        q = self.qn if q is None else q
        return self.cache.attend_expanded(0, q[..., :128], q[..., 128:], self.w[:, :128], self.w[:, 128:],
                                          *(args or self.args), self.key_offsets, self.n_keys, **kw)

    def weigh(self, weights, lse, args=None, q=None, cache=None, **kw):
        q = self.q if q is None else q
        return (cache or self.cache).weigh(0, weights, q[..., :self.latent], q[..., self.latent:], lse,
                                           *(args or self.args), scale=SCALE, **kw)


FEW, WIDE = dict(new=[1, 1, 1], past=[3000, 40, 999]), dict(new=[3, 40, 9], past=[900, 7, 200])


# --- attention where the score or the batch is unusual ------------------------------------


def test_absorbed_wide_tiles_split(P):
    """128 rows of a token and keys for many workgroups."""
    check(P, "bf16", 512, 16, 128, [1, 2], [9000, 500], seed=21)


@pytest.mark.parametrize("heads,new", [(16, [1, 1]), (4, [4, 1]), (64, [2, 1]), (3, [90, 5])])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 40, 2.0 ** 100])
def test_scores_past_an_exponential(P, heads, new, size):
    """One dimension of the shared part gives the scores. The others' weights, e^-380 at most, are nothing in 32
    bits: the output is the largest key's row and lse its score."""
    b = Batch(P, new, [300, 31], heads=heads, seed=5)
    b.q.zero_()
    b.q[..., 512] = size
    b.rows[..., 512] = -1.0
    offsets, context, table = b.host
    want = []
    for r in range(2):
        pos, block, slot = ref.keys_of(r, offsets, context, table, 16, b.blocks)
        top = (7, 30)[r]
        b.rows[block.cuda(), slot.cuda(), 512] = (-1.0 - (pos % 90).float() / 64).bfloat16().cuda()
        b.rows[block[top], slot[top], 512] = 8.0
        want += [b.rows[block[top], slot[top], :512]] * new[r]
    out, lse = b.attend(lse=True)
    assert torch.equal(out, torch.stack(want)[:, None].expand_as(out))
    score = 8.0 * size * SCALE
    assert bool(((lse.double() - score).abs() <= score * 2.0 ** -21).all())
    b.rows[..., 512] = -b.rows[..., 512].abs()  # all far below zero
    out, lse = b.attend(lse=True)
    assert bool(torch.isfinite(out).all()) and bool((lse < -size * SCALE * 0.9).all())
    if size > 2.0 ** 20:  # the keys nearest to zero have all the weight
        assert bool(((lse.double() + size * SCALE).abs() <= size * SCALE * 2.0 ** -20).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads,new", [(16, [1, 1, 1]), (2, [5, 3, 1])])
def test_hidden_values_of_few_rows(P, bad, heads, new):
    """What lies in slots that no row sees, and in a draft's later tokens, changes nothing before them."""
    b = Batch(P, new, [45, 20, 333], heads=heads, seed=6)
    clean = b.attend()
    offsets, context, table = b.host
    used = torch.zeros((b.blocks, 16), dtype=torch.bool)
    for r in range(3):
        _, block, slot = ref.keys_of(r, offsets, context, table, 16, b.blocks)
        used[block, slot] = True
    b.rows[~used.cuda()] = bad
    assert torch.equal(b.attend(), clean)
    last = 45 + new[0] - 1
    b.rows[int(table[0, last // 16]), last % 16, 100] = bad
    got = b.attend()
    before = new[0] - 1
    assert torch.equal(got[:before], clean[:before]) and torch.equal(got[new[0]:], clean[new[0]:])
    assert not bool(torch.isfinite(got[before, :, 100]).any())


@pytest.mark.parametrize("shape", [FEW, WIDE])
def test_rows_behind_the_last_request(P, shape):
    """A padded batch: rows that belong to no request keep what they held, and weigh nothing."""
    b = Batch(P, **shape, seed=7)
    n = b.q.shape[0]
    out, lse = b.attend(lse=True)
    want_weights = b.weigh(b.cache.weights()[0], lse)
    more, more_n = torch.cat((b.q, b.q)), torch.cat((b.qn, b.qn))
    padded = torch.full_like(more[..., :512], 7.0, memory_format=torch.contiguous_format)
    sums = torch.full(more.shape[:2], 5.0, device="cuda")
    ws = torch.empty(P.ptstore_latent_attention_workspace(b.cache.layer(0)), dtype=torch.uint8, device="cuda")
    args = (*b.args[:1], torch.cat((b.args[1], i32([4]))), torch.cat((b.args[2], b.args[2][:1])))
    args = (torch.cat((args[0], args[0][-1:])), *args[1:])  # a request without tokens at the end
    P.ptstore_latent_attention(b.cache.layer(0), more[..., :512], more[..., 512:], padded, sums, *args, SCALE, ws)
    assert bool((padded[n:] == 7.0).all()) and bool((sums[n:] == 5.0).all())
    # tiles are chosen by the average request, and sums so ordered
    assert float((padded[:n].float() - out.float()).abs().max()) < 0.02 and torch.allclose(sums[:n], lse, rtol=1e-5, atol=1e-5)
    got = b.weigh(b.cache.weights()[0], torch.cat((lse, lse)), args=args, q=more)
    assert torch.allclose(got, want_weights, rtol=1e-5, atol=1e-6)
    padded = torch.full_like(more_n[..., :128], 7.0, memory_format=torch.contiguous_format)
    b.key_offsets = torch.cat((b.key_offsets, b.key_offsets[-1:]))
    b.expanded(args=args, q=more_n, out=padded)
    b.key_offsets = b.key_offsets[:-1]
    assert bool((padded[n:] == 7.0).all()) and torch.equal(padded[:n], b.expanded())


@pytest.mark.parametrize("heads", [2, 64])
@pytest.mark.parametrize("bad", [[0, 5, 3, 9], [0, -1, 3, 9], [0, 100, 3, 9], [0, 1 << 62, 3, 9], [-7, 2, 3, 9]])
def test_offsets_that_are_none(P, heads, bad):
    """Offsets have to rise; of others the calls stay within their tensors. In the latent space the requests
    whose own are in order are as they would be alone (where two have the same tokens, rows are either's); the
    expanded form, which finds a tile's request by the offsets, computes their rows or leaves them."""
    b = Batch(P, [2, 1, 6], [50, 80, 200], heads=heads, seed=8)
    out, lse = b.attend(lse=True)
    args = (i64(bad), *b.args[1:])
    got, sums = b.attend(args=args, lse=True)
    assert float((got[5:].float() - out[5:].float()).abs().max()) < 0.02
    assert torch.allclose(sums[5:], lse[5:], rtol=1e-5, atol=1e-5)
    want = b.expanded()[5:]
    got = b.expanded(args=args, out=torch.full_like(b.qn[..., :128], 7.0, memory_format=torch.contiguous_format))[5:]
    assert bool(((got == want) | (got == 7.0)).all())
    weights = b.weigh(b.cache.weights()[0], lse, args=args)
    assert bool(torch.isfinite(weights).all())


def test_context_past_the_table(P):
    """Contexts far below zero and far past what the pages hold: keys are cut to the pages."""
    b = Batch(P, [1, 2, 1], [30, 60, 20], seed=9)
    args = (b.args[0], i32([-2 ** 31, 2 ** 31 - 1, -5]), b.args[2])
    out, lse = b.attend(args=args, lse=True)
    assert not bool(out[[0, 3]].any()) and bool((lse[[0, 3]] == -math.inf).all())
    whole = b.attend(args=(b.args[0], i32([0, 16 * b.args[2].shape[1], 0]), b.args[2]))
    assert float((out[1:3].float() - whole[1:3].float()).abs().max()) < 0.02
    b.expanded(args=args)
    weights = b.weigh(b.cache.weights()[0], lse, args=args)
    assert bool(torch.isfinite(weights).all())
    b.cache.evict(b.cache.weights(), args[1], args[2], i32([4, 9, 2 ** 31 - 1]), 9)


def test_requests_that_share_pages(P):
    """The same pages in two requests' tables give each what copies would."""
    b = Batch(P, [1, 1], [200, 260], seed=10)
    offsets, context, table = b.host
    shared = table.clone()
    shared[1, :8] = table[0, :8]
    got = b.attend(args=(b.args[0], b.args[1], shared.cuda()))
    for c in range(8):
        b.rows[int(table[1, c])] = b.rows[int(table[0, c])]
    assert torch.equal(b.attend(), got)


@pytest.mark.parametrize("heads", [2, 40, 65])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_expanded_hidden_values(P, heads, bad):
    """A later token's infinite row leaves the rows before it alone, in tiles of 32 tokens, and of 128 by eight waves
    and by four."""
    b = Batch(P, [140, 3, 1, 1], [45, 20, 300, 0], heads=heads, seed=19)
    clean = b.expanded()
    pos = 45 + 100  # the 101st new token
    b.rows[int(b.host[2][0, pos // 16]), pos % 16, 7] = bad
    got = b.expanded()
    assert torch.equal(got[:100], clean[:100]) and torch.equal(got[140:], clean[140:])
    assert not bool(torch.isfinite(got[100:140]).all(-1).any())


# --- planes past 32 bits -----------------------------------------------------------------


def test_latent_planes_past_32_bits(P):
    """Pages at both ends of a plane of 4.8 GB: the same bits as from a small cache."""
    small = Batch(P, [1, 1, 4], [700, 90, 300], heads=16, seed=11)
    offsets, context, table = small.host
    far = 260000
    big = P.LatentCache(1, 512, 64, far)
    where = torch.arange(small.blocks)
    where[::2] = far - 1 - where[::2]
    big_table = torch.where(table >= 0, where[table.clamp(min=0).long()].int(), table).cuda()
    slots = (where[:, None] * 16 + torch.arange(16)).view(-1).cuda()
    rows = small.rows.reshape(-1, 576)
    big.append(0, rows[:, :512], rows[:, 512:], slots)
    back, _ = big.read(0, slots)
    assert torch.equal(back, rows[:, :512])
    args = (*small.args[:2], big_table)
    out, lse = small.attend(lse=True)
    got, got_lse = small.attend(args=args, cache=big, lse=True)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    w, big_w = small.cache.weights(), big.weights()
    small.weigh(w[0], lse)
    small.weigh(big_w[0], lse, args=args, cache=big)
    assert torch.equal(big_w[0][where.cuda()], w[0])
    length, keep = small.args[1] + i32([1, 1, 4]), i32([100, 50, 200])
    assert torch.equal(big.evict(big_w, length, big_table, keep, 200, recent=7),
                       small.cache.evict(w, length, small.args[2], keep, 200, recent=7))
    assert torch.equal(big_w[0][where.cuda()], w[0])
    got, got_rope = big.read(0, slots)
    assert torch.equal(torch.cat((got, got_rope), 1), rows)
    wk = small.w
    a = small.cache.attend_expanded(0, small.qn[..., :128], small.qn[..., 128:], wk[:, :128], wk[:, 128:], *small.args,
                                    small.key_offsets, small.n_keys)
    b = big.attend_expanded(0, small.qn[..., :128], small.qn[..., 128:], wk[:, :128], wk[:, 128:], *args,
                            small.key_offsets, small.n_keys)
    assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_paged_planes_past_32_bits(P, kind):
    """The same of weights and eviction over a paged cache, planes of 4.6 and 2.6 GB, places past 2^31 bytes."""
    heads, dim, far, used = 8, 128, 140000 if kind == "bf16" else 300000, 60
    small, big = P.PagedCache(1, heads, dim, used, kind=kind), P.PagedCache(1, heads, dim, far, kind=kind)
    where = torch.arange(used)
    where[::2] = far - 1 - where[::2]
    slots = torch.arange(used * 16, device="cuda")
    big_slots = (where[:, None] * 16 + torch.arange(16)).view(-1).cuda()
    g = torch.Generator(device="cuda").manual_seed(12)
    k, v = (torch.randn((used * 16, heads, dim), device="cuda", generator=g).bfloat16() for _ in range(2))
    small.append(0, k, v, slots)
    big.append(0, k, v, big_slots)
    table = torch.randperm(used, generator=torch.Generator().manual_seed(1)).int().view(2, 30)
    big_table, table = where[table.long()].int().cuda(), table.cuda()
    q = torch.randn((3, 32, dim), device="cuda", generator=g).bfloat16()
    off, ctx, length = i64([0, 1, 3]), i32([470, 300]), i32([471, 302])
    out, lse = small.attend(0, q, off, ctx, table, lse=True)
    w, big_w = small.weights(), big.weights()
    small.weigh(0, w[0], q, lse, off, ctx, table)
    big.weigh(0, big_w[0], q, lse, off, ctx, big_table)
    assert torch.equal(big_w[0][where.cuda()], w[0])
    keep = i32([200, 77])
    small.evict(w, length, table, keep, 200, recent=16)
    big.evict(big_w, length, big_table, keep, 200, recent=16)
    assert torch.equal(big_w[0][where.cuda()], w[0])
    for a, b in zip(small.read(0, slots), big.read(0, big_slots)):
        assert torch.equal(a, b)


# --- streams, graphs, threads --------------------------------------------------------------


@pytest.mark.parametrize("shape", [FEW, WIDE])
def test_other_streams(P, shape):
    """Three streams at once, by stream and by raw handle, with workspaces of their own."""
    b = Batch(P, **shape, seed=13)
    out, lse = b.attend(lse=True)
    want = (out, b.weigh(b.cache.weights()[0], lse), b.expanded())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    weights = [b.cache.weights()[0] for _ in range(9)]
    torch.cuda.synchronize()
    got = []
    for i in range(9):
        s = streams[i % 3] if i % 2 else streams[i % 3].cuda_stream
        o, sums = b.attend(lse=True, stream=s)
        got.append((o, b.weigh(weights[i], sums, stream=s), b.expanded(stream=s)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(g, want))


def test_evict_on_another_stream(P):
    b = Batch(P, [1, 1], [900, 300], seed=14)
    b.weights.copy_(torch.rand_like(b.weights))
    other, rows = b.weights.clone(), b.cache.data.clone()
    want = b.cache.evict(b.weights, b.args[1], b.args[2], i32([300, 100]), 300, recent=9)
    moved = b.cache.data.clone()
    b.cache.data.copy_(rows)
    keep, s = i32([300, 100]), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = b.cache.evict(other, b.args[1], b.args[2], keep, 300, recent=9, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(other, b.weights) and torch.equal(b.cache.data, moved)


@pytest.mark.parametrize("heads", [16, 64])
def test_a_step_in_a_graph(P, heads):
    """Append, attention, weights and eviction of a step, captured once, the first calls of their cache: each
    replay goes on from the last, as eager steps on a copy do, with eager work of the program between."""
    b = Batch(P, [1, 1, 1], [500, 90, 200], heads=heads, seed=15, spare=80)
    other = P.LatentCache(1, 512, 64, b.blocks)
    other.data.copy_(b.cache.data)
    ones, table = i64([0, 1, 2, 3]), b.args[2].clone()
    table[:, :] = torch.randperm(b.blocks, device="cuda")[:table.numel()].view_as(table)
    keep = i32([300, 64, 4000])
    new = torch.randn((3, 576), device="cuda").bfloat16()
    context = i32([500, 90, 200])

    def step(cache, weights, context, q, new):
        slot = table.gather(1, (context[:, None] // 16).long())[:, 0].long() * 16 + context % 16
        cache.append(0, new[:, :512], new[:, 512:], slot)
        out, lse = cache.attend(0, q[..., :512], q[..., 512:], ones, context, table, SCALE, lse=True)
        cache.weigh(0, weights[0], q[..., :512], q[..., 512:], lse, ones, context, table, SCALE)
        after = cache.evict(weights, context + 1, table, keep, 400, recent=32)
        return out, after
    weights, other_weights = torch.rand_like(b.weights), None
    other_weights, other_context = weights.clone(), context.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, after = step(b.cache, weights, context, b.q, new)
        context.copy_(after)
    for i in range(4):
        b.q.copy_(torch.randn_like(b.q))
        new.copy_(torch.randn_like(new))
        graph.replay()
        torch.cuda.synchronize()
        want, other_context = step(other, other_weights, other_context, b.q, new)
        assert torch.equal(out, want) and torch.equal(context, other_context)
        assert torch.equal(weights, other_weights) and torch.equal(b.cache.data, other.data)


def test_two_graphs_at_once(P):
    """Graphs of one cache, captured on one stream, replayed on two: their workspaces are their own."""
    b, c = Batch(P, **WIDE, seed=16), Batch(P, **FEW, seed=16)
    b.cache = c.cache  # the larger
    want = [b.attend(), b.expanded(), c.attend()]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for call in (b.attend, b.expanded, c.attend):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_threads_of_one_stream(P):
    b = Batch(P, **WIDE, seed=17)
    q2 = torch.randn_like(b.q)
    want = [b.attend(lse=True), b.attend(q=q2, lse=True)]
    weighed = [b.weigh(b.cache.weights()[0], want[i][1], q=q) for i, q in enumerate((b.q, q2))]
    wrong = []

    def work(i, q):
        for _ in range(10):
            out, lse = b.attend(q=q, lse=True)
            w = b.weigh(b.cache.weights()[0], lse, q=q)
            torch.cuda.synchronize()
            if not (torch.equal(out, want[i][0]) and torch.equal(w, weighed[i])):
                wrong.append(i)
    threads = [threading.Thread(target=work, args=(i, q)) for i, q in enumerate((b.q, q2))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


# --- together ---------------------------------------------------------------------------


def test_attention_after_eviction(P):
    """What is kept attends as the same tokens in a cache of their own; a layer outside `layers` is left."""
    b = Batch(P, [1], [600], heads=16, seed=18)
    cache = P.LatentCache(3, 512, 64, b.blocks)
    cache.data.view(torch.bfloat16).normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    planes = cache.data.view(torch.bfloat16).view(4, b.blocks, 16, 576)
    before = planes.clone()
    weights = cache.weights((1, 3)).uniform_()
    w0, table = weights.cpu(), b.host[2]
    after = cache.evict(weights, b.args[1], b.args[2], i32([150]), 150, recent=20, layers=(1, 3))
    assert after.tolist() == [150]
    assert torch.equal(planes[0], before[0]) and torch.equal(planes[3], before[3])
    t = torch.arange(600)
    block, slot = table[0].long()[t // 16], t % 16
    for layer in (1, 2):
        stay = evict_ref(w0[layer - 1, block, 0, slot].tolist(), 600, 150, 20)
        own = P.LatentCache(1, 512, 64, 10)
        rows = before[layer, block[stay].cuda(), slot[stay].cuda()]
        own.append(0, rows[:, :512], rows[:, 512:], torch.arange(150, device="cuda"))
        ten = torch.arange(10, dtype=torch.int32, device="cuda")[None]
        q = b.q
        want = own.attend(0, q[..., :512], q[..., 512:], b.args[0], after - 1, ten, SCALE)
        assert torch.equal(cache.attend(layer, q[..., :512], q[..., 512:], b.args[0], after - 1, b.args[2], SCALE), want)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_latent_step(kind):
    spec = importlib.util.spec_from_file_location("latent_step", os.path.join(ROOT, "examples", "latent_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(kind, requests=5, passage=160, budget=96, steps=3) >= 5 * 160
