"""Accumulated attention weights and eviction by them, against 64 bits (MI355X)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import latent_ref as ref
import paged_ref

pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "mxfp4": torch.bfloat16}


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


def make(P, kind, heads, dim, blocks, page, seed, layers=1):
    """A cache of random values: PagedCache, or LatentCache where heads is None and dim the latent one."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if heads is None:
        cache = P.LatentCache(layers, dim, 64, blocks, block_tokens=page, kind=kind)
    else:
        cache = P.PagedCache(layers, heads, dim, blocks, block_tokens=page, kind=kind)
    if kind == "mxfp4":
        cache.data.random_(generator=g)
        planes = cache.data.view(2 * layers, blocks, -1)
        n = heads * page * dim // 2
        planes[..., n:] = planes[..., n:] % 3 + 124
    else:
        cache.data.view(DTYPE[kind]).normal_(generator=g)
    return cache


def key_values(cache, P, kind, heads, dim, blocks, page):
    """Layer 0's keys in 64 bits, [blocks, heads, page, dim] (CPU)."""
    if heads is None:
        return cache.data.view(DTYPE[kind]).view(-1, blocks, 1, page, dim + 64)[0].cpu().double()
    if kind != "mxfp4":
        return cache.data.view(DTYPE[kind]).view(-1, 2, blocks, heads, page, dim)[0, 0].cpu().double()
    raw = cache.data.view(-1, 2, blocks, cache.data.numel() // 2 // blocks)[0, 0].cpu().numpy()
    n = heads * page * dim // 2
    codes = raw[:, :n].reshape(blocks, heads, page, dim // 2)
    codes = np.stack((codes & 15, codes >> 4), -1).reshape(blocks, heads, page, dim)
    power = raw[:, n:n + heads * page * dim // 32].reshape(blocks, heads, page, dim // 32)
    return torch.from_numpy(paged_ref.values_of(codes, power))


def weigh_ref(weights, q, lse, keys, offsets, context, weighed, table, page, scale):
    """(weights after, what was added in magnitudes times the scores' sizes, for the bound)."""
    want, moved = weights.double().clone(), torch.zeros_like(weights, dtype=torch.float64)
    heads = keys.shape[1]
    group = q.shape[1] // heads
    for r in range(len(offsets) - 1):
        a, b = int(offsets[r]), int(offsets[r + 1])
        if b <= a:
            continue
        pos, block, slot = ref.keys_of(r, offsets, context, table, page, keys.shape[0])
        for h in range(heads):
            k = keys[block, h, slot]
            rows = q[a:b, h * group:(h + 1) * group].double()
            s = torch.einsum("tgd,kd->tgk", rows, k) * scale
            reach = torch.einsum("tgd,kd->tgk", rows.abs(), k.abs()) * scale
            less = lse[a:b, h * group:(h + 1) * group].double()[..., None]
            w = torch.exp(s - less)
            seen = pos <= (int(context[r]) + torch.arange(b - a))[:, None, None]
            w = torch.where(seen & (less > -math.inf), w, 0.0)
            old = torch.where(pos < int(weighed[r]), want[block, h, slot], 0.0)
            want[block, h, slot] = old + w.sum((0, 1))
            size = torch.where(seen, reach, 0.0) * q.shape[2] * 2.0 ** -24 + less.abs().clamp(max=1e30) * 2.0 ** -22 + 2.0 ** -20
            moved[block, h, slot] = (w * size).sum((0, 1)) * 1.1 + old * 2.0 ** -23
    return want, moved


def check_weigh(P, kind, heads, dim, page, group, new, past, seed=0, hole=False, weighed=None, stride=False, qscale=1.0):
    offsets, context, table, blocks = ref.batch(seed, new, past, page, hole=hole)
    cache = make(P, kind, heads, dim, blocks, page, seed)
    kv_heads, size = heads or 1, dim if heads else dim + 64
    n, g = int(offsets[-1]), torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((n, kv_heads * group, size), generator=g) * qscale).to(DTYPE[kind])
    scale = size ** -0.5
    weights = cache.weights()
    assert weights.shape == (1, blocks, kv_heads, page)
    weights[0] = torch.rand((blocks, kv_heads, page), generator=g).cuda()
    before = weights.cpu()[0]
    d = q.cuda()
    if stride:
        d = torch.cat((d, d), 1)[:, :q.shape[1]]
    batch = (offsets.cuda(), context.cuda(), table.cuda())
    if heads:
        _, lse = cache.attend(0, d, *batch, lse=True)
        args = (d,)
    else:
        _, lse = cache.attend(0, d[..., :dim], d[..., dim:], *batch, scale=scale, lse=True)
        args = (d[..., :dim], d[..., dim:])
    w = None if weighed is None else torch.tensor(weighed, dtype=torch.int32).cuda()
    got = cache.weigh(0, weights[0], *args, lse, *batch, scale=scale, weighed=w)
    assert got.data_ptr() == weights.data_ptr()
    want, tol = weigh_ref(before, q, lse.cpu(), key_values(cache, P, kind, heads, dim, blocks, page), offsets, context,
                          context if weighed is None else weighed, table, page, scale)
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol + want.abs() * 2.0 ** -23).all()), float((off / (tol + 1e-30)).max())
    # a token's weights sum to what each row has: one, where it sees anything
    again = before.cuda()
    assert torch.equal(cache.weigh(0, again, *args, lse, *batch, scale=scale, weighed=w), got)


CASES = [([1], [0]), ([1], [300]), ([1, 1, 0, 1], [5, 255, 9, 600]), ([1, 3, 2], [100, 33, 257]), ([140], [0]),
         ([33, 300], [64, 255]), ([700], [130])]


@pytest.mark.parametrize("kind,heads,dim,group", [("bf16", 2, 128, 4), ("fp16", 3, 64, 1), ("mxfp4", 2, 128, 4),
                                                  ("mxfp4", 1, 64, 8), ("bf16", None, 512, 16), ("fp16", None, 256, 5)])
@pytest.mark.parametrize("new,past", CASES)
def test_weigh(P, kind, heads, dim, group, new, past):
    check_weigh(P, kind, heads, dim, 16, group, new, past, seed=len(new) + group)


@pytest.mark.parametrize("page", [1, 7, 24, 64])
@pytest.mark.parametrize("heads,dim", [(2, 128), (None, 512)])
def test_weigh_pages_and_holes(P, page, heads, dim):
    check_weigh(P, "bf16", heads, dim, page, 4, [1, 40, 2], [130, 9, 300], seed=page, hole=True)


@pytest.mark.parametrize("kind,heads,dim,page", [("bf16", 2, 128, 1), ("fp16", 1, 64, 7), ("bf16", 3, 64, 24), ("fp16", 2, 128, 64),
                                                 ("mxfp4", 2, 128, 24), ("bf16", None, 256, 24)])
def test_weigh_steps_beside_a_prompt(P, kind, heads, dim, page):
    """Single tokens, drafts and requests without tokens, of lengths around a wave's 32 and 64 keys and a tile's 256,
    with missing pages; one prompt among them, and none."""
    new = [1, 1, 0, 2, 1, 1, 4, 1, 0, 1]
    past = [0, 31, 9, 62, 63, 255, 256, 800, 0, 1500]
    check_weigh(P, kind, heads, dim, page, 4, new, past, seed=page, hole=True)
    check_weigh(P, kind, heads, dim, page, 4, new + [60], past + [130], seed=page + 1, hole=True, stride=True)


@pytest.mark.parametrize("heads,dim", [(1, 128), (None, 256)])
def test_weigh_cut_tiles(P, heads, dim):
    """Few keys and many rows: key tiles that several workgroups share."""
    check_weigh(P, "bf16", heads, dim, 16, 32, [900], [37], seed=3)
    check_weigh(P, "bf16", heads, dim, 16, 8, [260, 1, 300, 515], [0, 500, 129, 255], seed=4)


def test_weigh_many_requests_strides_and_loaded_prefixes(P):
    check_weigh(P, "bf16", 2, 64, 16, 2, [1] * 600, [i % 90 for i in range(600)], seed=5)
    check_weigh(P, "bf16", 2, 128, 16, 2, [2, 30], [50, 40], seed=6, stride=True)
    check_weigh(P, "bf16", 2, 128, 16, 2, [2, 30], [50, 40], seed=7, weighed=[0, 17])
    check_weigh(P, "fp16", 2, 128, 16, 2, [2, 30], [50, 40], seed=8, qscale=6.0)


def test_weigh_touches_nothing_else_and_passes_nan(P):
    page, heads = 16, 2
    offsets, context, table, blocks = ref.batch(3, [2, 1], [20, 40], page)
    cache = make(P, "bf16", heads, 64, blocks, page, 3)
    cache.data.view(torch.bfloat16).view(2, blocks, heads, page, 64)[0, int(table[0, 0]), 1, 3] = math.nan
    q = torch.randn((3, 4, 64), device="cuda").bfloat16()
    batch = (offsets.cuda(), context.cuda(), table.cuda())
    lse = torch.tensor([[0.0, -math.inf, 1.0, 2.0], [1.0, 1.0, 1.0, 1.0], [math.nan, 1.0, 1.0, 1.0]], device="cuda")
    w = torch.full((blocks, heads, page), 7.0, device="cuda")
    cache.weigh(0, w, q, lse, *batch, weighed=torch.zeros(2, dtype=torch.int32, device="cuda"))
    w = w.cpu()
    used = torch.zeros((blocks, page), dtype=torch.bool)
    for r in range(2):
        _, block, slot = ref.keys_of(r, offsets, context, table, page, blocks)
        used[block, slot] = True
    assert bool((w.transpose(1, 2)[~used] == 7).all())
    nan = torch.isnan(w)
    assert bool(nan[int(table[0, 0]), 1, 3])
    _, block, slot = ref.keys_of(1, offsets, context, table, page, blocks)
    assert bool(nan[block, 0, slot].all()) and not bool(nan[block, 1, slot].any())
    assert int(nan.sum()) == 1 + len(block)


# --- eviction ---------------------------------------------------------------------------


@pytest.mark.parametrize("heads,dim", [(2, 128), (1, 64), (None, 512)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_weigh_steps_do_not_see_what_is_not_theirs(P, heads, dim, bad):
    """Single tokens and a draft: slots behind a request's last key and of missing pages hold what is not finite, and
    so does a draft's last token; rows whose lse is minus infinity give nothing, NaN passes to what they see."""
    new, past, page = [1, 1, 3], [45, 300, 20], 16
    offsets, context, table, blocks = ref.batch(5, new, past, page)
    cache = make(P, "bf16", heads, dim, blocks, page, 5)
    kv_heads, size = heads or 1, dim if heads else dim + 64
    rows = cache.data.view(torch.bfloat16).view(-1, blocks, kv_heads, page, size)
    q = torch.randn((5, kv_heads * 4, size), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    args = (q,) if heads else (q[..., :dim], q[..., dim:])
    batch = (offsets.cuda(), context.cuda(), table.cuda())
    lse = torch.full((5, kv_heads * 4), 3.0, device="cuda")
    start = cache.weights()[0]

    def weigh(lse):
        return cache.weigh(0, start.clone(), *args, lse, *batch, scale=0.05)
    clean = weigh(lse)
    used = torch.zeros((blocks, page), dtype=torch.bool)
    where = [ref.keys_of(r, offsets, context, table, page, blocks)[1:] for r in range(3)]
    for block, slot in where:
        used[block, slot] = True
    rows[0].transpose(1, 2)[~used.cuda()] = bad
    assert torch.equal(weigh(lse), clean)
    nothing = lse.clone()
    nothing[1] = -math.inf  # the second request's token
    block, slot = where[1]
    want = clean.clone()
    want[block.cuda(), :, slot.cuda()] = 0.0
    assert torch.equal(weigh(nothing), want)
    nothing[1] = math.nan
    got = weigh(nothing)
    assert bool(torch.isnan(got[block.cuda(), :, slot.cuda()]).all())
    keep = [r for r in (0, 2)]
    for r in keep:
        block, slot = (x.cuda() for x in where[r])
        assert torch.equal(got[block, :, slot], clean[block, :, slot])
    # the draft's last token: the others' weights are as they were
    block, slot = (x.cuda() for x in where[2])
    rows[0][block[-1], :, slot[-1]] = bad
    got = weigh(lse)
    assert torch.equal(got[block[:-1], :, slot[:-1]], clean[block[:-1], :, slot[:-1]])


@pytest.mark.parametrize("kind,dim,new", [("bf16", 128, [1, 1, 1]), ("mxfp4", 64, [1, 1, 1]), ("fp16", 64, [1, 70, 2])])
def test_weighing_and_eviction_in_a_graph(P, kind, dim, new):
    """Captured once, the first calls of their cache, replayed on other queries with eager work between: the same
    weights, pages and lengths as eager calls on a copy; and the same again on a stream of its own."""
    past, page, heads = [400, 90, 200], 16, 2
    offsets, context, table, blocks = ref.batch(7, new, past, page)
    cache, other = (make(P, kind, heads, dim, blocks, page, 7, layers=2) for _ in range(2))
    other.data.copy_(cache.data)
    n = int(offsets[-1])
    q = torch.randn((n, heads * 4, dim), device="cuda").to(cache.dtype)
    batch = (offsets.cuda(), context.cuda(), table.cuda())
    length, keep = (context + torch.tensor(new, dtype=torch.int32)).cuda(), torch.tensor([300, 64, 9], dtype=torch.int32).cuda()
    weights = cache.weights().uniform_()
    start = weights.clone()
    data = cache.data.clone()

    def step(cache, weights, stream=None):
        for layer in range(2):
            _, lse = cache.attend(layer, q, *batch, lse=True, stream=stream)
            cache.weigh(layer, weights[layer], q, lse, *batch, stream=stream)
        return cache.evict(weights, length, batch[2], keep, 300, recent=16, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        after = step(cache, weights)
    side = torch.cuda.Stream()
    for i in range(4):
        q.copy_(torch.randn_like(q))
        for c in (cache, other):
            c.data.copy_(data)
        weights.copy_(start)
        eager = start.clone()
        graph.replay()
        torch.cuda.synchronize()
        want = step(other, eager, side if i % 2 else None)
        torch.cuda.synchronize()
        assert torch.equal(after, want)
        assert torch.equal(weights.view(torch.int32), eager.view(torch.int32)) and torch.equal(cache.data, other.data)


def evict_ref(weights, n, keep, recent):
    """Positions that stay of n, in order: a token's (NaN first, weight down, position) decides."""
    m = min(n, keep)
    recent = min(recent, m)
    w = [float(x) for x in weights[:n - recent]]
    best = sorted(range(n - recent), key=lambda i: (0 if math.isnan(w[i]) else 1, -w[i] if not math.isnan(w[i]) else 0, i))
    return sorted(best[:m - recent]) + list(range(n - recent, n))


def check_evict(P, kind, heads, dim, page, past, keep, recent, seed=0, layers=2, place="other", special=False, most=None,
                ties=False):
    R = len(past)
    _, context, table, blocks = ref.batch(seed, [0] * R, past, page, spare=3 + sum(-(-k // page) for k in keep))
    cache = make(P, kind, heads, dim, blocks, page, seed, layers)
    kv_heads = heads or 1
    g = torch.Generator().manual_seed(seed + 1)
    weights = torch.rand((layers, blocks, kv_heads, page), generator=g)
    if ties:
        weights = (weights * 4).floor() / 4
    if special:
        flat = weights.view(-1)
        flat[torch.randperm(flat.numel(), generator=g)[:flat.numel() // 2]] = 0.0
        for x in (math.nan, -math.nan, math.inf, -math.inf, -0.0, -1.5, 1e-42, 3e38):
            flat[torch.randperm(flat.numel(), generator=g)[:9]] = x
    spare = torch.tensor(sorted(set(range(blocks)) - set(table.view(-1).tolist())), dtype=torch.int32)
    to, at = table.clone(), 0
    for r in range(R):
        need = -(-min(keep[r], past[r]) // page) if keep[r] > 0 else 0
        for c in range(need):
            if place == "other" or (place == "mixed" and c % 2):
                to[r, c] = spare[at]
                at += 1
    most = max(keep + [0]) if most is None else most
    dw, before = weights.cuda(), cache.data.clone()
    after = cache.evict(dw, context.cuda(), table.cuda(), torch.tensor(keep, dtype=torch.int32).cuda(), most,
                        recent=recent, to=None if place == "same" else to.cuda())
    # the same, row by row: each position's bytes
    four = kind == "mxfp4"
    planes = 1 if heads is None else 2
    size = dim + 64 if heads is None else dim
    pair = layers + layers % 2 if heads is None else layers * planes

    def rows(data):
        """[plane][block][head][slot] rows as bytes: a view, or (4 bits) codes and exponents."""
        x = data.view(pair, blocks, -1)
        if not four:
            return [x.view(pair, blocks, kv_heads, page, size * 2)]
        n = kv_heads * page * dim // 2
        return [x[..., :n].unflatten(-1, (kv_heads, page, dim // 2)),
                x[..., n:n + kv_heads * page * dim // 32].unflatten(-1, (kv_heads, page, dim // 32))]
    want = before.clone()
    ww = weights.clone()
    for r in range(R):
        n, k = max(0, min(past[r], table.shape[1] * page)), max(0, min(keep[r], most))
        for layer in range(layers):
            for h in range(kv_heads):
                t = np.arange(n)
                block, slot = table[r].long()[t // page], torch.from_numpy(t % page)
                stay = evict_ref(weights[layer, block, h, slot].tolist(), n, k, recent)
                i = torch.arange(len(stay))
                tb, ts = to[r].long()[i // page], i % page
                ww[layer, tb, h, ts] = weights[layer, block[stay], h, slot[stay]]
                for plane in range(layer * planes, layer * planes + planes):
                    for x, y in zip(rows(want), rows(before)):
                        x[plane, tb.cuda(), h, ts.cuda()] = y[plane, block[stay].cuda(), h, slot[stay].cuda()]
    assert after.tolist() == [max(0, min(a, max(0, min(k, most)))) for a, k in zip(past, keep)]
    assert torch.equal(dw.cpu().view(torch.int32), ww.view(torch.int32))
    assert torch.equal(cache.data, want)


KINDS = [("bf16", 2, 128), ("fp16", 3, 64), ("mxfp4", 2, 128), ("mxfp4", 3, 64), ("bf16", None, 512), ("fp16", None, 256)]


@pytest.mark.parametrize("kind,heads,dim", KINDS)
@pytest.mark.parametrize("place", ["other", "same", "mixed"])
def test_evict(P, kind, heads, dim, place):
    check_evict(P, kind, heads, dim, 16, [300, 0, 17, 1000], [100, 5, 40, 333], 20, seed=1, place=place)


@pytest.mark.parametrize("page", [1, 7, 24, 64])
@pytest.mark.parametrize("place", ["other", "same"])
def test_evict_pages(P, page, place):
    check_evict(P, "bf16", 2, 64, page, [130, 64], [50, 63], 5, seed=page, layers=1, place=place)


@pytest.mark.parametrize("recent", [0, 1, 50, 1000])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_ties_and_recent(P, recent, ties):
    check_evict(P, "bf16", 1, 64, 16, [600, 51, 1], [50, 51, 1], recent, seed=2, ties=ties, special=not ties)


def test_evict_sizes(P):
    """Budgets of nothing, of one, negative, above all, above max_keep; lengths past a chunk and past LDS."""
    check_evict(P, "bf16", 1, 64, 16, [40, 40, 40, 40, 9], [0, 1, -3, 41, 9], 3, seed=3, place="same", most=41)
    check_evict(P, "bf16", 1, 64, 16, [400, 300], [350, 100], 7, seed=4, place="same", most=120)
    check_evict(P, "bf16", 1, 64, 64, [30000, 12288 + 7], [9000, 5000], 7, seed=5, layers=1, place="same", ties=True)
    check_evict(P, "bf16", None, 256, 16, [2000], [1999], 0, seed=6, layers=3, place="same")


def test_evict_missing_pages(P):
    """Tokens on pages that do not exist stay last and move nowhere; places that do not exist get nothing."""
    page, blocks = 16, 12
    cache = make(P, "bf16", 1, 64, blocks, page, 7)
    table = torch.tensor([[3, -1, 5, 99]], dtype=torch.int32)
    weights = torch.rand((1, blocks, 1, page))
    before, w0 = cache.data.clone(), weights.clone()
    dw = weights.cuda()
    after = cache.evict(dw, torch.tensor([64], dtype=torch.int32).cuda(), table.cuda(),
                        torch.tensor([40], dtype=torch.int32).cuda(), 40, to=torch.tensor([[7, 8, -1, -1]], dtype=torch.int32).cuda())
    assert after.tolist() == [40]
    # the 32 tokens that are there, and 8 that are not, in order: 16 of block 3, 8 missing, 16 of block 5, of which 8 have a place
    x, y = cache.data.view(torch.bfloat16).view(2, blocks, page, 64), before.view(torch.bfloat16).view(2, blocks, page, 64)
    assert torch.equal(x[:, 7], y[:, 3]) and torch.equal(x[:, 8, :8], y[:, 8, :8]) and torch.equal(x[:, 8, 8:], y[:, 5, :8])
    assert torch.equal(dw.cpu()[0, 7], w0[0, 3]) and torch.equal(dw.cpu()[0, 8, 0, 8:], w0[0, 5, 0, :8])
    rest = [b for b in range(blocks) if b not in (7, 8)]
    assert torch.equal(x[:, rest], y[:, rest])
