"""The paged cache's operators against their definitions in 64 bits (MI355X)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "mxfp4": torch.bfloat16}


# --- block tables -------------------------------------------------------------


def batch(rng, R, most_new, most_past, page, width=None, short=0):
    new = rng.integers(0, most_new + 1, R)
    past = rng.integers(0, most_past + 1, R)
    off = np.zeros(R + 1, dtype=np.int64)
    off[1:] = np.cumsum(new)
    need = -(-(past + new) // page)
    width = int(max(1, need.max() if R else 1)) if width is None else width
    held = np.minimum(-(-past // page), width)
    taken = int((np.minimum(need, width) - held).clip(0).sum())
    ids = rng.permutation(int(held.sum()) + taken + 7).astype(np.int32)
    table = np.full((R, width), -7, dtype=np.int32)
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    free = ids[at:at + max(0, taken + 7 - short)]
    return off, past.astype(np.int32), held.astype(np.int32), table, free


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


@pytest.mark.parametrize("R,new,past,page", [
    (0, 1, 1, 16), (1, 1, 0, 16), (1, 5000, 33, 16), (3, 40, 0, 1), (64, 1, 500, 16), (65, 9, 100, 7),
    (130, 300, 77, 64), (700, 50, 200, 24), (2048, 3, 30, 16), (2049, 3, 30, 16), (5000, 7, 20, 8)])
@pytest.mark.parametrize("short", [0, 25])
def test_tables(P, R, new, past, page, short):
    rng = np.random.default_rng(R * 31 + page + short)
    off, ctx, held, table, free = batch(rng, R, new, past, page, short=short)
    first = 3 if len(free) > 3 else 0
    want = ref.tables(off, ctx, held, table, page, free, first)
    cache = P.PagedCache(1, 1, 64, 0, block_tokens=page)
    t = dev(table)
    slots, pos, after, nxt = cache.tables(dev(off), dev(ctx), t, dev(free), int(off[-1]), held=dev(held),
                                          first=torch.tensor([first], device="cuda"))
    for got, w in zip((t, slots, pos, after), want):
        assert np.array_equal(got.cpu().numpy(), w.reshape(got.shape))
    assert int(nxt) == want[4]


def test_tables_narrow_and_odd(P):
    """A table narrower than its requests, pasts beyond it or negative, no free list, nothing held."""
    off = np.array([0, 40, 40, 41, 60, 64], dtype=np.int64)
    ctx = np.array([0, 5, 1000, -3, 30], dtype=np.int32)
    table = np.full((5, 2), -1, dtype=np.int32)
    for free in (np.arange(20, dtype=np.int32), np.zeros(0, dtype=np.int32)):
        want = ref.tables(off, ctx, np.zeros(5, int), table, 16, free)
        cache = P.PagedCache(1, 1, 64, 0)
        t = dev(table)
        slots, pos, after, nxt = cache.tables(dev(off), dev(ctx), t, dev(free), 64)
        assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(slots.cpu().numpy(), want[1])
        assert np.array_equal(after.cpu().numpy(), want[3]) and int(nxt) == want[4]
        assert np.array_equal(pos.cpu().numpy(), want[2])


def test_tables_malformed_offsets_stay_in_bounds(P):
    """Decreasing, negative and over-long offsets: such a request takes no block."""
    off = np.array([0, 20, 10, 500, -4, 30], dtype=np.int64)
    table = torch.full((5, 4), -1, dtype=torch.int32, device="cuda")
    guard = torch.full((5,), -9, dtype=torch.int64, device="cuda")
    slots = torch.cat([torch.full((30,), -9, dtype=torch.int64, device="cuda"), guard])
    held, nxt = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    P.ptstore_block_tables(dev(off), dev(np.zeros(5, np.int32)), None, 16, dev(np.arange(9, dtype=np.int32)),
                           None, table, slots[:30], None, held, nxt)
    assert held.tolist() == [2, 0, 0, 0, 0] and int(nxt) == 2
    assert table.cpu()[0].tolist() == [0, 1, -1, -1] and bool((table[1:] == -1).all())
    assert torch.equal(slots[30:], guard) and int(slots[:30].max()) < 32


# --- appends and reads ----------------------------------------------------------


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,dim,page,n", [(1, 64, 1, 1), (8, 128, 16, 333), (2, 128, 24, 50), (3, 64, 7, 129)])
def test_append_16bit(P, kind, heads, dim, page, n):
    blocks = n // page + 3
    g = torch.Generator(device="cuda").manual_seed(n)
    cache = P.PagedCache(2, heads, dim, blocks, block_tokens=page, kind=kind)
    cache.data.random_(generator=g)
    before = cache.data.clone()
    qkv = torch.randn((n, 2 * heads + 1, dim), device="cuda", generator=g).to(DTYPE[kind])
    k, v = qkv[:, :heads], qkv[:, heads:2 * heads]  # strided rows
    slots = torch.randperm(blocks * page, device="cuda", generator=g)[:n]
    if n > 8:
        slots[3], slots[5], slots[7] = -1, blocks * page, 1 << 40
    cache.append(1, k, v, slots)
    want = before.view(2, 2, blocks, -1).view(DTYPE[kind]).view(2, 2, blocks, heads, page, dim).clone()
    ok = (slots >= 0) & (slots < blocks * page)
    s = slots[ok]
    want[1, 0, s // page, :, s % page] = k[ok]
    want[1, 1, s // page, :, s % page] = v[ok]
    assert torch.equal(cache.data, want.view(-1).view(torch.uint8))
    rk, rv = cache.read(1, slots)
    for got, x in ((rk, k), (rv, v)):
        assert torch.equal(got[ok].view(torch.int16), x[ok].contiguous().view(torch.int16))
        assert not bool(got[~ok].any())


def tricky_rows(n, heads, dim, seed):
    """Values of every kind a group meets: ties, saturated, tiny, zero and infinite ones."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, dim), generator=g) * torch.exp2(torch.randint(-12, 9, (n, heads, 1), generator=g).float())
    flat = x.view(-1, 32)
    flat[0] = torch.arange(32) * 0.25  # every tie, and 7.75 / 7 into the next exponent
    if flat.shape[0] > 6:
        flat[1] = -torch.arange(32) * 0.21875
        flat[1, 0] = 7.0
        flat[2] = 0
        flat[3] = torch.arange(32) * 2.0 ** -130
        flat[4, 5] = float("inf")
        flat[5, 9] = float("nan")
        flat[6] = 3.0e38
    return x.bfloat16()


@pytest.mark.parametrize("heads,dim,page,n", [(1, 64, 1, 1), (8, 128, 16, 40), (2, 128, 24, 50), (3, 64, 7, 33)])
def test_append_4bit(P, heads, dim, page, n):
    blocks = n // page + 3
    cache = P.PagedCache(1, heads, dim, blocks, block_tokens=page, kind="mxfp4")
    cache.data.fill_(0xA5)
    k, v = tricky_rows(n, heads, dim, 1), tricky_rows(n, heads, dim, 2)
    slots = torch.randperm(blocks * page, generator=torch.Generator().manual_seed(n))[:n]
    cache.append(0, k.cuda(), v.cuda(), slots.cuda())
    slab = P.ptstore_kv_slab_bytes(P.PTSTORE_KV_MXFP4, heads, dim, page)
    planes = cache.data.cpu().numpy().reshape(2, blocks, slab)
    rk, rv = cache.read(0, slots.cuda())
    for plane, x, got in ((planes[0], k, rk), (planes[1], v, rv)):
        codes, power = ref.four_bits(x.float().numpy())
        for t, s in enumerate(slots.tolist()):
            block, i = plane[s // page], s % page
            raw = block[:heads * page * dim // 2].reshape(heads, page, dim // 2)[:, i]
            exps = block[heads * page * dim // 2:][:heads * page * dim // 32].reshape(heads, page, dim // 32)[:, i]
            assert np.array_equal(exps, power[t])
            good = np.repeat(power[t] != 255, 32, axis=-1)  # a NaN group's codes mean nothing
            assert np.array_equal(np.where(good[..., 0::2], raw & 15, 0), np.where(good[..., 0::2], codes[t][..., 0::2], 0))
            assert np.array_equal(np.where(good[..., 1::2], raw >> 4, 0), np.where(good[..., 1::2], codes[t][..., 1::2], 0))
        want = ref.values_of(codes, power)
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    untouched = np.setdiff1d(np.arange(blocks * page), slots.numpy())
    for s in untouched[:50]:
        raw = planes[0, s // page, :heads * page * dim // 2].reshape(heads, page, dim // 2)[:, s % page]
        assert (raw == 0xA5).all()


# --- attention ------------------------------------------------------------------


class Case:
    """A batch over a random cache, and its 64-bit answer."""

    def __init__(self, P, kind, heads, group, dim, page, reqs, seed=0, scale=None, spread=1.0, poison=True,
                 extra=2, holes=()):
        g = torch.Generator().manual_seed(seed)
        self.P, self.page, self.dim, self.half = P, page, dim, kind == "fp16"
        new, past = [a for a, _ in reqs], [b for _, b in reqs]
        self.off = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int64)
        self.ctx = torch.tensor(past, dtype=torch.int32)
        need = [-(-max(0, a + b) // page) for a, b in reqs]
        self.width = max(need + [1]) + extra
        blocks = sum(need) + 3
        ids = torch.randperm(blocks, generator=g).int()
        self.table = torch.full((len(reqs), self.width), -1, dtype=torch.int32)
        at = 0
        for r, m in enumerate(need):
            self.table[r, :m] = ids[at:at + m]
            at += m
        for r, c, entry in holes:
            self.table[r, c] = entry
        self.q = (torch.randn((int(self.off[-1]), heads * group, dim), generator=g) * spread).to(DTYPE[kind])
        kv = torch.randn((2, blocks, heads, page, dim), generator=g)
        self.cache = P.PagedCache(1, heads, dim, blocks, block_tokens=page, kind=kind)
        n = blocks * page
        k, v = (x.permute(0, 2, 1, 3).reshape(n, heads, dim).to(DTYPE[kind]).cuda() for x in kv)
        self.cache.append(0, k, v, torch.arange(n, device="cuda"))
        k, v = self.cache.read(0, torch.arange(n, device="cuda"))
        self.kv = [x.double().cpu().view(blocks, page, heads, dim).transpose(1, 2) for x in (k, v)]
        if poison:  # what a cache holds where nothing was written: anything
            self.poison(reqs, need)
        self.blocks = blocks
        self.scale = dim ** -0.5 if scale is None else scale

    def poison(self, reqs, need):
        """NaN into the slots behind each request's last token and into unused blocks."""
        page, slots = self.page, []
        for r, (a, b) in enumerate(reqs):
            if need[r] and a + b > 0:
                last = int(self.table[r, need[r] - 1])
                if last >= 0:
                    slots += [last * page + i for i in range((a + b - 1) % page + 1, page)]
        used = set(self.table.flatten().tolist())
        for blk in range(self.cache.cache_blocks):
            if blk not in used:
                slots += [blk * page + i for i in range(page)]
        if slots:
            s = torch.tensor(slots, device="cuda")
            heads, dim = self.kv[0].shape[1], self.dim
            bad = torch.full((len(slots), heads, dim), float("nan"), dtype=self.cache.dtype, device="cuda")
            self.cache.append(0, bad, bad, s)

    def want(self):
        return ref.attention(self.q.double(), lambda b: self.kv[0][b], lambda b: self.kv[1][b], self.off, self.ctx,
                             self.table, self.page, self.blocks, self.scale)

    def run(self, **kw):
        return self.cache.attend(0, self.q.cuda(), self.off.cuda(), self.ctx.cuda(), self.table.cuda(),
                                 scale=self.scale, lse=True, **kw)

    def check(self):
        out, lse = self.run()
        self.compare(out, lse)
        return out, lse

    def compare(self, out, lse):
        o, l, mean, reach = self.want()
        near_o, near_l = ref.bounds(o, mean, reach, self.dim, self.half)
        out, lse = out.double().cpu(), lse.double().cpu()
        assert not bool(out.isnan().any()) and not bool(lse.isnan().any())
        empty = torch.isinf(l)
        assert torch.equal(torch.isinf(lse), empty) and bool((lse[empty] < 0).all())
        assert not bool(out[empty].any())
        assert bool(((out - o).abs() <= near_o)[~empty].all()), float(((out - o).abs() / near_o.clamp(min=1e-30)).max())
        assert bool(((lse - l).abs() <= near_l)[~empty].all())


MIXES = [
    [(1, 0)], [(1, 1)], [(1, 777)], [(2, 0)], [(17, 3)], [(129, 0)], [(65, 100)],
    [(1, 5), (1, 600), (1, 31), (1, 0), (1, 64)],
    [(0, 40), (1, 9), (0, 0), (5, 0), (70, 41), (1, 255), (0, 3)],
]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("mix", range(len(MIXES)))
def test_attention_lengths(P, kind, dim, mix):
    Case(P, kind, 2, 4, dim, 16, MIXES[mix], seed=mix).check()


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
@pytest.mark.parametrize("heads,group", [(1, 1), (3, 1), (2, 3), (1, 7), (1, 8), (1, 16), (1, 20)])
def test_attention_head_groups(P, kind, heads, group):
    Case(P, kind, heads, group, 64, 16, [(1, 50), (7, 30), (40, 0)], seed=group).check()


@pytest.mark.parametrize("byte", [0, 1, 252, 253, 254, 255])
def test_four_bit_exponents_at_the_ends(P, byte):
    """Values of the smallest and largest exponents; from 253 on, NaN: read, and attended to."""
    cache = P.PagedCache(1, 1, 64, 2, 16, "mxfp4")
    codes = torch.full((2, 2, 16 * 32), 0x21, dtype=torch.uint8)  # pairs of 0.5, 1
    plane = torch.cat([codes, torch.full((2, 2, 32), 127, dtype=torch.uint8)], dim=2)
    plane[1, 0, 512:] = byte  # V, block 0
    cache.data.copy_(plane.flatten().cuda())
    slots = torch.arange(16, device="cuda")
    v = cache.read(0, slots)[1].double().cpu()
    want = torch.tensor([0.5, 1.0], dtype=torch.float64).repeat(32) * 2.0 ** (byte - 127)
    bad = byte >= 253
    assert bool(v.isnan().all()) if bad else torch.equal(v, want.expand(16, 1, 64))
    for n in (1, 40):  # few rows, and many
        q = torch.zeros((n, 1, 64), dtype=torch.bfloat16, device="cuda")
        off = torch.tensor([0, n], device="cuda")
        out = cache.attend(0, q, off, torch.tensor([15], dtype=torch.int32, device="cuda"),
                           torch.tensor([[0]], dtype=torch.int32, device="cuda")).double().cpu()
        if bad:
            assert bool(out.isnan().all())
        else:  # a mean of equal values; the smallest are below bf16's normal range
            assert bool(((out - want).abs() <= 2.0 ** -7 * want + 2.0 ** -126).all())


@pytest.mark.parametrize("kind", ["fp16", "mxfp4"])
@pytest.mark.parametrize("page", [1, 2, 5, 8, 24, 33, 64])
def test_attention_page_sizes(P, kind, page):
    Case(P, kind, 2, 4, 128, page, [(1, 200), (45, 90), (3, 1)], seed=page).check()


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
def test_attention_long(P, kind):
    """Many parts to a request, and a request of one beside it."""
    Case(P, kind, 1, 4, 128, 16, [(1, 5000), (1, 3), (2, 2600)], seed=5).check()


@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 64), ("mxfp4", 128)])
@pytest.mark.parametrize("group,reqs", [
    (1, [(1, 9000)]), (8, [(1, 40000)]), (16, [(1, 20000), (1, 100)]), (5, [(3, 30000)]), (8, [(4, 6000), (2, 70)])])
def test_attention_many_parts(P, kind, dim, group, reqs):
    """Tiles of 1 to 16 rows whose parts are joined from a few to hundreds of shares."""
    Case(P, kind, 1, group, dim, 16, reqs, seed=23).check()


@pytest.mark.parametrize("n", [1, 90])
def test_attention_half_precision_tail(P, n):
    """One key of nearly all the weight and value 0, thousands of 2^-26 of it and value 64: their
    part of the output is kept, though a 16-bit float has no weight that small. Its steps
    below 2^-14 are 2^-24: a weight of 2^-19 is off by 2^-6 of itself at most."""
    past, dim, page = 3000, 64, 16
    blocks = (past + n + page - 1) // page
    cache = P.PagedCache(1, 1, dim, blocks, page, "fp16")
    slots = torch.arange(blocks * page, device="cuda")
    k = torch.zeros((blocks * page, 1, dim), dtype=torch.float16, device="cuda")
    v = torch.full_like(k, 64.0)
    k[0, 0, 0], v[0] = 16.0, 0.0
    cache.append(0, k, v, slots)
    q = torch.zeros((n, 4, dim), dtype=torch.float16, device="cuda")
    q[..., 0] = 1.125  # 18 nats, 2^25.97
    ctx = torch.tensor([past], dtype=torch.int32, device="cuda")
    table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
    out = cache.attend(0, q, torch.tensor([0, n], device="cuda"), ctx, table, scale=1.0).double().cpu()
    tail = torch.arange(past, past + n, dtype=torch.float64)[:, None, None]
    want = 64 * tail / (tail + np.exp(18.0))
    assert bool(((out - want).abs() <= (2.0 ** -6 + 2.0 ** -10) * want).all())


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_attention_prompts(P, kind):
    """Whole prompts and prompts behind a prefix, over several tiles of rows."""
    Case(P, kind, 1, 4, 128, 16, [(150, 0), (1, 0), (97, 333), (64, 64)], seed=6).check()


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_attention_mixed_batch(P, kind):
    """Single tokens behind long contexts beside prompts: a batch of both kernels' requests."""
    Case(P, kind, 1, 4, 64, 16, [(1, 8300), (150, 40), (1, 3), (8, 100), (9, 100), (0, 5), (40, 0)], seed=17).check()


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_attention_single_tokens_and_a_prompt(P, kind):
    """Few rows a request on average, but a prompt among them: both kernels' requests again."""
    reqs = [(1, 8300), (140, 33)] + [(1, 3 * i) for i in range(30)]
    Case(P, kind, 2, 4, 64, 16, reqs, seed=20).check()
    Case(P, kind, 2, 4, 64, 16, reqs[::-1], seed=21).check()


@pytest.mark.parametrize("new,past", [(130, 900), (300, 0), (513, 70)])
def test_attention_prompt_in_parts(P, new, past):
    """Few tiles, whose keys are split: one request, and several."""
    Case(P, "bf16", 1, 2, 128, 16, [(new, past)], seed=18).check()
    Case(P, "fp16", 2, 1, 64, 16, [(new, past), (90, past + 33)], seed=19).check()


@pytest.mark.parametrize("kind", ["fp16", "mxfp4"])
@pytest.mark.parametrize("requests", [24, 33, 40])
def test_attention_last_turn_in_parts(P, kind, requests):
    """More tiles than run at once: those of the last turn are split, or not."""
    Case(P, kind, 8, 1, 64, 16, [(300, 1000)] + [(300, 7 * i) for i in range(requests - 1)], seed=22).check()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_attention_large_scores(P, kind):
    """Scores in the hundreds: one key takes nearly all the weight, in either order."""
    Case(P, kind, 1, 4, 64, 16, [(1, 300), (90, 10)], seed=7, scale=4.0, spread=3.0).check()


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_attention_missing_pages(P, kind):
    """Pages that are not there, by a negative entry or one past the cache; a request
    without any page sees nothing."""
    holes = [(0, 1, -1), (0, 3, 1 << 25), (1, 0, -5), (2, 0, -1), (2, 1, -1), (2, 2, -1)]
    Case(P, kind, 2, 4, 64, 16, [(1, 90), (40, 3), (30, 10)], seed=8, holes=holes, poison=False).check()


def test_attention_no_room_and_negative_context(P):
    """Positions past the table's width or before the start: rows that see fewer keys, or none."""
    c = Case(P, "bf16", 2, 2, 64, 16, [(30, 0), (30, 20), (1, 40)], seed=9, extra=0, poison=False)
    c.table = c.table[:, :2].contiguous()  # keys 0..31 alone
    c.ctx = torch.tensor([-10, 20, 40], dtype=torch.int32)
    c.check()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("reqs", [[(6, 33)], [(150, 20)]])
def test_attention_hidden_keys_never_reach_a_row(P, kind, reqs):
    """A NaN or an infinity in a later token's K and V: earlier rows are as without it."""
    c = Case(P, kind, 2, 4, 64, 16, reqs, seed=10)
    n, past = reqs[0]
    o, lse = c.run()
    for bad in (float("nan"), float("inf"), -float("inf")):
        c2 = Case(P, kind, 2, 4, 64, 16, reqs, seed=10)
        at = past + n - 2  # the last but one token
        slot = torch.tensor([int(c2.table[0, at // 16]) * 16 + at % 16], device="cuda")
        row = torch.full((1, 2, 64), bad, dtype=c2.cache.dtype, device="cuda")
        c2.cache.append(0, row, row, slot)
        o2, lse2 = c2.run()
        tol, tol_l = ref.bounds(*[x for i, x in enumerate(c.want()) if i != 1], 64, c.half)
        assert not bool(o2[:n - 2].isnan().any())
        assert bool(((o2 - o).double().cpu().abs() <= 2 * tol)[:n - 2].all())
        assert bool(((lse2 - lse).double().cpu().abs() <= 2 * tol_l)[:n - 2].all())
        if bad != -float("inf"):
            assert bool(o2[n - 2:].isnan().any())  # rows that see it say so


def test_attention_nan_query_is_its_own_rows(P):
    c = Case(P, "bf16", 1, 4, 64, 16, [(40, 9)], seed=11)
    o, _ = c.run()
    c.q[17, 2] = float("nan")
    o2, _ = c.run()
    assert bool(o2[17, 2].isnan().all())
    keep = torch.ones((40, 4), dtype=torch.bool)
    keep[17, 2] = False
    assert torch.equal(o2.cpu()[keep], o.cpu()[keep])


def test_attention_strides_and_outputs(P):
    """Rows of a wider tensor, head-major order, an output of the caller's; every element outside kept."""
    c = Case(P, "bf16", 2, 2, 64, 16, [(20, 30), (3, 0)], seed=12)
    o, lse = c.check()
    n = c.q.shape[0]
    wide = torch.zeros((n, 9, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:7] = c.q.cuda()
    major = c.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    for q in (wide[:, 3:7], major):
        out = torch.full((4, n, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        buf = torch.full((n, 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        for dst in (out.transpose(0, 1), buf[:, 1:5]):
            c.cache.attend(0, q, c.off.cuda(), c.ctx.cuda(), c.table.cuda(), out=dst)
            assert torch.equal(dst, o)
        assert bool((buf[:, 0] == 7).all()) and bool((buf[:, 5] == 7).all())


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_attention_past_four_gigabytes(P, kind):
    """Blocks whose bytes lie past 2^32 of a plane."""
    heads, dim, page = 8, 128, 16
    slab = P.ptstore_kv_slab_bytes({"bf16": 0, "mxfp4": 2}[kind], heads, dim, page)
    blocks = (1 << 32) // slab + 40
    cache = P.PagedCache(1, heads, dim, blocks, kind=kind)
    ids = torch.tensor([[blocks - 1, 3, blocks - 7, blocks - 20]], dtype=torch.int32, device="cuda")
    small = P.PagedCache(1, heads, dim, 4, kind=kind)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((64, heads, dim), device="cuda", generator=g).bfloat16() for _ in range(2))
    t = torch.arange(64, device="cuda")
    cache.append(0, k, v, ids[0].long()[t // 16] * 16 + t % 16)
    small.append(0, k, v, t)
    for n, past in ((1, 60), (50, 10)):
        q = torch.randn((n, 32, dim), device="cuda", generator=g).bfloat16()
        off = torch.tensor([0, n], device="cuda")
        ctx = torch.tensor([past], dtype=torch.int32, device="cuda")
        a = cache.attend(0, q, off, ctx, ids)
        b = small.attend(0, q, off, ctx, torch.arange(4, dtype=torch.int32, device="cuda")[None])
        assert torch.equal(a, b)


@pytest.mark.parametrize("reqs", [[(1, 3000), (1, 40)], [(200, 70), (3, 9)]])
def test_attention_in_a_graph(P, reqs):
    """Captured once, replayed on changed inputs, eager work between the replays."""
    c = Case(P, "bf16", 2, 4, 128, 16, reqs, seed=13)
    q, off, ctx, table = c.q.cuda(), c.off.cuda(), c.ctx.cuda(), c.table.cuda()
    ws = torch.empty(P.ptstore_attention_workspace(c.cache.layer(0)) + 16,
                     dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    c.cache.attend(0, q, off, ctx, table, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.attend(0, q, off, ctx, table, out=out, workspace=ws)
    for i in range(4):
        q.copy_(torch.randn_like(q))
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.cache.attend(0, q, off, ctx, table))


def test_attention_first_call_in_a_graph(P):
    """A cache whose first attention is captured: replays and later eager calls agree."""
    c = Case(P, "bf16", 2, 4, 128, 16, [(1, 3000), (1, 40)], seed=13)
    q, off, ctx, table = c.q.cuda(), c.off.cuda(), c.ctx.cuda(), c.table.cuda()
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.attend(0, q, off, ctx, table, out=out)
    for i in range(4):
        q.copy_(torch.randn_like(q))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.cache.attend(0, q, off, ctx, table))


def test_attention_graph_of_a_used_stream(P):
    """A graph captured on a stream whose workspace the cache has: replayed on another
    stream beside calls on that one, both right."""
    c = Case(P, "bf16", 2, 4, 128, 16, [(1, 6000), (1, 5000)], seed=13)
    q, off, ctx, table = c.q.cuda(), c.off.cuda(), c.ctx.cuda(), c.table.cuda()
    q2 = torch.randn_like(q)
    out = torch.empty_like(q)
    want, want2 = c.cache.attend(0, q, off, ctx, table), c.cache.attend(0, q2, off, ctx, table)
    s = torch.cuda.Stream()
    c.cache.attend(0, q, off, ctx, table, out=out, stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c.cache.attend(0, q, off, ctx, table, out=out)
    for i in range(4):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        others = [c.cache.attend(0, q2, off, ctx, table, stream=s) for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(o, want2) for o in others)


def test_attention_on_other_streams(P):
    """Two streams at once, by stream and by raw handle, each with its own workspace."""
    c = Case(P, "bf16", 2, 4, 128, 16, [(1, 4000), (1, 3500)], seed=14)
    args = (0, c.q.cuda(), c.off.cuda(), c.ctx.cuda(), c.table.cuda())
    want = c.cache.attend(*args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for i in range(12):
        s = streams[i % 3]
        outs.append(c.cache.attend(*args, stream=s if i % 2 else s.cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_attention_same_bits_each_time(P):
    for reqs in ([(1, 3000), (1, 700)], [(300, 50)]):
        c = Case(P, "mxfp4", 2, 4, 128, 16, reqs, seed=15)
        (o, l), (o2, l2) = c.run(), c.run()
        assert torch.equal(o, o2) and torch.equal(l, l2)


# --- refusals -------------------------------------------------------------------


def test_refusals(P):
    c = Case(P, "bf16", 2, 4, 64, 16, [(3, 5)], seed=16)
    q, off, ctx, table = c.q.cuda(), c.off.cuda(), c.ctx.cuda(), c.table.cuda()
    kv = c.cache.layer(0)
    out = torch.empty_like(q)

    def refused(match, f, error=P.PTStoreError):
        with pytest.raises(error, match=match):
            f()

    refused("multiple of the cache's heads", lambda: c.cache.attend(0, q[:, :7], off, ctx, table))
    refused("scale", lambda: c.cache.attend(0, q, off, ctx, table, scale=0.0))
    refused("scale", lambda: c.cache.attend(0, q, off, ctx, table, scale=float("nan")))
    refused("torch.bfloat16", lambda: c.cache.attend(0, q.half(), off, ctx, table), ValueError)
    refused("shape", lambda: c.cache.attend(0, torch.empty((3, 8, 128), dtype=q.dtype, device="cuda"), off, ctx, table), ValueError)
    refused("contiguous", lambda: c.cache.attend(0, torch.empty((3, 8, 128), dtype=q.dtype, device="cuda")[..., ::2], off, ctx, table), ValueError)
    odd = torch.empty((3 * 8 * 64 + 1,), dtype=q.dtype, device="cuda")[1:].view(3, 8, 64)
    refused("16-byte", lambda: c.cache.attend(0, odd, off, ctx, table))
    refused("rows", lambda: c.cache.attend(0, q, off, ctx, table[:0]), ValueError)
    refused("context holds", lambda: c.cache.attend(0, q, off, ctx[:0], table), ValueError)
    refused("kind", lambda: P.PagedCache(1, 2, 64, 4, kind="int8"), ValueError)
    refused("slab", lambda: P.PagedCache(1, 2, 80, 4))
    refused("bytes", lambda: P.PagedCache(1, 2, 64, 4, data=c.cache.data[:100]), ValueError)
    k = torch.zeros((4, 2, 64), dtype=q.dtype, device="cuda")
    s = torch.zeros(4, dtype=torch.int64, device="cuda")
    refused("slots 3", lambda: c.cache.append(0, k, k, s[:3]), ValueError)
    refused("int64", lambda: c.cache.append(0, k, k, s.int()), ValueError)
    empty = P.PagedCache(1, 2, 64, 0)
    one_row = (kv, q[:1], out[:1], None, torch.tensor([0, 1], device="cuda"), ctx, table, 1.0)
    refused("workspace", lambda: P.ptstore_attention(*one_row, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda")))
    refused("no blocks", lambda: empty.attend(0, q, off, ctx, table))
    # nothing to do is no error
    assert c.cache.attend(0, q[:0], torch.zeros(2, dtype=torch.int64, device="cuda"), ctx, table).shape[0] == 0
    c.cache.append(0, k[:0], k[:0], s[:0])
    held = torch.zeros(1, dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int64, device="cuda")
    free = torch.arange(4, dtype=torch.int32, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    refused("held_out", lambda: P.ptstore_block_tables(off, ctx, held, 16, free, None, table, slots, None, held, one))
    refused("next", lambda: P.ptstore_block_tables(off, ctx, None, 16, free, one, table, slots, None, held, one))
    refused("range", lambda: P.ptstore_block_tables(off, ctx, None, 65, free, None, table, slots, None, held, one))
    torch.cuda.synchronize()
    del out
