"""Latent caches: rows, and attention in the latent space, against 64 bits (MI355X)."""
from __future__ import annotations

import math

import pytest
import torch

import latent_ref as ref

pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


def make(P, kind, latent, blocks, page, seed, layers=1):
    cache = P.LatentCache(layers, latent, 64, blocks, block_tokens=page, kind=kind)
    planes = cache.data.view(DTYPE[kind]).view(-1, blocks, page, latent + 64)
    planes.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
    return cache, planes


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("latent,page,n", [(512, 16, 1), (512, 24, 333), (256, 1, 50), (256, 64, 129), (512, 16, 0)])
def test_rows(P, kind, latent, page, n):
    blocks = n // page + 3
    cache, planes = make(P, kind, latent, blocks, page, 5, layers=3)
    before = planes.clone()
    assert planes.shape[0] == 4  # an odd number of layers has room for one more
    both = torch.randn((n, latent + 72), device="cuda").to(DTYPE[kind])
    rope, c = both[:, :64], both[:, 72:]  # strided rows
    slots = torch.randperm(blocks * page, device="cuda")[:n]
    if n > 8:
        slots[3], slots[5], slots[7] = -1, blocks * page, 1 << 40
    cache.append(1, c, rope, slots)
    ok = (slots >= 0) & (slots < blocks * page)
    before[1].view(-1, latent + 64)[slots[ok]] = torch.cat((c, rope), 1)[ok]
    assert torch.equal(planes, before)
    got_c, got_rope = cache.read(1, slots)
    assert torch.equal(got_c[ok], c[ok]) and torch.equal(got_rope[ok], rope[ok])
    assert not bool(got_c[~ok].any()) and not bool(got_rope[~ok].any())


def check(P, kind, latent, page, heads, new, past, seed=0, scale=None, hole=False, qscale=1.0, stride=False, wide=0):
    offsets, context, table, blocks = ref.batch(seed, new, past, page, hole=hole)
    if wide:
        table = torch.cat((table, torch.full((len(new), wide), -1, dtype=torch.int32)), 1)
    cache, planes = make(P, kind, latent, blocks, page, seed)
    n = int(offsets[-1])
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((n, heads, latent + 64), generator=g) * qscale).to(DTYPE[kind])
    scale = (latent + 64) ** -0.5 if scale is None else scale
    want, lse, mean, reach = ref.attention(q.double(), planes[0].cpu().double(), offsets, context, table, page, scale)
    d = q.cuda()
    ql, qr = d[..., :latent], d[..., latent:]
    out = None
    if stride:
        ql, qr = ql.contiguous(), qr.contiguous()
        out = torch.full((heads, n, latent + 8), 7.0, dtype=DTYPE[kind], device="cuda")[..., :latent].transpose(0, 1)
    got, sums = cache.attend(0, ql, qr, offsets.cuda(), context.cuda(), table.cuda(), scale, out=out, lse=True)
    tol, ltol = ref.bounds(want, mean, reach, latent + 64, kind == "fp16")
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    sums = sums.cpu().double()
    none = lse == -math.inf
    assert torch.equal(sums == -math.inf, none)
    assert bool(((sums - lse).abs()[~none] <= (ltol + lse.abs() * 2.0 ** -22)[~none]).all())
    again = cache.attend(0, ql, qr, offsets.cuda(), context.cuda(), table.cuda(), scale)
    assert torch.equal(again, got)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads,new,past", [
    (16, [1], [0]), (16, [1], [31]), (16, [1], [32]), (16, [1], [777]), (1, [1, 1, 0, 1], [5, 64, 9, 0]),
    (20, [1, 3, 2], [100, 33, 257]), (128, [1, 1, 2], [40, 300, 95]), (64, [4, 1], [63, 0]), (33, [70], [11]),
    (130, [3], [50])])
def test_absorbed(P, kind, latent, heads, new, past):
    check(P, kind, latent, 16, heads, new, past, seed=heads + len(new))


@pytest.mark.parametrize("page", [1, 7, 24, 64])
def test_absorbed_pages(P, page):
    check(P, "bf16", 512, page, 16, [1, 2, 1], [130, 63, 300], seed=page, hole=page != 64)


def test_absorbed_strided_and_wide(P):
    check(P, "bf16", 512, 16, 24, [2, 1], [50, 200], seed=3, stride=True, wide=500)


def test_absorbed_split_requests(P):
    """Long requests: tiles whose keys many workgroups share, and several tiles a workgroup."""
    check(P, "bf16", 512, 16, 2, [1], [30000], seed=4)
    check(P, "fp16", 256, 16, 1, [1] * 40, [37 * i for i in range(40)], seed=5)
    check(P, "bf16", 512, 16, 4, [1] * 600, [i % 50 for i in range(600)], seed=6)


def test_absorbed_short_requests(P):
    """Tiles that are not cut beside some that are, at the sizes where that begins."""
    check(P, "bf16", 256, 16, 33, [2, 1, 3, 1, 2, 4], [126, 127, 128, 30, 500, 95], seed=11)
    check(P, "fp16", 512, 16, 16, [1] * 9, [126, 127, 128, 129, 255, 0, 600, 127, 1000], seed=12)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_absorbed_sharp_scores(P, kind):
    """Scores of tens to hundreds: nearly all the weight on one key, maxima that rise by much."""
    check(P, kind, 512, 16, 16, [1, 3], [500, 129], seed=7, scale=0.5, qscale=3.0)


def test_absorbed_holes_and_nothing(P):
    """Missing pages within a request, a request without any page, an empty batch."""
    check(P, "bf16", 512, 16, 16, [1, 5], [400, 70], seed=8, hole=True)
    cache, _ = make(P, "bf16", 512, 4, 16, 9)
    q = torch.randn((2, 16, 576), device="cuda").bfloat16()
    off = torch.tensor([0, 1, 2], device="cuda")
    out, lse = cache.attend(0, q[..., :512], q[..., 512:], off, torch.tensor([40, -3], dtype=torch.int32, device="cuda"),
                            torch.full((2, 3), -1, dtype=torch.int32, device="cuda"), 0.1, lse=True)
    assert not bool(out.any()) and bool((lse == -math.inf).all())
    none = cache.attend(0, q[:0, :, :512], q[:0, :, 512:], off[:1], off[:0].int(), torch.zeros((0, 1), dtype=torch.int32,
                                                                                             device="cuda"), 0.1)
    assert none.shape == (0, 16, 512)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_absorbed_hidden_values_are_not_seen(P, bad):
    """Infinities and NaN in slots behind the last key, in missing pages' neighbours, and in a draft's
    later tokens: rows that do not see them are as without them, rows that do have them."""
    latent, page, heads = 512, 16, 16
    offsets, context, table, blocks = ref.batch(3, [3, 1], [45, 20], page)
    cache, planes = make(P, "bf16", latent, blocks, page, 3)
    q = torch.randn((4, heads, 576), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    args = (offsets.cuda(), context.cuda(), table.cuda(), 576 ** -0.5)
    clean = cache.attend(0, q[..., :latent], q[..., latent:], *args)
    flat = planes[0]
    used = torch.zeros((blocks, page), dtype=torch.bool)
    for r in range(2):
        pos, block, slot = ref.keys_of(r, offsets, context, table, page, blocks)
        used[block, slot] = True
    flat[~used.cuda()] = bad
    got = cache.attend(0, q[..., :latent], q[..., latent:], *args)
    assert torch.equal(got, clean)
    flat[table[0, 47 // page].item(), 47 % page, 100] = bad  # the last of the three new tokens
    got = cache.attend(0, q[..., :latent], q[..., latent:], *args)
    assert torch.equal(got[[0, 1, 3]], clean[[0, 1, 3]])
    # its score is infinite or NaN for every head, so the row is NaN or, where minus infinity, that value's
    assert not bool(torch.isfinite(got[2, :, 100]).any())


# --- the expanded form ---------------------------------------------------------------


def expanded_bounds(want, mean, reach, q, rows, w, latent, scale, half):
    """As paged_ref.bounds, with what forming keys and values adds: the sum of `latent` products in 32 bits is off
    by latent 2^-24 of the sum of their magnitudes, and two 16-bit values leave u u of it (of an fp16 pair at
    least 2^-25 where the second is that small). Scores move by u u reach and by the keys' sums, outputs by
    u u |v| and the values'."""
    u = 2.0 ** -11 if half else 2.0 ** -8
    tiny = 2.0 ** -25 if half else 0.0
    spread = float((rows[..., :latent].abs().amax((0, 1)) * w.abs().amax((0, 1))).sum())
    formed = latent * 2.0 ** -24 * spread + tiny
    d = reach * (u * u + 320 * 2.0 ** -24 + 2.0 ** -21) + q[..., :128].abs().sum(-1) * scale * formed + 2.0 ** -20
    tol = ((2 * torch.expm1(d)[..., None] + u + u * u + 2.0 ** -16) * mean * 1.02 + u * want.abs() + formed * 1.1
           + 2 * tiny)
    return tol, d + 2.0 ** -20


def check_expanded(P, kind, latent, page, heads, new, past, seed=0, hole=False, split=False, more=0, qscale=1.0):
    offsets, context, table, blocks = ref.batch(seed, new, past, page, hole=hole)
    cache, planes = make(P, kind, latent, blocks, page, seed)
    n, g = int(offsets[-1]), torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((n, heads, 192), generator=g) * qscale).to(DTYPE[kind])
    w = (torch.randn((heads, 256, latent), generator=g) * latent ** -0.5).to(DTYPE[kind])
    counts = torch.tensor([a + b + more for a, b in zip(new, past)])
    key_offsets = torch.zeros(len(new) + 1, dtype=torch.int64)
    key_offsets[1:] = counts.cumsum(0)
    scale = 192 ** -0.5
    wd, rows = w.double(), planes[0].cpu().double()
    want, lse, mean, reach = ref.attention(
        q.double(), rows, offsets, context, table, page, scale,
        k_of=lambda x, h: torch.cat((x[:, :latent] @ wd[h, :128].T, x[:, latent:]), 1),
        v_of=lambda x, h: x[:, :latent] @ wd[h, 128:].T)
    d, dw = q.cuda(), w.cuda()
    wk, wv = dw[:, :128], dw[:, 128:]
    out = None
    if split:
        wk, wv = wk.contiguous(), torch.cat((wv, wv), 2)[..., :latent]
        out = torch.full((n, heads, 256), 3.0, dtype=DTYPE[kind], device="cuda")[..., 128:]
    got, sums = cache.attend_expanded(0, d[..., :128], d[..., 128:], wk, wv, offsets.cuda(), context.cuda(),
                                      table.cuda(), key_offsets.cuda(), int(key_offsets[-1]), out=out, lse=True)
    tol, ltol = expanded_bounds(want, mean, reach, q.double(), rows, wd, latent, scale, kind == "fp16")
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    sums, none = sums.cpu().double(), lse == -math.inf
    assert torch.equal(sums == -math.inf, none)
    assert bool(((sums - lse).abs()[~none] <= (ltol + lse.abs() * 2.0 ** -22)[~none]).all())


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads,new,past", [
    (1, [1], [0]), (4, [65], [0]), (3, [33, 0, 130], [0, 7, 64]), (2, [1, 260], [200, 1]), (5, [128, 1], [128, 63])])
def test_expanded(P, kind, latent, heads, new, past):
    check_expanded(P, kind, latent, 16, heads, new, past, seed=heads)


@pytest.mark.parametrize("kind,latent,heads,new,past,hole", [
    ("bf16", 512, 7, [3, 40], [2400, 90], True), ("fp16", 256, 8, [1, 2, 0, 3], [1500, 300, 0, 500], False),
    ("bf16", 256, 33, [1, 2], [600, 20], True), ("fp16", 512, 16, [2], [1030], False),
    ("bf16", 256, 33, [1, 2, 0, 40, 7], [60, 20, 9, 0, 129], False),
    ("fp16", 256, 33, [1, 2, 0, 40, 7, 3, 1, 130, 1], [60, 20, 9, 0, 129, 5, 0, 31, 64], True)])
def test_expanded_many_keys(P, kind, latent, heads, new, past, hole):
    """More than 1,024 (32 keys, head, keys or values): 128 keys and pairs of heads a workgroup. The last two: more
    than 128 (128 tokens, head), tiles of 128 tokens by eight waves, and more than 256, by four."""
    check_expanded(P, kind, latent, 16, heads, new, past, seed=heads, hole=hole)


@pytest.mark.parametrize("page", [1, 7, 24, 64])
def test_expanded_pages_and_holes(P, page):
    check_expanded(P, "bf16", 512, page, 3, [40, 150], [100, 9], seed=page, hole=True)


def test_expanded_strided_and_spare_keys(P):
    check_expanded(P, "bf16", 512, 16, 4, [70, 20], [31, 0], seed=2, split=True, more=5)


def test_expanded_sharp_scores(P):
    check_expanded(P, "fp16", 256, 16, 2, [100], [50], seed=3, qscale=4.0)


def test_expanded_hidden_values_and_odd_offsets(P):
    """A later token's infinite row leaves the rows before it alone; a request whose key offsets fall or
    reach past n_keys, or give too few keys, has those only."""
    latent, page, heads = 512, 16, 2
    offsets, context, table, blocks = ref.batch(3, [140, 3], [45, 20], page)
    cache, planes = make(P, "bf16", latent, blocks, page, 3)
    g = torch.Generator().manual_seed(4)
    q = torch.randn((143, heads, 192), generator=g).bfloat16().cuda()
    w = (torch.randn((heads, 256, latent), generator=g) * latent ** -0.5).bfloat16().cuda()

    def call(key_offsets, n_keys):
        return cache.attend_expanded(0, q[..., :128], q[..., 128:], w[:, :128], w[:, 128:], offsets.cuda(),
                                     context.cuda(), table.cuda(), torch.tensor(key_offsets, device="cuda"), n_keys)
    clean = call([0, 185, 208], 208)
    pos = 45 + 100  # the 101st new token
    planes[0][int(table[0, pos // page]), pos % page, 7] = math.inf
    got = call([0, 185, 208], 208)
    assert torch.equal(got[:100], clean[:100]) and torch.equal(got[140:], clean[140:])
    assert not bool(torch.isfinite(got[100:140]).all(-1).any())
    for bad in ([0, 500, 208], [0, -5, 208], [0, 1 << 40, 208], [7, 185, 100]):
        odd = call(bad, 208)
        assert odd.shape == clean.shape
    few = call([0, 45, 68], 208)  # the past only, for the first request
    assert bool(torch.isfinite(few[:140]).all()) and torch.equal(few[140:], clean[140:])
