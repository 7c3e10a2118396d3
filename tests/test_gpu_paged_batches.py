"""Attention over batches of many requests, and over tiles whose keys are split (MI355X)."""
from __future__ import annotations

import math

import pytest
import torch

from test_gpu_paged import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


class Batch(Case):
    """A case whose 64-bit answer is formed a request at a time, all its rows and heads at once."""

    def want(self):
        n, q_heads, dim = self.q.shape
        kv_heads = self.kv[0].shape[1]
        out, mean = (torch.zeros((n, q_heads, dim), dtype=torch.float64) for _ in range(2))
        lse = torch.full((n, q_heads), -math.inf, dtype=torch.float64)
        reach = torch.zeros((n, q_heads), dtype=torch.float64)
        off, ctx = self.off.tolist(), self.ctx.tolist()
        for r, (a, b) in enumerate(zip(off, off[1:])):
            end = ctx[r] + b - a
            if b == a or end <= 0:
                continue
            rows = self.table[r, :-(-end // self.page)].long()
            k, v = (x[rows].transpose(0, 1).flatten(1, 2)[:, :end] for x in self.kv)  # [heads, keys, dim]
            q = self.q[a:b].double().view(b - a, kv_heads, -1, dim).permute(1, 2, 0, 3)  # [heads, group, n, dim]
            k, v = k[:, None], v[:, None]
            hidden = torch.arange(end) > ctx[r] + torch.arange(b - a)[:, None]
            s = (torch.matmul(q, k.transpose(2, 3)) * self.scale).masked_fill(hidden, -math.inf)
            size = torch.matmul(q.abs(), k.abs().transpose(2, 3)).masked_fill(hidden, 0.0) * self.scale
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top)
            total = w.sum(-1, keepdim=True)
            for to, x in ((out, torch.matmul(w, v) / total), (mean, torch.matmul(w, v.abs()) / total)):
                to[a:b] = x.permute(2, 0, 1, 3).reshape(b - a, q_heads, dim)
            for to, x in ((lse, (top + total.log())[..., 0]), (reach, size.amax(-1))):
                to[a:b] = x.permute(2, 0, 1).reshape(b - a, q_heads)
        return out, lse, mean, reach


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
@pytest.mark.parametrize("requests", [64, 65, 257, 513, 1100, 4200])
def test_many_requests_of_few_rows(P, kind, requests):
    """None, one or two tokens each, behind up to 70."""
    Batch(P, kind, 1, 2, 64, 16, [((i * 7) % 3, (i * 13) % 71) for i in range(requests)], seed=requests).check()


@pytest.mark.parametrize("kind", ["fp16", "mxfp4"])
@pytest.mark.parametrize("requests", [64, 65, 257, 513, 4200])
def test_many_requests_of_many_rows(P, kind, requests):
    """None to nine tokens each, of 16 query heads: 72 rows a request on average."""
    reqs = [((i * 7) % 10, (i * 13) % 41) for i in range(requests)]
    Batch(P, kind, 1, 16, 64, 16, reqs, seed=requests).check()


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
@pytest.mark.parametrize("requests", [65, 513, 4200])
def test_many_requests_of_both_kinds(P, kind, requests):
    """Few rows and many, in a table with room for 8,192 keys: each kernel finds its own."""
    reqs = [(40 if i % 9 == 4 else (i * 7) % 4, (i * 13) % 41) for i in range(requests)]
    Batch(P, kind, 1, 4, 64, 16, reqs, seed=requests, extra=512).check()


def parts_written(P, c):
    """Runs and checks a case with a marked workspace; how many of its bytes were written."""
    ws = torch.full((P.ptstore_attention_workspace(c.cache.layer(0)),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = c.run(workspace=ws)  # the marks are NaN: what is read unwritten shows
    c.compare(out, lse)
    return int((ws != 0xFF).sum())


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("reqs", [[(70, 2000)], [(130, 3900)], [(40, 2600), (33, 2100), (90, 700)]])
def test_prompts_whose_keys_are_split(P, kind, dim, reqs):
    """Fewer tiles than the device holds, behind keys enough for two parts or more."""
    c = Batch(P, kind, 2, 4, dim, 16, reqs, seed=dim)
    rows = 2 * 4 * sum(a for a, _ in reqs)
    assert parts_written(P, c) > 1.9 * rows * dim * 4  # two parts of every row


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
@pytest.mark.parametrize("dim", [64, 128])
def test_parts_that_have_no_keys(P, kind, dim):
    """A table far wider than its requests: more parts than a tile has steps of keys."""
    c = Batch(P, kind, 1, 4, dim, 16, [(70, 300), (40, 0)], seed=dim, extra=1500)
    assert parts_written(P, c) > 1.9 * 4 * 110 * dim * 4


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
def test_last_turn_of_wide_rows_in_parts(P, kind):
    """More tiles of 128 dimensions than run at once, the last ones split."""
    reqs = [(300, 1000)] + [(300, 7 * i) for i in range(24)]
    c = Batch(P, kind, 8, 1, 128, 16, reqs, seed=22)
    assert 0 < parts_written(P, c) < 2 * 8 * 25 * 300 * 128 * 4


def test_whole_prompts_write_no_parts(P):
    assert parts_written(P, Batch(P, "bf16", 2, 4, 128, 16, [(130, 300)], seed=3)) == 0
