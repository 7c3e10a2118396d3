"""Calls of the paged cache that are too large for one launch: refused on the host, before any device
is asked for (CPU; every pointer here is made up)."""
from __future__ import annotations

import ctypes as C

import pytest

from paper_2607_22648_amd import ptstore as P


def refused(rc, *words):
    text = P.lib().ptstore_last_error().decode()
    assert rc == P.PTSTORE_ERR_INVALID and all(w in text for w in words), (rc, text)


@pytest.mark.parametrize("call", ["ptstore_kv_append", "ptstore_kv_read"])
@pytest.mark.parametrize("kind", [P.PTSTORE_KV_BF16, P.PTSTORE_KV_MXFP4])
@pytest.mark.parametrize("heads,dim,n", [
    (1, 128, (1 << 28) - 15), (8, 128, 1 << 25), (2, 64, 1 << 28), (1, 64, (1 << 29) - 31), (3, 128, 1 << 27),
    (8, 128, 1 << 61), (8, 64, (1 << 61) + 1), (2, 128, (1 << 63) - 1), (1, 64, 1 << 31)])
def test_rows_past_a_launch(call, kind, heads, dim, n):
    """From 2^32 work-items on, and products of sizes that leave 64 bits."""
    kv = P.ptstore_kv_t(0x1000, 0x2000, 4, heads, dim, 16, kind)
    rc = getattr(P.lib(), call)(C.byref(kv), 0x1000, 0, 0, 0x1000, 0, 0, 0x1000, n, None)
    refused(rc, call, "2^35")


def attention(heads, group, n, R, max_blocks=1, dim=64, page=1):
    a = P.ptstore_attention_t()
    a.kv = P.ptstore_kv_t(0x1000, 0x2000, 4, heads, dim, page, P.PTSTORE_KV_BF16)
    a.q_heads, a.R, a.max_blocks, a.n_tokens, a.scale = heads * group, R, max_blocks, n, 1.0
    a.q = a.out = a.offsets = a.context = a.block_table = 0x1000
    a.out = 0x3000
    return P.lib().ptstore_attention(C.byref(a), None)


@pytest.mark.parametrize("heads,group,n,R,max_blocks,page", [
    (8, 4, 9 << 21, 1 << 21, 1, 1),  # short prompts of many requests
    (1, 16, (1 << 27) - 8, 1 << 24, 1, 16),
    (8, 4, 1 << 22, 1 << 21, 128, 64)])  # few rows each, but room for 8,192 keys
def test_tiles_past_a_launch(heads, group, n, R, max_blocks, page):
    refused(attention(heads, group, n, R, max_blocks, page=page), "tiles")


def test_heads_past_a_launch():
    refused(attention(1 << 23, 1, 1, 1), "heads")


@pytest.mark.parametrize("heads,group,n", [(1, 1, (1 << 31) - 127), (1, 2, 1 << 30), (2, 1, (1 << 30) - 63)])
def test_rows_past_32_bits(heads, group, n):
    """Numbers of rows up to the end of a last tile."""
    refused(attention(heads, group, n, 1 << 20), "2^31")
