"""The paged cache's calls on the host: struct layouts, slab sizes, refusals without a GPU."""
from __future__ import annotations

import ctypes as C
import os
import re

import pytest

from test_abi import HEADER, _c_layout


@pytest.fixture(scope="module")
def P():
    from paper_2607_22648_amd import ptstore
    return ptstore


def test_struct_layouts_match_header(P, tmp_path):
    for cls, name in ((P.ptstore_kv_t, "ptstore_kv_t"), (P.ptstore_attention_t, "ptstore_attention_t")):
        fields = [f for f, _ in cls._fields_]
        size, offs = _c_layout(tmp_path, name, fields)
        assert C.sizeof(cls) == size, name
        assert [getattr(cls, f).offset for f in fields] == offs, name


def test_kinds_match_header(P):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    kinds = {n: int(v) for n, v in re.findall(r"\b(PTSTORE_KV_[A-Z0-9]+)\s*=\s*(\d+)", text)}
    assert len(kinds) == 3 and all(getattr(P, n) == v for n, v in kinds.items())


def test_slab_bytes(P):
    assert P.ptstore_kv_slab_bytes(P.PTSTORE_KV_BF16, 8, 128, 16) == 8 * 16 * 128 * 2
    assert P.ptstore_kv_slab_bytes(P.PTSTORE_KV_MXFP4, 8, 128, 16) == 8 * 16 * (64 + 4)
    assert P.ptstore_kv_slab_bytes(P.PTSTORE_KV_MXFP4, 1, 64, 1) == 48  # 34, padded
    for bad in ((3, 8, 128, 16), (0, 0, 128, 16), (0, 8, 80, 16), (0, 8, 128, 65), (0, 8, 128, 0),
                (0, 1 << 20, 128, 64)):
        with pytest.raises(P.PTStoreError):
            P.ptstore_kv_slab_bytes(*bad)


def test_attention_refuses_on_the_host(P):
    """Every check that needs no device comes before any HIP call."""
    lib = P.lib()
    text = lambda: lib.ptstore_last_error().decode()  # noqa: E731
    a = P.ptstore_attention_t()
    assert lib.ptstore_attention(None, None) == P.PTSTORE_ERR_INVALID
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "kind" in text()
    a.kv = P.ptstore_kv_t(0x1000, 0x2000, 4, 2, 64, 16, 0)
    a.q_heads, a.R, a.max_blocks, a.n_tokens, a.scale = 3, 1, 4, 1, 1.0
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "multiple" in text()
    a.q_heads, a.scale = 4, float("inf")
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "scale" in text()
    a.scale, a.max_blocks = 1.0, (1 << 26) + 1
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "2^30" in text()
    a.max_blocks, a.n_tokens = 4, 1 << 29
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "2^31" in text()
    a.n_tokens, a.R = 1, 0
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "out of range" in text()
    a.R = 1
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "null" in text()
    a.offsets = a.context = a.block_table = 0x1000
    a.q, a.out = 0x1008, 0x1000
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "16-byte" in text()
    a.kv.k = 0x1004
    assert lib.ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID and "planes" in text()
    kv = P.ptstore_kv_t(0x1000, 0x2000, (1 << 30) + 1, 2, 64, 16, 0)
    with pytest.raises(P.PTStoreError, match="2\\^30"):
        P.ptstore_attention_workspace(kv)
    kv.cache_blocks = (1 << 36) // 4096 + 1
    with pytest.raises(P.PTStoreError, match="64 GiB"):
        P.ptstore_attention_workspace(kv)
    assert lib.ptstore_kv_append(C.byref(kv), 1, 1, 1, 1, 1, 1, 1, 1, None) == P.PTSTORE_ERR_INVALID
    assert lib.ptstore_kv_append(None, 1, 1, 1, 1, 1, 1, 1, 1, None) == P.PTSTORE_ERR_INVALID
    assert os.path.exists(HEADER)
