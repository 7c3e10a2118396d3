"""An attention whose output is its input is refused on the host (CPU; every pointer is made up)."""
from __future__ import annotations

import ctypes as C

from paper_2607_22648_amd import ptstore as P


def test_out_must_not_be_q():
    """No order is promised between one row's output and the reads of another's queries. With equal
    strides and with others."""
    a = P.ptstore_attention_t()
    a.kv = P.ptstore_kv_t(0x1000, 0x2000, 4, 2, 64, 16, P.PTSTORE_KV_BF16)
    a.q_heads, a.R, a.max_blocks, a.n_tokens, a.scale = 4, 1, 4, 1, 1.0
    a.q = a.out = a.offsets = a.context = a.block_table = 0x1000
    for a.out_token_stride, a.out_head_stride in ((0, 0), (256, 64)):
        assert P.lib().ptstore_attention(C.byref(a), None) == P.PTSTORE_ERR_INVALID
        assert "out must not be q" in P.lib().ptstore_last_error().decode()
