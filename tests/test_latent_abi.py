"""Latent caches, attention weights and eviction on the host: struct layouts, workspace sizes, refusals before
any device is asked for (CPU; every pointer here is made up)."""
from __future__ import annotations

import ctypes as C
from types import SimpleNamespace

import pytest
import torch

from paper_2607_22648_amd import ptstore as P
from test_abi import _c_layout

AT = 0x1000  # an aligned address that no call may reach


@pytest.mark.parametrize("name", ["ptstore_latent_t", "ptstore_latent_attention_t", "ptstore_latent_expanded_t",
                                  "ptstore_weigh_t", "ptstore_latent_weigh_t", "ptstore_evict_t"])
def test_struct_layouts_match_header(name, tmp_path):
    cls = getattr(P, name)
    fields = [f for f, _ in cls._fields_]
    size, offs = _c_layout(tmp_path, name, fields)
    assert C.sizeof(cls) == size
    assert [getattr(cls, f).offset for f in fields] == offs


def latent(**over):
    f = dict(rows=AT, cache_blocks=4, latent_dim=512, rope_dim=64, block_tokens=16, kind=P.PTSTORE_KV_BF16)
    f.update(over)
    return P.ptstore_latent_t(*f.values())


def refused(rc, *words):
    text = P.lib().ptstore_last_error().decode()
    assert rc == P.PTSTORE_ERR_INVALID and all(w in text for w in words), (rc, text)


BAD_CACHES = [(dict(kind=P.PTSTORE_KV_MXFP4), "kind"), (dict(latent_dim=384), "latent_dim"), (dict(rope_dim=32), "rope_dim"),
              (dict(block_tokens=0), "block_tokens"), (dict(block_tokens=65), "block_tokens"),
              (dict(cache_blocks=-1), "cache_blocks"), (dict(cache_blocks=(1 << 30) + 1), "cache_blocks"),
              (dict(cache_blocks=(1 << 36) // (16 * 1152) + 1), "64 GiB"), (dict(rows=AT + 8), "16-byte"),
              (dict(rows=None), "16-byte")]


@pytest.mark.parametrize("over,word", BAD_CACHES)
def test_caches_that_no_call_takes(over, word):
    cache, lib = latent(**over), P.lib()
    n = C.c_int64()
    refused(lib.ptstore_latent_append(C.byref(cache), AT, 512, AT, 64, AT, 1, None), "ptstore_latent_append", word)
    refused(lib.ptstore_latent_read(C.byref(cache), AT, 512, AT, 64, AT, 1, None), "ptstore_latent_read", word)
    refused(lib.ptstore_latent_attention_workspace(C.byref(cache), C.byref(n)), word)
    refused(lib.ptstore_latent_evict(C.byref(cache), C.byref(evict_args()), None), "ptstore_latent_evict", word)
    for args, call in ((attention_args(), lib.ptstore_latent_attention),
                       (expanded_args(), lib.ptstore_latent_attention_expanded), (latent_weigh_args(), lib.ptstore_latent_weigh)):
        args.cache = cache
        refused(call(C.byref(args), None), word)


def test_null_arguments():
    lib, n = P.lib(), C.c_int64()
    refused(lib.ptstore_latent_append(None, AT, 512, AT, 64, AT, 1, None), "null cache")
    refused(lib.ptstore_latent_attention(None, None), "null")
    refused(lib.ptstore_latent_attention_expanded(None, None), "null")
    refused(lib.ptstore_kv_weigh(None, None), "null")
    refused(lib.ptstore_latent_weigh(None, None), "null")
    refused(lib.ptstore_kv_evict(None, C.byref(evict_args()), None), "null")
    refused(lib.ptstore_latent_evict(C.byref(latent()), None, None), "null")
    refused(lib.ptstore_latent_attention_workspace(C.byref(latent()), None), "null")
    refused(lib.ptstore_latent_expanded_workspace(8, 100, None), "null")
    refused(lib.ptstore_weigh_workspace(1, None), "null")
    refused(lib.ptstore_evict_workspace(1, 1, 1, 1, None), "null")
    assert lib.ptstore_latent_expanded_workspace(8, 100, C.byref(n)) == 0


@pytest.mark.parametrize("call", ["ptstore_latent_append", "ptstore_latent_read"])
def test_rows_refused(call):
    fn, cache = getattr(P.lib(), call), latent()
    for a in ((None, 512, AT, 64, AT), (AT, 512, None, 64, AT), (AT, 512, AT, 64, None), (AT + 8, 512, AT, 64, AT),
              (AT, 516, AT, 64, AT), (AT, 512, AT, 68, AT), (AT, 512, AT + 2, 64, AT)):
        refused(fn(C.byref(cache), *a, 1, None), call)
    for n in (-1, (1 << 31) // 72 + 1, 1 << 62):
        refused(fn(C.byref(cache), AT, 512, AT, 64, AT, n, None), "2^34")
    assert fn(C.byref(cache), None, 0, None, 0, None, 0, None) == 0  # nothing to do


def attention_args(**over):
    a = P.ptstore_latent_attention_t(cache=latent(), q_latent=AT, q_latent_token_stride=4096, q_latent_head_stride=512,
                                     q_rope=AT + 16, q_rope_token_stride=512, q_rope_head_stride=64, out=AT + 32,
                                     out_token_stride=4096, out_head_stride=512, offsets=AT, context=AT, block_table=AT,
                                     n_tokens=2, R=1, max_blocks=4, heads=8, scale=0.1)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def expanded_args(**over):
    a = P.ptstore_latent_expanded_t(cache=latent(), q_nope=AT, q_nope_token_stride=1024, q_nope_head_stride=128,
                                    q_rope=AT + 16, q_rope_token_stride=512, q_rope_head_stride=64, w_k=AT, w_k_head_stride=65536,
                                    w_k_row_stride=512, w_v=AT, w_v_head_stride=65536, w_v_row_stride=512, out=AT + 32,
                                    out_token_stride=1024, out_head_stride=128, offsets=AT, context=AT, block_table=AT,
                                    key_offsets=AT, n_tokens=2, n_keys=50, R=1, max_blocks=4, heads=8, scale=0.1)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def weigh_args(**over):
    a = P.ptstore_weigh_t(kv=P.ptstore_kv_t(AT, 2 * AT, 4, 2, 64, 16, P.PTSTORE_KV_BF16), q=AT, q_token_stride=512,
                          q_head_stride=64, lse=AT, offsets=AT, context=AT, block_table=AT, n_tokens=2, R=1, max_blocks=4,
                          q_heads=8, scale=0.1, weights=AT)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def latent_weigh_args(**over):
    a = P.ptstore_latent_weigh_t(cache=latent(), q_latent=AT, q_latent_token_stride=4096, q_latent_head_stride=512,
                                 q_rope=AT, q_rope_token_stride=512, q_rope_head_stride=64, lse=AT, offsets=AT, context=AT,
                                 block_table=AT, n_tokens=2, R=1, max_blocks=4, heads=8, scale=0.1, weights=AT)
    for k, v in over.items():
        setattr(a, k, v)
    return a


BATCH = [(dict(R=0), "out of range"), (dict(R=-1), "out of range"), (dict(max_blocks=0), "out of range"),
         (dict(n_tokens=-1), "out of range"), (dict(R=1 << 20, max_blocks=1 << 10), "out of range"),
         (dict(max_blocks=(1 << 26) + 1), "2^30"), (dict(n_tokens=1 << 29), "2^31"), (dict(n_tokens=1 << 62), "2^31"),
         (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("inf")), "scale"),
         (dict(scale=float("nan")), "scale"), (dict(scale=3e38), "scale"),
         (dict(offsets=None), "null"), (dict(context=None), "null"), (dict(block_table=None), "null")]
QUERIES = [(dict(q_rope=None), "null"), (dict(q_rope=AT + 8), "16-byte"), (dict(q_rope_token_stride=4), "16-byte"),
           (dict(q_rope_head_stride=65), "16-byte")]


@pytest.mark.parametrize("over,word", BATCH + QUERIES + [
    (dict(heads=0), "heads"), (dict(heads=-1), "heads"), (dict(q_latent=None), "null"), (dict(q_latent=AT + 2), "16-byte"),
    (dict(q_latent_token_stride=4100), "16-byte"), (dict(q_latent_head_stride=513), "16-byte"), (dict(out=None), "null"),
    (dict(out=AT + 40), "16-byte"), (dict(out_head_stride=513), "16-byte"), (dict(out=AT), "neither"),
    (dict(out=AT + 16), "neither"), (dict(lse=AT + 2), "4-byte"), (dict(cache=latent(cache_blocks=0)), "no blocks")])
def test_attention_refused(over, word):
    refused(P.lib().ptstore_latent_attention(C.byref(attention_args(**over)), None), "ptstore_latent_attention", word)


@pytest.mark.parametrize("over,word", BATCH + QUERIES + [
    (dict(heads=0), "heads"), (dict(q_nope=None), "null"), (dict(q_nope=AT + 2), "16-byte"),
    (dict(q_nope_token_stride=1028), "16-byte"), (dict(out=AT), "neither"), (dict(out=AT + 16), "neither"), (dict(out=None), "null"),
    (dict(w_k=None), "w_k"), (dict(w_v=AT + 8), "w_v"), (dict(w_k_row_stride=500), "w_k"), (dict(w_v_head_stride=4), "w_v"),
    (dict(lse=AT + 1), "4-byte"), (dict(key_offsets=None), "null"), (dict(n_keys=-1), "n_keys"), (dict(n_keys=(1 << 31) - 255), "n_keys"),
    (dict(n_keys=1 << 30, heads=8), "tiles"), (dict(R=1 << 21, heads=8, n_tokens=2), "tiles"),
    (dict(cache=latent(cache_blocks=0)), "no blocks"), (dict(), "workspace"),
    (dict(workspace=AT + 8, workspace_bytes=1 << 40), "workspace"), (dict(workspace=AT, workspace_bytes=1000), "workspace")])
def test_expanded_refused(over, word):
    refused(P.lib().ptstore_latent_attention_expanded(C.byref(expanded_args(**over)), None),
            "ptstore_latent_attention_expanded", word)


ROWS = [(dict(lse=None), "null"), (dict(weights=None), "null"), (dict(lse=AT + 2), "4-byte"), (dict(weights=AT + 1), "4-byte")]


@pytest.mark.parametrize("over,word", BATCH + ROWS + [
    (dict(q=None), "q null"), (dict(q=AT + 8), "16-byte"), (dict(q_head_stride=63), "16-byte"), (dict(q_heads=7), "multiple"),
    (dict(q_heads=0), "multiple"), (dict(kv=P.ptstore_kv_t(AT, 2 * AT, 0, 2, 64, 16, 0)), "no blocks"),
    (dict(kv=P.ptstore_kv_t(AT, 2 * AT, 4, 2, 80, 16, 0)), "kind")])
def test_weigh_refused(over, word):
    refused(P.lib().ptstore_kv_weigh(C.byref(weigh_args(**over)), None), "ptstore_kv_weigh", word)


def test_weigh_of_too_many_heads():
    kv = P.ptstore_kv_t(AT, 2 * AT, 1, 1 << 22, 64, 1, 0)
    refused(P.lib().ptstore_kv_weigh(C.byref(weigh_args(kv=kv, q_heads=1 << 22)), None), "too many heads")
    refused(P.lib().ptstore_weigh_workspace(1 << 22, C.byref(C.c_int64())), "kv_heads")


@pytest.mark.parametrize("over,word", BATCH + ROWS + QUERIES + [
    (dict(q_latent=None), "null"), (dict(q_latent=AT + 8), "16-byte"), (dict(heads=0), "heads"),
    (dict(cache=latent(cache_blocks=0)), "no blocks")])
def test_latent_weigh_refused(over, word):
    refused(P.lib().ptstore_latent_weigh(C.byref(latent_weigh_args(**over)), None), "ptstore_latent_weigh", word)


def evict_args(**over):
    a = P.ptstore_evict_t(layers=2, R=3, max_blocks=4, max_keep=20, recent=4, layer_bytes=1 << 20, weights=AT, context=AT,
                          keep=AT + 64, context_out=AT + 128, block_table=AT, to_table=AT, workspace=AT,
                          workspace_bytes=1 << 20)
    for k, v in over.items():
        setattr(a, k, v)
    return a


EVICT = [(dict(layers=-1), "layers"), (dict(R=-1), "R"), (dict(max_blocks=0), "max_blocks"), (dict(max_keep=-1), "max_keep"),
         (dict(recent=-1), "recent"), (dict(R=1 << 20, max_blocks=1 << 10), "out of range"), (dict(max_blocks=(1 << 26) + 1), "2^30"),
         (dict(layer_bytes=24), "layer_bytes"), (dict(layer_bytes=16), "layer_bytes"), (dict(layer_bytes=-(1 << 20)), "layer_bytes"),
         (dict(layers=1 << 22), "too many"), (dict(layers=(1 << 31) - 1, R=1 << 20), "too many"), (dict(weights=None), "null"),
         (dict(context=None), "null"), (dict(keep=None), "null"), (dict(context_out=None), "null"), (dict(block_table=None), "null"),
         (dict(to_table=None), "null"), (dict(weights=AT + 2), "4-byte"), (dict(context_out=AT), "neither"),
         (dict(context_out=AT + 64), "neither"), (dict(workspace=None), "workspace"), (dict(workspace=AT + 4), "workspace"),
         (dict(workspace_bytes=100), "workspace")]


@pytest.mark.parametrize("over,word", EVICT)
def test_evict_refused(over, word):
    lib, a = P.lib(), evict_args(**over)
    kv = P.ptstore_kv_t(AT, 2 * AT, 4, 2, 64, 16, 0)
    refused(lib.ptstore_kv_evict(C.byref(kv), C.byref(a), None), "ptstore_kv_evict", word)
    refused(lib.ptstore_latent_evict(C.byref(latent()), C.byref(a), None), "ptstore_latent_evict", word)


def test_evict_of_no_blocks_and_of_nothing():
    lib = P.lib()
    refused(lib.ptstore_latent_evict(C.byref(latent(cache_blocks=0)), C.byref(evict_args()), None), "no blocks")
    for nothing in (dict(R=0), dict(layers=0)):
        assert lib.ptstore_latent_evict(C.byref(latent()), C.byref(evict_args(**nothing)), None) == 0
    for args, call in ((attention_args, "ptstore_latent_attention"), (expanded_args, "ptstore_latent_attention_expanded"),
                       (weigh_args, "ptstore_kv_weigh"), (latent_weigh_args, "ptstore_latent_weigh")):
        assert getattr(lib, call)(C.byref(args(n_tokens=0, R=0)), None) == 0


def test_workspace_sizes():
    assert P.ptstore_evict_workspace(2, 3, 8, 21) == 2 * 3 * 8 * 21 * 4
    assert P.ptstore_evict_workspace(1, 1, 1, 1) == 16
    assert P.ptstore_evict_workspace(4, 2, 1, 0) == 0 and P.ptstore_evict_workspace(0, 2, 1, 9) == 0
    for bad in ((-1, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, -1), (1 << 20, 1 << 20, 8, 1)):
        with pytest.raises(P.PTStoreError):
            P.ptstore_evict_workspace(*bad)
    for bad in ((0, 1), (8, -1), (8, (1 << 31) - 255)):
        with pytest.raises(P.PTStoreError):
            P.ptstore_latent_expanded_workspace(*bad)
    sizes = [P.ptstore_latent_expanded_workspace(8, n) for n in (1, 128, 10000)]
    assert sizes == sorted(sizes) and sizes[2] >= 10000 * (8 * 1024 + 132) and all(s % 16 == 0 for s in sizes)


def stand_in(nbytes):
    return SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, numel=lambda: nbytes, element_size=lambda: 1,
                           data_ptr=lambda: 0x10000, device="cpu")


def test_cache_of_python():
    row = 2 * (256 + 64)
    c = P.LatentCache(3, 256, 64, 5, 8, data=stand_in(4 * 5 * 8 * row))
    assert c.shape == P.StoreShape(2, 1, 320, 8, 2) and c.shape.chunk_bytes == 8 * row
    assert [c.layer(i).rows - 0x10000 for i in range(3)] == [i * 5 * 8 * row for i in range(3)]
    for bad in (dict(kind="mxfp4"), dict(kind="fp8"), dict(latent_dim=128), dict(rope_dim=32), dict(block_tokens=0),
                dict(block_tokens=65), dict(layers=0), dict(cache_blocks=-1), dict(data=stand_in(3 * 5 * 8 * row))):
        args = dict(layers=3, latent_dim=256, rope_dim=64, cache_blocks=5, block_tokens=8, data=stand_in(4 * 5 * 8 * row))
        args.update(bad)
        with pytest.raises(ValueError):
            P.LatentCache(**args)
    table, one = torch.zeros((1, 4), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    for layers in ((0, 4), (2, 2), (-1, 2)):
        with pytest.raises(ValueError, match="layers"):
            c.evict(torch.zeros(1), one, table, one, 1, layers=layers)


def test_layers_of_other_heads_are_not_evicted_together():
    sizes = [P.ptstore_kv_slab_bytes(P.PTSTORE_KV_BF16, h, 64, 16) for h in (1, 2)]
    c = P.PagedCache(3, (1, 2, 2), 64, 4, data=stand_in(2 * 4 * (sizes[0] + 2 * sizes[1])))
    one = torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="differ"):
        c.evict(torch.zeros(1), one, torch.zeros((1, 4), dtype=torch.int32), one, 1)
    with pytest.raises(ValueError, match="differ"):
        c.weights()


@pytest.mark.parametrize("name,shape", [("q_latent", (2, 8, 256)), ("q_rope", (2, 8, 32)), ("out", (2, 4, 512))])
def test_shapes_of_python(name, shape, monkeypatch):
    """Shapes are compared before anything is launched (device tensors stood in for)."""
    t = {"q_latent": (2, 8, 512), "q_rope": (2, 8, 64), "out": (2, 8, 512)}
    t[name] = shape
    t = {k: SimpleNamespace(is_cuda=True, dtype=torch.bfloat16, dim=lambda s=s: len(s), shape=s,
                            stride=lambda i=None, s=s: 1 if i else (s[1] * s[2], s[2], 1), data_ptr=lambda: AT)
         for k, s in t.items()}
    monkeypatch.setattr(P, "_table", lambda offsets, table: (1, 4))
    with pytest.raises(ValueError, match=name):
        P.ptstore_latent_attention(latent(), t["q_latent"], t["q_rope"], t["out"], None, None, None, None, 0.1, None)
    cpu = torch.zeros((2, 8, 512), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        P.ptstore_latent_append(latent(), cpu[:, 0], cpu[:, 0, :64], torch.zeros(2, dtype=torch.int64))
