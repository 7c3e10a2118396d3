"""What the binding of latent caches, attention weights and eviction refuses before a call is made (CPU: device
tensors are stood in for)."""
from __future__ import annotations

from types import SimpleNamespace

import pytest
import torch

from paper_2607_22648_amd import ptstore as P
from test_latent_abi import latent, stand_in

AT = 0x1000


def device(*shape, dtype=torch.float32):
    t = torch.zeros((), dtype=dtype).expand(shape)
    return SimpleNamespace(is_cuda=True, dtype=dtype, shape=torch.Size(shape), numel=t.numel, dim=t.dim,
                           is_contiguous=lambda: True, data_ptr=lambda: AT,
                           stride=lambda i=None: torch.empty(shape, device="meta").stride(*(() if i is None else (i,))))


@pytest.fixture
def calls(monkeypatch):
    """The weighings and evictions that reach the library, with their structs."""
    made, library = [], P._lib

    class Library:
        def __getattr__(self, name):
            if not name.endswith(("_weigh", "_evict")):
                return getattr(library, name)

            def call(*args):
                made.append((name, [getattr(a, "_obj", a) for a in args]))
                return 0
            return call
    monkeypatch.setattr(P, "_lib", Library())
    monkeypatch.setattr(P, "_stream", lambda stream: 0)
    return made


def batch(tokens=3):
    i32 = torch.int32
    return device(2, dtype=torch.int64), device(1, dtype=i32), device(1, 8, dtype=i32)


WORKSPACE = device(1 << 22, dtype=torch.uint8)


def paged(layers=4, heads=2):
    size = 2 * layers * 5 * P.ptstore_kv_slab_bytes(P.PTSTORE_KV_BF16, heads, 64, 16)
    return P.PagedCache(layers, heads, 64, 5, data=stand_in(size))


@pytest.mark.parametrize("shape,ok", [((5, 2, 16), True), ((1, 5, 2, 16), True), ((4, 5, 2, 16), False), ((5, 1, 16), False),
                                      ((2, 5, 2, 16), False), ((6, 2, 16), False), ((0,), False)])
def test_weigh_takes_the_weights_of_one_layer(calls, shape, ok):
    """All layers' weights in the place of one's would add to layer 0's."""
    cache = paged()
    w = device(*shape)

    def weigh():
        return cache.weigh(3, w, device(3, 4, 64, dtype=torch.bfloat16), device(3, 4), *batch(), workspace=WORKSPACE)
    if ok:
        assert weigh() is w and [c[0] for c in calls] == ["ptstore_kv_weigh"]
    else:
        with pytest.raises(ValueError, match="weights"):
            weigh()
        assert not calls


@pytest.mark.parametrize("shape,ok", [((4, 1, 16), True), ((1, 4, 1, 16), True), ((4, 16), True), ((3, 4, 1, 16), False),
                                      ((4, 1, 15), False)])
def test_latent_weigh_takes_the_weights_of_one_layer(calls, shape, ok):
    args = (device(3, 8, 512, dtype=torch.bfloat16), device(3, 8, 64, dtype=torch.bfloat16), device(3, 8), *batch(), 0.1, WORKSPACE)
    if ok:
        P.ptstore_latent_weigh(latent(), device(*shape), *args)
        assert [c[0] for c in calls] == ["ptstore_latent_weigh"]
    else:
        with pytest.raises(ValueError, match="weights"):
            P.ptstore_latent_weigh(latent(), device(*shape), *args)
        assert not calls


@pytest.mark.parametrize("layers,shape,ok", [((1, 3), (2, 5, 2, 16), True), ((1, 3), (4, 5, 2, 16), False),
                                             ((0, 4), (4, 5, 2, 16), True), ((0, 4), (2, 5, 2, 16), False),
                                             (None, (4, 5, 2, 16), True), ((3, 4), (5, 2, 16), True)])
def test_evict_takes_the_weights_of_its_layers(calls, monkeypatch, layers, shape, ok):
    """Weights of all layers with a part of the layers would choose by, and move, the first layers' weights."""
    cache = paged()
    monkeypatch.setattr(torch, "empty_like", lambda t, **kw: device(*t.shape, dtype=t.dtype))
    one, table = device(1, dtype=torch.int32), device(1, 8, dtype=torch.int32)

    def evict():
        return cache.evict(device(*shape), one, table, one, 20, layers=layers, workspace=WORKSPACE)
    if ok:
        evict()
        (name, (kv, a, _)), = calls
        first, past = layers or (0, 4)
        assert name == "ptstore_kv_evict" and kv.k == cache.layer(first).k and a.layers == past - first
    else:
        with pytest.raises(ValueError, match="weights"):
            evict()
        assert not calls


@pytest.mark.parametrize("most,recent", [(1 << 32, 0), ((1 << 32) + 20, 0), (1 << 31, 0), (20, 1 << 32), (20, (1 << 32) + 3),
                                         (20, -(1 << 32))])
def test_evict_refuses_what_32_bits_do_not_hold(calls, monkeypatch, most, recent):
    """A max_keep of 2^32 must not keep nothing, nor a `recent` of 2^32 no recent tokens."""
    cache = paged()
    monkeypatch.setattr(torch, "empty_like", lambda t, **kw: device(*t.shape, dtype=t.dtype))
    one, table = device(1, dtype=torch.int32), device(1, 8, dtype=torch.int32)
    with pytest.raises(ValueError, match="max_keep" if recent == 0 else "recent"):
        cache.evict(device(4, 5, 2, 16), one, table, one, most, recent=recent, workspace=WORKSPACE)
    assert not calls


@pytest.mark.parametrize("call,args", [
    ("ptstore_evict_workspace", ((1 << 32) + 1, 1, 1, 1)), ("ptstore_evict_workspace", (1, (1 << 32) + 1, 1, 1)),
    ("ptstore_evict_workspace", (1, 1, (1 << 32) + 1, 1)), ("ptstore_evict_workspace", (1, 1, 1, (1 << 32) + 1)),
    ("ptstore_latent_expanded_workspace", ((1 << 32) + 8, 100)), ("ptstore_latent_expanded_workspace", (8, (1 << 64) + 100)),
    ("ptstore_weigh_workspace", ((1 << 32) + 1,))])
def test_workspaces_of_sizes_past_the_calls_numbers(call, args):
    with pytest.raises(ValueError, match="bits"):
        getattr(P, call)(*args)


@pytest.mark.parametrize("heads,keys", [((1 << 31) - 1, (1 << 31) - 256), (1 << 24, 1 << 30), (8, (1 << 31) - 256), (1 << 24, 0),
                                        ((1 << 24) - (1 << 13) + 1, 1), (128, 1 << 24)])
def test_expanded_workspaces_of_calls_that_are_refused(heads, keys):
    """(n_keys / 128 + 1) * heads past 2^24 - 2^13, which the call refuses: no size, and no product that overflows."""
    with pytest.raises(P.PTStoreError, match="out of range"):
        P.ptstore_latent_expanded_workspace(heads, keys)


@pytest.mark.parametrize("heads,keys", [((1 << 24) - (1 << 13), 127), (8, 268304383), (1, (1 << 31) - 1048577), (128, 16769023)])
def test_expanded_workspaces_of_the_largest_calls(heads, keys):
    assert P.ptstore_latent_expanded_workspace(heads, keys) == heads * keys * 1024 + keys * 128 + -(-keys * 4 // 16) * 16
    with pytest.raises(P.PTStoreError):
        P.ptstore_latent_expanded_workspace(heads, keys + 1)


def test_weights_are_required(calls, monkeypatch):
    cache = paged()
    monkeypatch.setattr(torch, "empty_like", lambda t, **kw: device(*t.shape, dtype=t.dtype))
    one, table = device(1, dtype=torch.int32), device(1, 8, dtype=torch.int32)
    with pytest.raises(ValueError, match="weights is required"):
        cache.evict(None, one, table, one, 20, workspace=WORKSPACE)
    with pytest.raises(ValueError, match="weights is required"):
        cache.weigh(0, None, device(3, 4, 64, dtype=torch.bfloat16), device(3, 4), *batch(), workspace=WORKSPACE)
    assert not calls
