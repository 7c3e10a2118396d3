"""Host threads that share a paged cache (CPU: the device and the library are stood in for)."""
from __future__ import annotations

import threading
import time
from types import SimpleNamespace

import pytest
import torch

from paper_2607_22648_amd import ptstore as P


@pytest.fixture
def cache(monkeypatch):
    """A cache whose attention calls note which workspaces are in use, and by how many at most."""
    size = 2 * 4 * P.ptstore_kv_slab_bytes(P.PTSTORE_KV_BF16, 1, 64, 16)
    data = SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, numel=lambda: size, element_size=lambda: 1,
                           data_ptr=lambda: 0x10000, device="cpu")
    cache = P.PagedCache(1, 1, 64, 4, data=data)
    cache.calls, cache.most, cache.busy = 0, 0, {}
    guard = threading.Lock()

    def attention(args, stream):
        at = args._obj.workspace
        with guard:
            cache.calls += 1
            cache.busy[at] = cache.busy.get(at, 0) + 1
            cache.most = max(cache.most, cache.busy[at])
        time.sleep(0.002)  # as the library, which holds no Python lock
        with guard:
            cache.busy[at] -= 1
        return 0

    monkeypatch.setattr(P, "_lib", SimpleNamespace(ptstore_attention=attention))
    monkeypatch.setattr(P, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(P, "_arg", lambda t, dtype, n, name: t.data_ptr())
    monkeypatch.setattr(P, "_token_rows", lambda t, kv, heads, name: (t.data_ptr(), 64, 64))
    monkeypatch.setattr(P, "ptstore_attention_workspace", lambda kv: 256)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return cache


def run(cache, threads, calls, **kw):
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    off, ctx = torch.tensor([0, 1]), torch.zeros(1, dtype=torch.int32)
    table, failed = torch.zeros((1, 4), dtype=torch.int32), []
    start = threading.Barrier(threads)

    def work(i):
        start.wait()
        try:
            for _ in range(calls):
                cache.attend(0, q, off, ctx, table, **{k: v[i] for k, v in kw.items()})
        except Exception as e:  # a thread's own failure would go unseen
            failed.append(e)
    ts = [threading.Thread(target=work, args=(i,)) for i in range(threads)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert not failed and cache.calls == threads * calls


def test_threads_on_one_stream_take_turns(cache):
    """The kernels of two calls never mix in one workspace."""
    run(cache, 4, 6)
    assert cache.most == 1 and len(cache.busy) == 1


def test_a_failed_call_gives_the_turn_back(cache, monkeypatch):
    monkeypatch.setattr(P._lib, "ptstore_attention", lambda args, stream: P.PTSTORE_ERR_INVALID)
    monkeypatch.setattr(P._lib, "ptstore_last_error", lambda: b"no", raising=False)
    q, table = torch.zeros((1, 1, 64), dtype=torch.bfloat16), torch.zeros((1, 4), dtype=torch.int32)
    for _ in range(2):
        with pytest.raises(P.PTStoreError):
            cache.attend(0, q, torch.tensor([0, 1]), torch.zeros(1, dtype=torch.int32), table)
    assert not cache._turn.locked()


def test_workspaces_of_the_caller_need_no_turn(cache):
    """Threads that bring their own run at the same time."""
    spaces = [torch.empty(256, dtype=torch.uint8) for _ in range(3)]
    run(cache, 3, 4, workspace=spaces)
    assert cache.most == 1 and set(cache.busy) == {w.data_ptr() for w in spaces}
