"""The workspace that a Kv4Cache keeps, with the entry points replaced (no GPU): what a captured call was given must not go back to the allocator while the cache lives."""
import gc
import weakref

import pytest
import torch

from paper_2509_21302_amd import Kv4Cache
from paper_2509_21302_amd import binding as B


@pytest.fixture
def cache(monkeypatch):
    used = []
    monkeypatch.setattr(B, "qvggt_kv4_attention", lambda *a, **kw: used.append(None if a[13] is None else weakref.ref(a[13])))
    monkeypatch.setattr(B, "capturing", lambda t: cache.recording, raising=False)
    cache = Kv4Cache(4, 16, 2, 64, device="cpu")
    cache.recording, cache.used = False, used
    return cache


def attend(cache, max_kv, recording=False):
    one = torch.zeros(2, dtype=torch.int32)
    cache.recording = recording
    cache.attend(torch.zeros(1, 2, 64), torch.zeros(1, -(-max_kv // 16), dtype=torch.int32), one, one[:1], 1, max_kv)
    gc.collect()
    return cache.used[-1]


def test_a_captured_calls_workspace_outlives_a_larger_call(cache):
    first = attend(cache, 2000, recording=True)
    assert attend(cache, 20000)() is not first()
    assert first() is not None                               # replays write into it
    second = attend(cache, 20000, recording=True)
    attend(cache, 20000, recording=True)
    attend(cache, 200000)
    assert first() is not None and second() is not None and first() is not second()
    assert len(cache._captured) == 2


def test_a_workspace_that_nobody_recorded_is_replaced(cache):
    first = attend(cache, 2000)
    assert attend(cache, 20000)() is not None and first() is None
    assert attend(cache, 2000)() is cache._ws                # the larger one serves smaller calls
    assert attend(cache, 100) is not None and not cache._captured


@pytest.mark.gpu
def test_a_replay_after_a_larger_call_writes_into_nobodys_tensor():
    dev = "cuda:0"
    g = torch.Generator(dev).manual_seed(0)
    cache = Kv4Cache(300, 16, 2, 64, device=dev)
    x = torch.randn(4800, 4, 64, device=dev, generator=g).to(torch.bfloat16)
    cache.append(x[:, :2], x[:, 2:], torch.arange(4800, device=dev, dtype=torch.int32))
    table = torch.arange(300, device=dev, dtype=torch.int32)[None]
    starts, lens = torch.tensor([0, 1], device=dev, dtype=torch.int32), torch.tensor([2000], device=dev, dtype=torch.int32)
    query, out = x[:1].clone(), torch.empty(1, 4, 64, dtype=torch.bfloat16, device=dev)
    want = cache.attend(query, table, starts, lens, 1, 2000)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.attend(query, table, starts, lens, 1, 2000, out=out)
    small = cache._ws.numel()
    cache.attend(x[:200], table, torch.tensor([0, 200], device=dev, dtype=torch.int32), torch.tensor([4800], device=dev, dtype=torch.int32), 200, 4800)
    assert cache._ws.numel() > small
    others = [torch.full((small,), 77, dtype=torch.uint8, device=dev) for _ in range(20)]         # whatever the allocator has of that size
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 77).all()) for t in others)
        cache.attend(x[:200], table, torch.tensor([0, 200], device=dev, dtype=torch.int32), torch.tensor([4800], device=dev, dtype=torch.int32), 200, 4800)
