"""The workspace that a DsfqLinear keeps: what a captured call was given must not go back to the allocator while the layer lives."""
import copy
import gc
import pickle
import weakref

import pytest
import torch

from paper_2509_21302_amd import DsfqLinear
from paper_2509_21302_amd import binding as B


@pytest.fixture
def layer(monkeypatch):
    """A layer without device tensors whose calls do not run."""
    recording, used = [False], []

    def native_linear(kind, X, *a):
        used.append(weakref.ref(a[7]))
        return torch.empty(X.shape[0], 16, dtype=torch.bfloat16)
    monkeypatch.setattr(B, "native_linear", native_linear)
    monkeypatch.setattr(B, "capturing", lambda t: recording[0], raising=False)
    layer = DsfqLinear.__new__(DsfqLinear)
    layer.__dict__.update(N=16, K=1024, bits=4, act_bits=4, bias=None, signs=None, packed=True, pre_gelu=False, gelu_table=None, w_scale=None, inv_smooth=None, Wq=torch.empty(0),
                          Wf=torch.empty(0), _ws=(-1, None))

    def call(M, captured=False):
        recording[0] = captured
        layer(torch.zeros(M, 1024, dtype=torch.bfloat16))
        gc.collect()
        return used[-1]
    return layer, call


def test_a_captured_calls_workspace_outlives_more_rows(layer):
    layer, call = layer
    first = call(100, captured=True)
    assert call(1000)() is not first() and first() is not None
    second = call(1000, captured=True)
    call(900, captured=True)
    call(5000)
    assert first() is not None and second() is not None and len(layer._captured) == 2
    for other in (copy.copy(layer), pickle.loads(pickle.dumps(layer))):                  # a copy has no captured calls
        assert not other._captured


def test_a_workspace_that_nobody_recorded_is_replaced(layer):
    layer, call = layer
    first = call(100)
    assert call(1000)() is not None and first() is None and not layer._captured


@pytest.mark.gpu
def test_a_replay_after_more_rows_writes_into_nobodys_tensor():
    dev = "cuda:0"
    g = torch.Generator(dev).manual_seed(0)
    X = torch.randn(20000, 1024, device=dev, generator=g).to(torch.bfloat16)
    layer = DsfqLinear(torch.randn(512, 1024, device=dev, generator=g).to(torch.bfloat16), calibration=X[:256])
    few, out = X[:4500].clone(), torch.empty(4500, 512, dtype=torch.bfloat16, device=dev)
    want = layer(few)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(few, out)
    small = layer._ws[1].numel()
    layer(X)
    assert layer._ws[1].numel() > small
    others = [torch.full((small,), 77, dtype=torch.uint8, device=dev) for _ in range(8)]
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 77).all()) for t in others)
        layer(X)
