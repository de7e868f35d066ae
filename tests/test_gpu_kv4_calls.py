"""Ways to the 4-bit key/value cache: Kv4Cache, the native calls beside the Python ones, the example that streams frames through it."""
import importlib.util
import os

import pytest
import torch

import paper_2509_21302_amd as q
from paper_2509_21302_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _cache(pages=8, page=32, heads=2, d=64, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    angle = torch.rand(100, d // 2, device=DEV, generator=g) * 6
    return q.Kv4Cache(pages, page, heads, d, (torch.randint(0, 2, (d,), device=DEV, generator=g) * 2 - 1).to(torch.int8), torch.cat([angle.cos(), angle.sin()], 1), d // 2, DEV), g


def test_tokens_come_back_and_attention_follows_them():
    cache, g = _cache()
    T, n = 100, 7
    k, v = (torch.randn(T, 2, 64, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    table = torch.randperm(8, device=DEV, generator=g).int()[None].contiguous()
    at = torch.arange(T, device=DEV)
    slots = table[0, at // 32] * 32 + (at % 32).int()
    cache.append(k, v, slots, at.int() % 100)
    k4, v4 = cache.read(slots, torch.float32)
    assert 0.05 < float((v4 - v.float()).norm() / v.float().norm()) < 0.2            # 4 bits of a normal row
    queries = torch.randn(n, 4, 64, device=DEV, generator=g)
    y = cache.attend(queries, table, torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([T], dtype=torch.int32, device=DEV), n, T,
                     torch.arange(T - n, T, device=DEV).int())
    cos, sin = cache.rope[T - n:, None, :32], cache.rope[T - n:, None, 32:]
    turned = torch.cat([queries[..., :32] * cos - queries[..., 32:] * sin, queries[..., 32:] * cos + queries[..., :32] * sin], 2)
    x = torch.einsum("nhd,thd->hnt", turned, k4.repeat_interleave(2, 1)) / 8
    x = x.masked_fill(torch.arange(T, device=DEV) > T - n + torch.arange(n, device=DEV)[:, None], -torch.inf)
    want = torch.einsum("hnt,thd->nhd", torch.softmax(x, 2), v4.repeat_interleave(2, 1))
    assert float((y.float() - want).norm() / want.norm()) <= 4e-3
    with pytest.raises(q.QvggtError):
        q.Kv4Cache(4, 24, 2, 64, device=DEV)


def test_native_calls_are_the_python_ones(monkeypatch):
    if B._call is None:
        pytest.skip("the native calls are not built")
    taken, got = [], []
    for native in (True, False):
        if native:
            for name in ("kv4_append", "kv4_read", "kv4_attention"):
                f = getattr(B._call, name)
                monkeypatch.setattr(B, "_native", lambda f, name, *a, real=B._native: taken.append((name, real(f, name, *a))) or taken[-1][1])
        else:
            monkeypatch.setattr(B, "_call", None)
        cache, g = _cache()
        cache.pages.zero_()
        rows = torch.randn(5, 8, 64, device=DEV, generator=g).to(torch.bfloat16)
        slots = torch.tensor([3, 40, -1, 4, 5], dtype=torch.int32, device=DEV)
        at = torch.arange(5, device=DEV, dtype=torch.int32)
        cache.append(rows[:, 4:6], rows[:, 6:], slots, at)
        y = cache.attend(rows[:, :4], torch.arange(8, device=DEV, dtype=torch.int32)[None], torch.tensor([0, 5], dtype=torch.int32, device=DEV),
                         torch.tensor([6], dtype=torch.int32, device=DEV), 5, 6, at)
        got.append([cache.pages, y, *cache.read(slots)])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and len(taken) >= 3 and all(ok for _, ok in taken)


def test_what_the_native_calls_do_not_know_is_refused_or_taken_by_python():
    cache, g = _cache()
    k = torch.randn(4, 2, 64, device=DEV, generator=g)
    slots = torch.arange(4, dtype=torch.int32, device=DEV)
    at = slots.clone()
    for bad in (dict(k=k.half()), dict(k=k[:, :, ::2]), dict(k=k.cpu()), dict(slots=slots.long()), dict(slots=slots[:3]), dict(at=at.long()), dict(at=None)):
        a = dict(dict(k=k, slots=slots, at=at), **bad)
        with pytest.raises(ValueError):
            cache.append(a["k"], k, a["slots"], a["at"])
    cache.append(k[:0], k[:0], slots[:0], at[:0])                                     # no tokens: nothing to do
    with pytest.raises(q.QvggtError) as e:
        q.qvggt_kv4_append(k, k, None, slots, cache.pages, 32, rope=cache.rope, positions=at, rope_pair=3)
    assert e.value.status == 2


def test_frames_stream_through_the_example(capsys):
    """A block's attention is that of its own queries over what its cache stands for: rounding the result to bf16, weights and queries to fp16, as in test_gpu_kv4.py."""
    spec = importlib.util.spec_from_file_location("streaming_attention", os.path.join(ROOT, "examples", "streaming_attention.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    block, g = module.Block(1024, 16, 3, 9), torch.Generator(DEV).manual_seed(2)
    for frame in range(3):
        x = torch.randn(81, 1024, device=DEV, generator=g).to(torch.bfloat16)
        queries = block.turned(block.rows(x)[:, :16])
        got = block.attention(x)
        k, v = block.cache.read(block.slots(0, 81 * (frame + 1)), torch.float32)
        want = module.plain_attention(queries, k, v)
        assert float((got.float() - want).norm() / want.norm()) <= 4e-3
    y = block.out(got.view(81, 1024))
    assert y.shape == (81, 1024) and bool(torch.isfinite(y.float()).all())
    assert len(module.main(["--frames", "2", "--side", "9"])) == 2 and capsys.readouterr().out.count("from float32") == 2
