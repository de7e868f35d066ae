"""Arguments that the entry points of the 4-bit key/value cache refuse before anything is launched (no GPU)."""
import ctypes as C

import pytest

import paper_2509_21302_amd as q

OK, NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, ARG = 0, 1, 2, 3, 4, 5, 6
P = 0x10000  # a fake, aligned, non-NULL device address: validation failures return before any use


def test_sizes():
    assert q.qvggt_kv4_page_bytes(16, 8, 128) == 16 * 8 * 132 and q.qvggt_kv4_page_bytes(1024, 1, 64) == 1024 * 68
    for page, heads, d in ((8, 1, 64), (24, 1, 64), (2048, 1, 64), (16, 0, 64), (16, 1, 96), (16, 1, 256), (0, 1, 64), (-16, 1, 64), (16, 65536, 64)):
        assert q.qvggt_kv4_page_bytes(page, heads, d) == 0
    size = q.qvggt_kv4_attention_workspace_bytes
    assert size(1, 1, 1, 131072, 32, 8, 128) > 0 and size(4, 4, 1, 0, 32, 8, 128) == 0
    assert size(1, 1, 1, 131072, 30, 8, 128) == 0 and size(-1, 1, 1, 5000, 8, 8, 128) == 0 and size(1, 65536, 1, 5000, 8, 8, 128) == 0


APPEND = dict(K=P, V=P, dtype=0, T=4, ks=1024, vs=1024, heads=8, d=128, rope=P, rows=50, dim=128, pair=64, at=P, signs=P, slots=P, cache=P, pages=9, page=16)
READ = dict(cache=P, pages=9, page=16, heads=8, d=128, signs=P, slots=P, T=4, dtype=0, K=P, V=P)
ATTEND = dict(Q=P, dtype=0, T=4, qs=4096, heads=32, rope=P, rows=50, dim=128, pair=64, at=P, signs=P, scale=0.1, causal=1, cache=P, pages=9, page=16, kv_heads=8, d=128, table=P,
              width=9, starts=P, lens=P, seqs=4, max_q=1, max_kv=144, out=P, ws=P, size=1 << 30)
NAMES = {"append": (q.load_library().qvggt_kv4_append, APPEND), "read": (q.load_library().qvggt_kv4_read, READ), "attention": (q.load_library().qvggt_kv4_attention, ATTEND)}


def call(name, **other):
    f, good = NAMES[name]
    assert set(other) <= set(good)
    args = dict(good, **other)
    return f(*(C.c_float(v) if k == "scale" else v for k, v in args.items()), None)


@pytest.mark.parametrize("name,other,status", [
    ("append", dict(dtype=2), DTYPE), ("append", dict(T=-1), SHAPE), ("append", dict(d=96), SHAPE), ("append", dict(heads=0), SHAPE), ("append", dict(page=24), SHAPE),
    ("append", dict(pages=-1), SHAPE), ("append", dict(pages=1 << 27, page=16), SHAPE), ("append", dict(ks=-8), SHAPE), ("append", dict(ks=1020), ALIGN),
    ("append", dict(vs=1022, dtype=1), ALIGN), ("append", dict(K=P + 8), ALIGN), ("append", dict(slots=P + 4), ALIGN), ("append", dict(cache=P + 8), ALIGN),
    ("append", dict(K=None), NULL), ("append", dict(V=None), NULL), ("append", dict(slots=None), NULL), ("append", dict(cache=None), NULL), ("append", dict(at=None), NULL),
    ("append", dict(dim=132), SHAPE), ("append", dict(dim=144), SHAPE), ("append", dict(dim=24, pair=4), SHAPE), ("append", dict(dim=0), SHAPE), ("append", dict(pair=0), SHAPE),
    ("append", dict(pair=24, dim=96), SHAPE), ("append", dict(pair=128), SHAPE), ("append", dict(pair=32, dim=96), SHAPE), ("append", dict(rows=0), SHAPE),
    ("append", dict(T=0, K=None, V=None), OK), ("append", dict(pages=0, cache=None), OK),
    ("read", dict(dtype=5), DTYPE), ("read", dict(d=32), SHAPE), ("read", dict(T=-3), SHAPE), ("read", dict(slots=None), NULL), ("read", dict(cache=None), NULL),
    ("read", dict(K=P + 4), ALIGN), ("read", dict(signs=P + 2), ALIGN), ("read", dict(K=None, V=None), OK), ("read", dict(T=0), OK),
    ("attention", dict(dtype=-1), DTYPE), ("attention", dict(heads=30), SHAPE), ("attention", dict(heads=4), SHAPE), ("attention", dict(kv_heads=0), SHAPE), ("attention", dict(d=256), SHAPE),
    ("attention", dict(max_kv=145), SHAPE), ("attention", dict(max_kv=-1), SHAPE), ("attention", dict(max_q=-1), SHAPE), ("attention", dict(seqs=65536), SHAPE),
    ("attention", dict(width=-1, max_kv=0), SHAPE), ("attention", dict(pages=0), SHAPE), ("attention", dict(qs=-4096), SHAPE), ("attention", dict(max_q=1 << 29), SHAPE),
    ("attention", dict(scale=float("nan")), ARG), ("attention", dict(scale=float("inf")), ARG), ("attention", dict(causal=2), ARG), ("attention", dict(qs=4092), ALIGN),
    ("attention", dict(Q=None), NULL), ("attention", dict(table=None), NULL), ("attention", dict(cache=None), NULL), ("attention", dict(starts=None), NULL),
    ("attention", dict(lens=None), NULL), ("attention", dict(out=None), NULL), ("attention", dict(at=None), NULL), ("attention", dict(out=P + 8), ALIGN), ("attention", dict(ws=P + 4), ALIGN),
    ("attention", dict(T=0, Q=None), OK), ("attention", dict(seqs=0), OK), ("attention", dict(max_q=0), OK)])
def test_refusals(name, other, status):
    assert call(name, **other) == status


def test_workspace_is_checked():
    big = dict(width=8192, max_kv=131072, pages=9000)
    need = q.qvggt_kv4_attention_workspace_bytes(4, 4, 1, 131072, 32, 8, 128)
    assert need > 0 and call("attention", size=need - 1, **big) == WORKSPACE and call("attention", ws=None, **big) == NULL


def test_binding_refuses_host_tensors():
    import torch
    x, one = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        q.qvggt_kv4_append(x, x, None, one, torch.zeros(1, 16 * 68, dtype=torch.uint8), 16)
    with pytest.raises(ValueError):
        q.qvggt_kv4_attention(x, None, 1.0, True, torch.zeros(1, 16 * 68, dtype=torch.uint8), 16, 1, torch.zeros(1, 1, dtype=torch.int32), one, one[:1], 2, 2, x, None)
