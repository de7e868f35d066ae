"""Arguments that qvggt_heads_norm_rope, qvggt_attention and qvggt_residual_norm refuse before anything is launched, and the attention's plan (no GPU)."""
import ctypes as C
import itertools
import os
import shutil
import subprocess

import pytest
import torch

import paper_2509_21302_amd as q

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, ARG = 0, 1, 2, 3, 4, 5, 6
P = 0x10000  # a fake, aligned, non-NULL device address: validation failures return before any use

HEADS = dict(Q=P, K=P, dtype=0, T=4, qs=6144, ks=6144, heads=32, kv_heads=8, d=128, norm=2, eps=1e-6, qg=P, qb=None, kg=P, kb=None, rope=P, rows=50, dim=128, pair=64, at=P, axes=3,
             lanes=P, qo=P, ko=P, qos=4096, kos=1024)
ATTEND = dict(Q=P, K=P, V=P, dtype=0, T=40, S=100, qs=6144, ks=6144, vs=6144, heads=32, kv_heads=8, d=128, scale=0.1, causal=1, starts=P, kv_starts=P, lens=None, seqs=3, max_q=20, max_kv=50,
              out=P, ws=P, size=1 << 30)
RESIDUAL = dict(x=P, xt=0, y=2 * P, yt=0, M=10, C=1024, post=1, pg=P, pb=P, scale=P, gate=P, norm=2, g=P, b=P, ms=P, mt=P, ct=0, rows=3, cs=6144, row_of=P, eps=1e-6, xo=3 * P, h=4 * P, ht=0)
NAMES = {"heads": (q.load_library().qvggt_heads_norm_rope, HEADS), "attention": (q.load_library().qvggt_attention, ATTEND), "residual": (q.load_library().qvggt_residual_norm, RESIDUAL)}


def call(name, **other):
    f, good = NAMES[name]
    assert set(other) <= set(good)
    args = dict(good, **other)
    return f(*(C.c_float(v) if k == "eps" or k == "scale" and name == "attention" else v for k, v in args.items()), None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("name,other,status", [
    ("heads", dict(dtype=2), DTYPE), ("heads", dict(T=-1), SHAPE), ("heads", dict(d=96), SHAPE), ("heads", dict(heads=-1), SHAPE), ("heads", dict(kv_heads=65536), SHAPE),
    ("heads", dict(T=1 << 22), SHAPE), ("heads", dict(T=(1 << 25) + 1, heads=1, kv_heads=0), SHAPE), ("heads", dict(qs=-8), SHAPE), ("heads", dict(ks=-8), SHAPE), ("heads", dict(qos=4088), SHAPE), ("heads", dict(kos=8), SHAPE), ("heads", dict(dim=24), SHAPE),
    ("heads", dict(dim=144), SHAPE), ("heads", dict(pair=3), SHAPE), ("heads", dict(pair=0), SHAPE), ("heads", dict(pair=128), SHAPE), ("heads", dict(rows=0), SHAPE), ("heads", dict(axes=0), SHAPE),
    ("heads", dict(axes=5), SHAPE), ("heads", dict(norm=3), ARG), ("heads", dict(norm=-1), ARG), ("heads", dict(eps=-1e-6), ARG), ("heads", dict(eps=NAN), ARG), ("heads", dict(eps=INF), ARG),
    ("heads", dict(Q=None), NULL), ("heads", dict(K=None), NULL), ("heads", dict(qo=None), NULL), ("heads", dict(ko=None), NULL), ("heads", dict(at=None), NULL), ("heads", dict(Q=P + 8), ALIGN),
    ("heads", dict(qs=6140), ALIGN), ("heads", dict(ks=6142, dtype=1), ALIGN), ("heads", dict(qos=4100), ALIGN), ("heads", dict(kg=P + 4), ALIGN), ("heads", dict(at=P + 2), ALIGN),
    ("heads", dict(rope=P + 8), ALIGN), ("heads", dict(T=0, Q=None, K=None), OK), ("heads", dict(heads=0, kv_heads=0, Q=None), OK),
    ("attention", dict(dtype=1), DTYPE), ("attention", dict(T=-1), SHAPE), ("attention", dict(S=-1), SHAPE), ("attention", dict(S=0), SHAPE), ("attention", dict(d=96), SHAPE),
    ("attention", dict(heads=30), SHAPE), ("attention", dict(heads=4), SHAPE), ("attention", dict(kv_heads=0), SHAPE), ("attention", dict(seqs=65536), SHAPE), ("attention", dict(max_q=-1), SHAPE),
    ("attention", dict(max_kv=-1), SHAPE), ("attention", dict(max_kv=(1 << 30) + 1), SHAPE), ("attention", dict(max_q=1 << 29), SHAPE), ("attention", dict(qs=-8), SHAPE),
    ("attention", dict(ks=1 << 24), SHAPE), ("attention", dict(vs=1 << 24), SHAPE), ("attention", dict(ks=-8), SHAPE), ("attention", dict(scale=NAN), ARG), ("attention", dict(scale=INF), ARG),
    ("attention", dict(causal=2), ARG), ("attention", dict(Q=None), NULL), ("attention", dict(K=None), NULL), ("attention", dict(V=None), NULL), ("attention", dict(starts=None), NULL),
    ("attention", dict(kv_starts=None), NULL), ("attention", dict(out=None), NULL), ("attention", dict(K=P + 8), ALIGN), ("attention", dict(qs=6140), ALIGN), ("attention", dict(vs=6148), ALIGN),
    ("attention", dict(starts=P + 2), ALIGN), ("attention", dict(lens=P + 1), ALIGN), ("attention", dict(out=P + 8), ALIGN), ("attention", dict(T=0, Q=None), OK), ("attention", dict(seqs=0), OK),
    ("attention", dict(max_q=0), OK),
    ("residual", dict(xt=2), DTYPE), ("residual", dict(yt=-1), DTYPE), ("residual", dict(ht=5), DTYPE), ("residual", dict(ct=2), DTYPE), ("residual", dict(M=-1), SHAPE), ("residual", dict(C=0), SHAPE),
    ("residual", dict(C=1020), SHAPE), ("residual", dict(C=8200), SHAPE), ("residual", dict(rows=0), SHAPE), ("residual", dict(cs=-8), SHAPE), ("residual", dict(row_of=None), SHAPE),
    ("residual", dict(post=3), ARG), ("residual", dict(norm=-1), ARG), ("residual", dict(eps=-1.0), ARG), ("residual", dict(eps=INF), ARG), ("residual", dict(h=3 * P), ARG),
    ("residual", dict(xo=2 * P), ARG), ("residual", dict(h=P, ht=1), ARG), ("residual", dict(h=2 * P, ht=1), ARG), ("residual", dict(x=None), NULL), ("residual", dict(x=P + 8), ALIGN),
    ("residual", dict(gate=P + 8), ALIGN), ("residual", dict(cs=6148), ALIGN), ("residual", dict(pg=P + 4), ALIGN), ("residual", dict(row_of=P + 2), ALIGN), ("residual", dict(h=4 * P + 8), ALIGN),
    ("residual", dict(M=0, x=None), OK), ("residual", dict(xo=None, h=None), OK)])
def test_refusals(name, other, status):
    assert call(name, **other) == status


@pytest.mark.parametrize("other", [dict(qo=P), dict(ko=2 * P), dict(qo=4 * P, ko=4 * P), dict(qo=2 * P), dict(ko=P), dict(qo=P, qos=6144, ko=2 * P)])
def test_heads_outputs_in_a_place_that_others_have(other):
    """Rows at another distance than the input's in its place; queries and keys in one place."""
    assert call("heads", **dict(dict(Q=P, K=2 * P, qo=3 * P, ko=4 * P), **other)) == ARG


@pytest.mark.parametrize("scale", [1.1e38, -3e38, -INF])
def test_scales_that_leave_fp32(scale):
    assert call("attention", scale=scale) == ARG


@pytest.mark.parametrize("other", [dict(out=P), dict(out=2 * P), dict(out=3 * P), dict(out=3 * P, heads=8, ws=None, size=0), dict(out=P, T=1, S=0, max_kv=0)])
def test_attention_output_in_the_place_of_an_input(other):
    assert call("attention", **dict(dict(Q=P, K=2 * P, V=3 * P, out=4 * P), **other)) == ARG


def test_workspace():
    size = q.qvggt_attention_workspace_bytes
    need = size(1, 1, 1, 131072, 32, 8, 128)
    assert need > 0 and size(4, 4, 1, 0, 32, 8, 128) == 0 and size(1, 1, 1, 131072, 30, 8, 128) == 0 and size(-1, 1, 1, 5000, 8, 8, 128) == 0 and size(1, 65536, 1, 5000, 8, 8, 128) == 0
    one = dict(T=1, S=131072, seqs=1, max_q=1, max_kv=131072)
    assert call("attention", size=need - 1, **one) == WORKSPACE and call("attention", ws=None, **one) == NULL and call("attention", ws=P + 8, **one) == ALIGN


PLAN = r"""
#include "attention_plan.h"
#include <cstdio>
#include <cstdlib>
int main(int, char **v)
{
    for (int causal = 0; causal < 2; ++causal) {
        const auto p = qvggt::attention_plan(atoi(v[1]), atoi(v[2]), atoi(v[3]), atoi(v[4]), atoi(v[5]), atoi(v[6]), causal);
        std::printf("%d %d %d %d %d %zu %zu\n", p.few, p.waves, p.tiles, p.chunk, p.splits, p.bytes, qvggt::attention_workspace(atoi(v[1]), atoi(v[2]), atoi(v[3]), atoi(v[4]), atoi(v[5]), atoi(v[6])));
    }
}
"""


def test_plan_covers_all_rows_and_keys(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "plan.cpp").write_text(PLAN)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2509_21302_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", exe], check=True)
    for seqs, max_q, max_kv, (heads, kv), d in itertools.product((1, 7, 64, 65535), (1, 9, 129, 12289), (0, 1, 127, 1000, 131071, 1 << 30), ((1, 1), (32, 8), (64, 1), (16, 16)), (64, 128)):
        if seqs * kv * -(-max_q * (heads // kv) // 32) > 1 << 23:
            continue
        for line in subprocess.run([exe, *map(str, (seqs, max_q, max_kv, heads, kv, d))], check=True, capture_output=True, text=True).stdout.splitlines():
            few, waves, tiles, chunk, splits, size, whole = map(int, line.split())
            rows = max_q * (heads // kv)
            assert tiles * (32 if few else 128) >= rows and (few == 0 or rows <= 32) and waves in ((4, 8) if few else (4,)) and chunk % 64 == 0 and chunk > 0 and 1 <= splits <= 256
            assert chunk * splits >= max_kv and (splits == 1 or chunk * (splits - 1) < max_kv)
            assert size == (0 if splits == 1 else seqs * kv * rows * splits * (d + 2) * 4) and whole >= size and seqs * kv * tiles * splits < 1 << 31


def test_binding_refuses():
    x, one = torch.zeros(2, 1, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        q.qvggt_heads_norm_rope(x, x, x, x)
    with pytest.raises(ValueError):
        q.qvggt_heads_norm_rope(x, x, x, x, norm="batch")
    with pytest.raises(ValueError):
        q.qvggt_attention(x, x, x, 1.0, True, one, one, None, 2, 2, x, None)
    with pytest.raises(ValueError):
        q.qvggt_residual_norm(x[:, 0], x[:, 0], x[:, 0], x[:, 0])
    with pytest.raises(ValueError):
        q.qvggt_residual_norm(x[:, 0], x[:1, 0], x[:, 0], x[:, 0])
