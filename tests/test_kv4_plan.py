"""How a call of qvggt_kv4_attention is cut up (csrc/kv4_plan.h, compiled for the host), and what the compiler says of its kernels (no GPU)."""
import os
import random
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import paper_2509_21302_amd as q
from paper_2509_21302_amd import build as B

DRIVER = r"""
#include "kv4_plan.h"
#include <cstdio>
int main()
{
    int s, mq, mk, h, kh, d;
    while (std::scanf("%d %d %d %d %d %d", &s, &mq, &mk, &h, &kh, &d) == 6) {
        if ((long long)mq * (h / kh) <= qvggt::kKv4SharedRows) {
            const qvggt::Kv4Shares p = qvggt::kv4_shares(s, mq, mk, h, kh, d);
            std::printf("1 %d %d %d %d %d %zu %zu\n", p.nt, p.tiles, p.blocks, p.unit_shift, p.least, p.map_bytes, p.bytes);
        } else {
            const qvggt::Kv4Tiles p = qvggt::kv4_tiles(s, mq, mk, h, kh, d);
            std::printf("0 %d %d %d %d 0 0 %zu\n", p.nt, p.tiles, p.chunk, p.splits, p.bytes);
        }
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    folder = tmp_path_factory.mktemp("kv4_plan")
    (folder / "driver.cpp").write_text(DRIVER)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", B.CSRC, "-o", folder / "driver", folder / "driver.cpp"],
                   check=True)

    def ask(problems):
        text = "\n".join(" ".join(map(str, p)) for p in problems)
        lines = subprocess.run([folder / "driver"], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
        assert len(lines) == len(problems)
        return [list(map(int, line.split())) for line in lines]
    return ask


def _problems():
    rng, some = random.Random(0), []
    spread = lambda hi: int(2 ** rng.uniform(0, hi))  # noqa: E731
    while len(some) < 4000:
        kh = rng.choice((1, 2, 3, 8, 16, 20, 128))
        p = (spread(16) - 1 or 1, spread(14), rng.choice((0, 1, 1024, 1025, spread(21), spread(30) - 1)), kh * rng.choice((1, 2, 4, 7, 16, 64)), kh, rng.choice((64, 128)))
        if p[0] * kh * -(-p[1] * (p[3] // kh) // 64) <= 1 << 23:
            some.append(p)
    return some + [(65535, 1, 1 << 30, 128, 128, 64), (1, 1 << 20, 1 << 30, 8, 8, 128), (65535, 1, 0, 1, 1, 128)]


def test_plans_cover_every_key_and_row(plans):
    problems = _problems()
    for (seqs, max_q, max_kv, heads, kv_heads, d), (shared, nt, tiles, a, b, least, map_bytes, size) in zip(problems, plans(problems)):
        rows = max_q * (heads // kv_heads)
        assert size == q.qvggt_kv4_attention_workspace_bytes(1, seqs, max_q, max_kv, heads, kv_heads, d)
        if shared:
            blocks, shift = a, b
            assert rows <= 64 and nt in (1, 2) and 16 * nt * tiles >= rows and 16 * nt * (tiles - 1) < rows
            units = seqs * kv_heads * tiles * (-(-max_kv // (1 << shift)) + 2)           # with what a head costs besides its keys
            assert shift >= 7 and units < 1 << 31 and 0 <= blocks <= 768
            if blocks:
                assert max_kv > 1024 and map_bytes >= 4 * (1 + seqs) and size == map_bytes + blocks * 2 * 16 * nt * (d + 2) * 4
                assert blocks * max(-(-units // blocks), least) >= units                    # the shares hold everything
            else:
                assert size == 0 and seqs * kv_heads * tiles < 1 << 24
        else:
            chunk, splits = a, b
            assert nt in (1, 2, 4) and (nt < 4 or d == 64) and 64 * nt * tiles >= rows and 64 * nt * (tiles - 1) < rows
            assert splits >= 1 and chunk * splits >= max_kv and (splits == 1 or chunk * (splits - 1) < max_kv and chunk % 128 == 0)
            assert size == (0 if splits == 1 else seqs * heads * max_q * splits * (d + 2) * 4)
            assert seqs * kv_heads * tiles * splits < 1 << 24                               # a launch has less than 2^32 threads


def test_kernels_keep_their_registers(tmp_path):
    """No scratch memory in the loops: none at all where rows are shared, a few bytes around the loops of the largest tile."""
    if shutil.which(B.HIPCC) is None:
        pytest.skip("hipcc is not installed")
    files = ("kv4_shared_rows.hip", "kv4_own_rows.hip", "kv4_cache.hip")

    def compile(f):
        out = tmp_path / (f + ".s")
        subprocess.run([B.HIPCC, *B.FLAGS, "--cuda-device-only", "-S", os.path.join(B.CSRC, f), "-o", out], check=True, capture_output=True)
        return out.read_text()
    with ThreadPoolExecutor(3) as ex:
        texts = list(ex.map(compile, files))
    for f, text in zip(files, texts):
        sizes = dict(zip(re.findall(r"\.amdhsa_kernel (\w+)", text), map(int, re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text))))
        assert len(sizes) >= 6
        for name, size in sizes.items():
            assert size <= (16 if "own_rows_kernelILi64ELi4E" in name else 8 if "shared_rows" in name else 0), (name, size)
        assert not re.search(r"v_pk_(add|mul|fma)_f32", text)
