"""qvggt_attention through every way in which a call is cut up (csrc/attention_plan.h), batches of hundreds of sequences among them, and at the end of the strides that it takes."""
import os
import random
import shutil
import subprocess

import pytest
import torch

from oracle import block as O
from tests import gpu_util as G
from tests.test_block_refusals import PLAN, ROOT
from tests.test_gpu_attention import attend, inputs, near, starts_of, whole

DEV = G.DEV

# seqs, max_q, max_kv, heads, kv_heads, d -> few rows, two tiles of them, waves, in parts.  Whole sequences of few rows, more than 256 of them times their key heads, have four waves
CASES = {
    "few_64": (300, 1, 40, 1, 1, 64), "few_64_group": (80, 1, 700, 16, 4, 64), "few_64_some": (90, 2, 90, 24, 4, 64), "few_64_two": (90, 3, 90, 24, 4, 64), "few_64_two_long": (300, 2, 1000, 16, 1, 64),
    "few_64_two_alone": (270, 31, 260, 1, 1, 64), "few_128": (513, 1, 33, 1, 1, 128), "few_128_group": (40, 4, 500, 32, 8, 128), "few_128_two": (70, 5, 300, 20, 4, 128),
    "few_128_two_alone": (260, 17, 500, 1, 1, 128), "few_128_two_full": (65, 32, 64, 4, 4, 128), "eight_64": (8, 1, 300, 8, 8, 64), "eight_64_two": (4, 9, 200, 16, 8, 64), "eight_128": (2, 4, 100, 32, 8, 128),
    "eight_128_two": (2, 30, 100, 8, 8, 128), "parts_64": (3, 1, 9000, 8, 8, 64), "parts_64_two": (3, 20, 9000, 4, 4, 64), "parts_128": (3, 2, 9000, 32, 8, 128), "parts_128_two": (3, 8, 9000, 32, 8, 128),
    "many_64": (200, 70, 70, 8, 4, 64), "many_128": (120, 65, 300, 16, 8, 128), "many_parts_64": (3, 50, 7000, 8, 4, 64), "many_parts_128": (3, 50, 7000, 8, 4, 128),
}
PLANS = {"few_64": (1, 0, 4, 0), "few_128": (1, 0, 4, 0), "few_64_two": (1, 1, 4, 0), "few_128_two": (1, 1, 4, 0), "eight": (1, None, 8, 0), "parts_64": (1, 0, 4, 1), "parts_128": (1, 0, 4, 1),
         "parts_64_two": (1, 1, 4, 1), "parts_128_two": (1, 1, 4, 1), "many_64": (0, 1, 4, 0), "many_128": (0, 1, 4, 0), "many_parts": (0, 1, 4, 1)}


def test_the_cases_take_the_plans_that_they_are_for(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "plan.cpp").write_text(PLAN)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2509_21302_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", exe], check=True)
    for name, case in CASES.items():
        want = PLANS[max((p for p in PLANS if name.startswith(p)), key=len)]
        for line in subprocess.run([exe, *map(str, case)], check=True, capture_output=True, text=True).stdout.splitlines():
            few, waves, _, _, splits, _, _ = map(int, line.split())
            got = few, int(case[1] * (case[3] // case[4]) > 16), waves, int(splits > 1)
            assert all(w is None or w == g for w, g in zip(want, got)), (name, got)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["buffer", "packed", "bidirectional"])
@pytest.mark.parametrize("name", CASES)
def test_every_plan(name, form):
    """Sequences of any lengths, some without queries or keys."""
    seqs, max_q, max_kv, heads, kv_heads, d = CASES[name]
    rng = random.Random(name + form)
    lengths = [(max_q, max_kv) if i == seqs // 2 else (rng.randint(0, max_q), rng.choice((0, 1, rng.randint(1, max_kv), max_kv))) for i in range(seqs)]
    q_lens, kv_lens = zip(*lengths)
    T, capacity = sum(q_lens), max_kv + 1
    first = starts_of(kv_lens) if form == "packed" else [i * capacity for i in range(seqs)]
    S = first[-1] if form == "packed" else seqs * capacity
    Q, K, V = inputs(T, S, heads, kv_heads, d, seqs + max_kv)
    if form != "packed":
        for i, n in enumerate(kv_lens):
            K[first[i] + n:first[i] + capacity] = float("nan")
            V[first[i] + n:first[i] + capacity] = float("nan")
    causal = form != "bidirectional"
    got = attend(Q, K, V, 0.1, causal, whole(starts_of(q_lens)), whole(first), None if form == "packed" else whole(kv_lens), max_q, max_kv)
    near(got, *O.attention(Q, K, V, 0.1, causal, lengths, first))


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(12))
def test_random_batches_of_many_sequences(seed):
    rng = random.Random(1000 + seed)
    d, group, kv_heads, causal = rng.choice((64, 128)), rng.choice((1, 2, 4, 7)), rng.choice((1, 2, 4)), rng.random() < 0.6
    seqs, top_q, top_kv = rng.randint(60, 300), rng.choice((1, 3, 9, 40)), rng.choice((1, 50, 300))
    lengths = [(rng.randint(0, top_q), rng.randint(0, top_kv)) for _ in range(seqs - 1)] + [(top_q, top_kv)]
    q_lens, kv_lens = zip(*lengths)
    first = starts_of(kv_lens)
    Q, K, V = inputs(sum(q_lens), first[-1], group * kv_heads, kv_heads, d, seed)
    got = attend(Q, K, V, 0.125, causal, whole(starts_of(q_lens)), whole(first), None, top_q, top_kv)
    near(got, *O.attention(Q, K, V, 0.125, causal, lengths, first))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m", [(1, 200), (33, 129), (150, 257), (60, 700)])
def test_the_widest_strides(d, n, m):
    """Keys and values 2^24 - 8 elements apart: the last of a tile lies nearly 2^31 bytes behind its first."""
    stride = (1 << 24) - 8
    base = torch.empty((m + 1) * stride + 2 * d, dtype=torch.bfloat16, device=DEV)
    K, V = (base[i * d:].as_strided((m, 1, d), (stride, d, 1)) for i in (0, 1))
    g = torch.Generator(DEV).manual_seed(n)
    for t in (K, V):
        t.copy_(torch.randn(m, 1, d, device=DEV, generator=g).to(torch.bfloat16))
    Q = torch.randn(n, 2, d, device=DEV, generator=g).to(torch.bfloat16)
    got = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0]), whole([m]), n, m)
    near(got, *O.attention(Q, K.contiguous(), V.contiguous(), 0.1, True, [(n, m)], [0]))
