"""Attention over very many keys in the 4-bit key/value cache, all of the same weight: what a wave sums is the small difference of numbers that grow with every key.

The result is the mean of the values, some 1 / sqrt(keys) of one of them, from weights of 2^7 or less times a step in fp16 (2^-12 of each: they add up as the values themselves do, so 2^-12 of
the result, rms) and codes that are exact.  What fp32 sums add: the differences from folding every few hundred steps, below 2^-24 times 8 times the sum of those steps' weights each, together
below 1e-4 of the mean at 2^20 keys; a sum of n terms 2^-25 sqrt(n), 1e-5.  So the bar is that of test_gpu_kv4.py, 4e-3 of the row, mostly its rounding to bf16."""
import numpy as np
import pytest
import torch

import paper_2509_21302_amd as q
from tests.test_gpu_kv4 import BAR, DEV, dev, rel
from tests.test_kv4_plan import plans  # noqa: F401

PAGE, N = 1024, 1 << 20
# d, sequences, rows of the first, stated max_q: who sums how many keys
CASES = {"own rows, one wave, 2^20 keys": (64, 1, 70, 1 << 28, 0), "own rows of 128 channels, the same": (128, 1, 70, 1 << 28, 0), "own rows in parts of 2^15": (64, 1, 70, 70, 32),
         "shared rows, four waves": (128, 513, 1, 1, 0), "shared rows of 64 channels": (64, 513, 2, 2, 0), "shared rows, two tiles": (64, 513, 40, 40, 0)}


def test_the_cases_have_the_plans_that_they_are_for(plans):  # noqa: F811
    for name, (d, seqs, rows, max_q, splits) in CASES.items():
        p, = plans([(seqs, max_q, N, 1, 1, d)])
        if "own" in name:
            assert p[0] == 0 and p[4] == max(splits, 1), (name, p)
        else:
            assert p[0] == 1 and p[3] == 0, (name, p)


def test_a_wave_of_own_rows_adds_up_a_million_keys_at_most(plans):  # noqa: F811
    """... where there may be parts: 32 at most, and fewer than 2^20 blocks in all."""
    problems = [(seqs, max_q, (1 << 20) * n + extra, 8 * group, 8, d) for seqs in (1, 3) for max_q in (65, 4096, 100000) for n in (1, 2, 7, 31, 32, 100) for extra in (0, 1, 12345)
                for group in (1, 4) for d in (64, 128) if n < 32 or n == 32 and extra == 0 or n == 100]
    for problem, (shared, _, tiles, chunk, splits, *_) in zip(problems, plans(problems)):
        if not shared:
            no_more = splits in (31, 32) and problem[2] > 1 << 25 or problem[0] * 8 * tiles * (splits + 1) >= 1 << 20
            assert chunk <= 1 << 20 or no_more, (problem, chunk, splits)


@pytest.fixture(scope="module")
def pools():
    made = {}

    def pool(d):
        if d not in made:
            g = torch.Generator(DEV).manual_seed(d)
            cache = torch.zeros(N // PAGE, q.qvggt_kv4_page_bytes(PAGE, 1, d), dtype=torch.uint8, device=DEV)
            mean = torch.zeros(1, d, dtype=torch.float64, device=DEV)
            for i in range(0, N, 1 << 17):
                slots = torch.arange(i, i + (1 << 17), dtype=torch.int32, device=DEV)
                x = torch.randn(1 << 17, 2, d, device=DEV, generator=g)
                q.qvggt_kv4_append(x[:, :1], x[:, 1:], None, slots, cache, PAGE)
                v = torch.empty(1 << 17, 1, d, device=DEV)
                q.qvggt_kv4_read(cache, PAGE, None, slots, None, v)
                mean += v.double().sum(0)
            made[d] = cache, (mean / N).cpu().numpy()
        return made[d]
    return pool


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_the_mean_of_many_values(pools, name):
    d, seqs, rows, max_q, _ = CASES[name]
    cache, want = pools(d)
    table = torch.arange(N // PAGE, dtype=torch.int32, device=DEV).expand(seqs, -1).contiguous()
    starts, lens = np.full(seqs + 1, rows, np.int32), np.zeros(seqs, np.int32)
    starts[0], lens[0] = 0, N
    queries = torch.zeros(rows, 1, d, device=DEV)            # every score is 0
    out = torch.full((rows, 1, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    size = q.qvggt_kv4_attention_workspace_bytes(rows, seqs, max_q, N, 1, 1, d)
    q.qvggt_kv4_attention(queries, None, 0.1, False, cache, PAGE, 1, table, dev(starts), dev(lens), max_q, N, out, torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)
    got = out.float().cpu().numpy().astype(np.float64)
    errors = [rel(got[i], want) for i in range(rows)]
    print(name, max(errors))
    assert max(errors) <= BAR
