"""Attention over the 4-bit key/value cache through every kernel and plan that a call can reach: sizes are stated larger than the sequences are, as a caller that captures a call does, so
that small problems take the plans of large ones.  Bars as in test_gpu_kv4.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import Problem
from tests.test_kv4_plan import plans  # noqa: F401

RNG = np.random.default_rng(0)
MANY = [1] * 65 + [2, 0, 1, 1, 0] + [1] * 30
MANY_KV = [int(n) for n in RNG.integers(0, 40, 64)] + [1300, 5, 0, 0, 77, 9] + [int(n) for n in RNG.integers(0, 90, 29)] + [700]
# d, page, heads, kv_heads, q_lens, kv_lens, causal, stated max_q and max_kv, what the plan has to be: (shared, tiles of 16 rows, ...)
CASES = {
    # own rows, two tiles a wave, 128 channels: whole sequences; parts of the keys, some of which a row does not see
    "own_128_whole": (128, 16, 4, 4, [150, 33, 0, 129], [190, 20, 9, 140], True, 150000, 200, dict(shared=0, nt=2, splits=1)),
    "own_128_whole_all_keys": (128, 64, 2, 1, [70, 5], [33, 199], False, 80000, 200, dict(shared=0, nt=2, splits=1)),
    "own_128_parts": (128, 32, 4, 2, [70, 3, 66], [900, 3, 530], True, 70, 3000, dict(shared=0, nt=2, splits=12)),
    "own_128_parts_all_keys": (128, 16, 2, 2, [70, 65], [600, 255], False, 70, 1500, dict(shared=0, nt=2, splits=6)),
    # four tiles a wave
    "own_64_four": (64, 16, 2, 2, [260, 1, 0, 70], [260, 200, 3, 90], True, 600000, 300, dict(shared=0, nt=4)),
    "own_64_four_all_keys": (64, 32, 2, 1, [130, 20], [100, 190], False, 600000, 200, dict(shared=0, nt=4, splits=1)),
    "own_64_four_parts": (64, 64, 2, 1, [127, 40, 4], [700, 300, 0], True, 250, 8192, dict(shared=0, nt=4, splits=32)),
    "own_64_four_parts_all_keys": (64, 16, 1, 1, [257, 3], [513, 600], False, 500, 8192, dict(shared=0, nt=4, splits=32)),
    "own_64_two_parts": (64, 16, 3, 1, [50, 70], [500, 71], True, 70, 3000, dict(shared=0, nt=2)),
    # shared rows, even shares of all keys: more sequences than a wave has lanes, some without queries or keys
    "shares_of_100": (128, 16, 4, 2, MANY, MANY_KV, True, 2, 1500, dict(shared=1, nt=1, tiles=1, unit_shift=7)),
    "shares_of_100_64": (64, 32, 6, 2, MANY, MANY_KV, True, 2, 1500, dict(shared=1, nt=1, tiles=1)),
    "shares_of_100_two_tiles": (64, 16, 8, 1, MANY, MANY_KV, True, 5, 1500, dict(shared=1, nt=2, tiles=2)),
    # two tiles of rows a head, shares and whole heads
    "shares_two_tiles_128": (128, 32, 8, 2, [12, 9, 1], [1400, 30, 1030], True, 12, 2000, dict(shared=1, nt=2, tiles=2)),
    "shares_two_tiles_64": (64, 16, 1, 1, [40, 17], [1200, 1025], False, 64, 1500, dict(shared=1, nt=2, tiles=2)),
    "shares_32_rows": (128, 16, 4, 1, [8, 5, 0], [1300, 40, 2], True, 8, 1500, dict(shared=1, nt=2, tiles=1)),
    "whole_two_tiles": (128, 16, 3, 1, [20, 7], [60, 900], True, 20, 1000, dict(shared=1, nt=2, tiles=2, blocks=0)),
    # units of 256 keys
    "shares_of_long_units": (64, 1024, 16, 8, [1] * 16, [2900, 1, 255, 256, 257, 0] + [300] * 10, True, 1, 1 << 30, dict(shared=1, nt=1, unit_shift=8)),
}


def test_the_cases_have_the_plans_that_they_are_for(plans):  # noqa: F811
    found = plans([(len(q_lens), max_q, max_kv, heads, kv_heads, d) for d, _, heads, kv_heads, q_lens, _, _, max_q, max_kv, _ in CASES.values()])
    for (name, case), p in zip(CASES.items(), found):
        names = ("shared", "nt", "tiles", "blocks", "unit_shift") if p[0] else ("shared", "nt", "tiles", "chunk", "splits")
        plan = dict(zip(names, p))
        assert case[-1].items() <= plan.items(), (name, plan)
        assert max(case[4]) <= case[7] and max(case[5]) <= case[8]
        if name.startswith("shares"):
            assert plan["blocks"] > 0
        if "parts" in name:
            assert plan["splits"] > 1 and max(case[5]) > plan["chunk"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_attention_of_stated_sizes(name):
    d, page, heads, kv_heads, q_lens, kv_lens, causal, max_q, max_kv, _ = CASES[name]
    p = Problem(len(name), d, page, heads, kv_heads, q_lens, kv_lens, d, d // 2, causal, spare=max_kv // page + 1 - max(-(-m // page) for m in kv_lens))
    p.check(max_q=max_q, max_kv=max_kv)
    again = p.run(max_q=max_q, max_kv=max_kv)
    assert torch.equal(again.view(torch.int16), p.run(max_q=max_q, max_kv=max_kv).view(torch.int16))
