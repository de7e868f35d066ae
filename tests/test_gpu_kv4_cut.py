"""Sequences that are longer than the caller states: as many queries are answered as it states, each from the keys that it would see among as many as it states."""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.test_gpu_kv4 import BAR, DEV, Problem, rel

# d, page, heads, kv_heads, q_lens, kv_lens, stated max_q and max_kv.  Shared rows whole and in shares, own rows whole and in parts
CASES = {
    "queries": (128, 16, 4, 2, [10, 3], [10, 40], 5, 40), "keys": (64, 16, 2, 1, [10, 10], [100, 30], 10, 50), "both": (128, 16, 2, 2, [8, 1], [70, 30], 3, 66),
    "both, all queries before the first key": (64, 16, 2, 1, [30, 2], [10, 5], 7, 4), "shares": (64, 32, 4, 2, [7, 2, 6], [1600, 40, 1520], 4, 1504),
    "own rows": (128, 16, 2, 1, [120, 70], [130, 200], 80, 96), "own rows in parts": (64, 64, 2, 1, [100, 90], [900, 300], 70, 600), "two tiles in shares": (64, 16, 1, 1, [60, 50], [1400, 60], 40, 1310),
}


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", CASES)
def test_what_is_cut_off_shifts_nothing(name, causal):
    d, page, heads, kv_heads, q_lens, kv_lens, max_q, max_kv = CASES[name]
    p = Problem(len(name), d, page, heads, kv_heads, q_lens, kv_lens, causal=causal)
    out = torch.full((sum(q_lens), heads, d), 7.0, dtype=torch.bfloat16, device=DEV)
    got = p.run(max_q=max_q, max_kv=max_kv, out=out).float().cpu().numpy().astype(np.float64)
    for i, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for j in range(n):
            row = p.starts[i] + j
            if j >= max_q:
                assert (got[row] == 7.0).all()               # not answered, not written
                continue
            seen = min(m, max_kv) if not causal else min(max(m - n + j + 1, 0), max_kv)
            want = kv4.attention(p.turned[row:row + 1], p.k[i][:seen], p.v[i][:seen], p.scale, False)[0]
            if seen == 0:
                assert not got[row].any()
            else:
                assert rel(got[row], want) <= 3 * BAR, (i, j, seen)
