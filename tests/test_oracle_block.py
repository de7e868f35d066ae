"""Pins of oracle/block.py: loops over single numbers, closed forms, and bounds that hold for float32 arithmetic and fail for a mistake."""
import math

import pytest
import torch

from oracle import block as O


def test_attention_is_the_sum_over_visible_keys():
    g = torch.Generator().manual_seed(0)
    lengths, starts, heads, group, d = [(3, 5), (2, 1), (4, 4), (1, 0)], [1, 8, 10, 0], 4, 2, 8
    q, k, v = torch.randn(10, heads, d, generator=g), torch.randn(14, 2, d, generator=g), torch.randn(14, 2, d, generator=g)
    for causal in (True, False):
        got, off = O.attention(q, k, v, 0.7, causal, lengths, starts)
        row = 0
        for (n, m), first in zip(lengths, starts):
            for i in range(n):
                for h in range(heads):
                    seen = [j for j in range(m) if not causal or j <= m - n + i]
                    w = [math.exp(0.7 * sum(float(q[row + i, h, c]) * float(k[first + j, h // group, c]) for c in range(d))) for j in seen]
                    for c in range(d):
                        want = sum(p * float(v[first + j, h // group, c]) for p, j in zip(w, seen)) / sum(w) if seen else 0.0
                        assert abs(float(got[row + i, h, c]) - want) < 1e-12
            row += n
    assert float(off.max()) < 0.05


def test_attention_of_longer_sequences_than_stated():
    q, k, v = (torch.randn(6, 1, 4, generator=torch.Generator().manual_seed(i)) for i in range(3))
    got, _ = O.attention(q, k, v, 1.0, True, [(6, 6)], [0], max_q=4, max_kv=3)
    whole, _ = O.attention(q, k, v, 1.0, True, [(6, 6)], [0])
    assert torch.equal(got[:3], whole[:3]) and not torch.equal(got[3], whole[3]) and not bool(got[4:].any())


@pytest.mark.parametrize("kind", ["layer", "rms", "none"])
def test_norm_and_its_bound(kind):
    g = torch.Generator().manual_seed(1)
    x, gain, bias = torch.randn(50, 96, generator=g) * 3 + 2, torch.randn(96, generator=g), torch.randn(96, generator=g)
    want, off = O.norm(x.double(), kind, 1e-5, gain, bias)
    if kind == "layer":
        y = torch.nn.functional.layer_norm(x, (96,), gain, bias, 1e-5)
    else:
        y = (x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) if kind == "rms" else x) * gain + bias
    assert bool(((y.double() - want).abs() <= off).all()) and float(off.max()) < 1e-3
    assert not bool((((y * (1 + 1e-3)).double() - want).abs() <= off).all())


def test_turn_by_axes():
    g = torch.Generator().manual_seed(2)
    x, table = torch.randn(4, 2, 16, generator=g).double(), torch.randn(9, 16, generator=g)
    positions = torch.tensor([[0, 1, 8, 99], [3, 3, -1, 2]])
    y, off = O.turn(x, torch.zeros_like(x), table, positions, 8)
    for t in range(4):
        for p in range(8):
            row = table[min(max(int(positions[p // 4, t]), 0), 8)].double()
            assert torch.allclose(y[t, :, p], x[t, :, p] * row[p] - x[t, :, p + 8] * row[8 + p], atol=1e-12)
            assert torch.allclose(y[t, :, p + 8], x[t, :, p + 8] * row[p] + x[t, :, p] * row[8 + p], atol=1e-12)
    lanes = torch.tensor([1, 0, 1, 0, 1, 0, 1, 7], dtype=torch.uint8)
    z, _ = O.turn(x, off, table, positions, 8, lanes)
    assert torch.equal(z[..., 1], y[..., 1]) and torch.equal(z[..., 15], y[..., 15])


def test_residual_is_its_formula():
    g = torch.Generator().manual_seed(3)
    x, y, v = torch.randn(5, 8, generator=g), torch.randn(5, 8, generator=g), torch.randn(7, 8, generator=g)
    rows = torch.tensor([0, 2, 1, 9, -1])
    (s, s_off), (h, h_off) = O.residual_norm(x, y, x.dtype, torch.float32, "rms", v[0], v[1], v[2], v[3:6], "layer", v[3], v[4], v[4:7], v[1:4], rows, 1e-5)
    for t in range(5):
        r = min(max(int(rows[t]), 0), 2)
        u = y[t].double() / math.sqrt(float((y[t].double() ** 2).mean()) + 1e-5) * v[0].double() + v[1].double()
        want = x[t].double() + v[2].double() * v[3 + r].double() * u
        mean = want.mean()
        n = (want - mean) / math.sqrt(float(((want - mean) ** 2).mean()) + 1e-5) * v[3].double() + v[4].double()
        assert torch.allclose(s[t], want, atol=1e-12) and torch.allclose(h[t], n * (1 + v[4 + r].double()) + v[1 + r].double(), atol=1e-12)
    assert float(s_off.max()) < 1e-4 and float(h_off.max()) < 1e-3


def test_attention_of_infinite_scores():
    """Zeros are for rows without keys only."""
    q, k, v = (torch.randn(4, 1, 4, generator=torch.Generator().manual_seed(i)) for i in range(3))
    k[:, :, 1] = k[:, :, 1].abs() + 1
    q[2, 0, 1] = -math.inf
    got, _ = O.attention(q, k, v, 1.0, True, [(4, 3)], [0])
    assert bool((got[0] == 0).all()) and bool(torch.isnan(got[2]).all()) and bool(torch.isfinite(got[[1, 3]]).all())
    got, _ = O.attention(q, k, v, 1.0, False, [(4, 3)], [0])
    assert bool(torch.isnan(got[2]).all()) and bool(torch.isfinite(got[[0, 1, 3]]).all())
