"""GPU parity of qvggt_attention with oracle/block.py (float64), value by value within the bound that the oracle derives."""
import math

import pytest
import torch

import paper_2509_21302_amd as q
from oracle import block as O
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
DEV = G.DEV


def whole(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def starts_of(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def workspace(T, seqs, max_q, max_kv, heads, kv_heads, d, fill=0xff):
    need = q.qvggt_attention_workspace_bytes(T, seqs, max_q, max_kv, heads, kv_heads, d)
    return torch.full((need,), fill, dtype=torch.uint8, device=DEV) if need else None


def attend(Q, K, V, scale, causal, starts, kv_starts, kv_lens, max_q, max_kv, out=None, ws=None):
    T, heads, d = Q.shape
    out = torch.full((T, heads, d), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    ws = workspace(T, starts.numel() - 1, max_q, max_kv, heads, K.shape[1], d) if ws is None else ws
    q.qvggt_attention(Q, K, V, scale, causal, starts, kv_starts, kv_lens, max_q, max_kv, out, ws)
    return out


def inputs(T, S, heads, kv_heads, d, seed, loud=1.5):
    g = torch.Generator(DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    # rows of fused products
    Q = (loud * randn(T, heads + 2, d)).to(torch.bfloat16)[:, 1:heads + 1]
    K, V = (randn(max(S, 1), kv_heads + i, d).to(torch.bfloat16)[:, i:] for i in (1, 2))
    return Q, K, V


def near(got, want, off):
    worst = ((got.double() - want).abs() / off).max() if got.numel() else torch.zeros(())
    assert float(worst) <= 1.0, float(worst)


@pytest.mark.parametrize("heads,kv_heads,d,causal,q_lens", [
    (1, 1, 64, True, [1]), (2, 1, 128, True, [2]), (16, 16, 64, False, [70, 1, 129]), (8, 2, 128, True, [33, 0, 200, 64]), (4, 4, 128, True, [128, 65]),
    (6, 6, 64, True, [257]), (7, 1, 128, False, [61, 63, 64]), (12, 3, 64, True, [31, 500]), (2, 2, 128, False, [1030]), (64, 1, 64, True, [90]), (3, 3, 128, True, [385, 1, 1, 2])])
def test_packed(heads, kv_heads, d, causal, q_lens):
    starts, T = starts_of(q_lens), sum(q_lens)
    Q, K, V = inputs(T, T, heads, kv_heads, d, T)
    at = whole(starts)
    got = attend(Q, K, V, 1 / math.sqrt(d), causal, at, at, None, max(q_lens), max(q_lens))
    near(got, *O.attention(Q, K, V, 1 / math.sqrt(d), causal, [(n, n) for n in q_lens], starts))


@pytest.mark.parametrize("heads,kv_heads,d,causal,lengths,slack", [
    (32, 8, 128, True, [(1, 601)], 0), (8, 8, 64, True, [(1, 1), (1, 0), (1, 64), (1, 65), (1, 1000)], 5), (4, 1, 128, True, [(3, 700), (8, 8), (5, 3), (1, 0)], 1),
    (16, 2, 64, True, [(4, 5000), (2, 128)], 3), (8, 8, 128, True, [(30, 4096), (17, 33)], 0), (8, 4, 128, True, [(61, 9000), (40, 100)], 7), (4, 4, 64, True, [(100, 6001)], 0),
    (5, 5, 128, False, [(50, 3000), (7, 0), (20, 1)], 2), (2, 1, 64, False, [(200, 31), (16, 4000)], 0), (1, 1, 64, True, [(1, 20000)], 0), (32, 1, 128, True, [(1, 3333)], 1),
    (1, 1, 128, True, [(300, 40)], 0), (33, 1, 64, True, [(1, 2049)], 9), (2, 2, 64, True, [(64, 33000)], 0)])
def test_buffers(heads, kv_heads, d, causal, lengths, slack):
    """Keys in a buffer for every sequence; what lies behind their ends is no number."""
    q_lens, kv_lens = zip(*lengths)
    T, capacity = sum(q_lens), max(kv_lens) + slack
    Q, K, V = inputs(T, capacity * len(lengths), heads, kv_heads, d, T + capacity)
    first = [i * capacity for i in range(len(lengths))]
    for i, n in enumerate(kv_lens):
        K[first[i] + n:first[i] + capacity] = math.nan
        V[first[i] + n:first[i] + capacity] = math.inf
    got = attend(Q, K, V, 0.1, causal, whole(starts_of(q_lens)), whole(first), whole(kv_lens), max(q_lens), max(kv_lens))
    near(got, *O.attention(Q, K, V, 0.1, causal, lengths, first))


@pytest.mark.parametrize("d,n,m,group", [(64, 1, 500, 4), (128, 1, 500, 4), (64, 150, 150, 1), (128, 150, 150, 1), (128, 40, 3000, 2), (64, 20, 3000, 1)])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-30, 4.0])
def test_scales(d, n, m, group, scale):
    """Negative ones turn the order of the scores around, 0 gives the mean; large ones leave a key or two."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    got = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    near(got, *O.attention(Q, K, V, scale, True, [(n, m)], [0]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", [(8, 33, 4), (4, 70, 1), (30, 98, 1), (40, 20, 1), (300, 40, 2), (20, 5, 1), (61, 3010, 4)])
@pytest.mark.parametrize("scale", [0.79, 1.0, -4.0, 1e4])
def test_rows_that_see_nothing_of_a_step_at_large_scales(d, n, m, group, scale):
    """A starting maximum times the scale has no place in fp32; rows without keys, and waves whose keys a row does not see, add zeros all the same."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    if abs(scale) > 100:
        Q[:], K[:] = Q / 128, K / 128
    got = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    assert bool(torch.isfinite(got.float()).all())
    near(got, *O.attention(Q, K, V, scale, True, [(n, m)], [0]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m", [(1, 900), (130, 130), (40, 2500), (700, 700)])
def test_scores_rise_along_the_keys(d, n, m):
    """Every step has a new maximum, by much and by little; and falls: all later weights vanish."""
    Q, K, V = inputs(n, m, 2, 2, d, 5)
    at = torch.arange(m, device=DEV)[:, None, None]
    for slope in (0.02, 0.3, -0.3):
        Q[:] = 1.0
        K[:] = (slope * at + 0.01 * torch.randn(m, 2, d, device=DEV, generator=torch.Generator(DEV).manual_seed(1))).to(torch.bfloat16)
        got = attend(Q, K, V, 1 / d, True, whole([0, n]), whole([0, m]), None, n, m)
        near(got, *O.attention(Q, K, V, 1 / d, True, [(n, m)], [0]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", [(1, 333, 4), (8, 333, 2), (200, 200, 1), (200, 333, 2), (60, 5000, 1)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_no_numbers_stay_with_the_rows_that_see_them(d, n, m, group, bad):
    Q, K, V = inputs(n, m, 2 * group, 2, d, 9)
    clean = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    key = m - 1 - n // 2                    # rows from n - 1 - n // 2 on see it
    V[key, 1, 5] = bad
    V[key, 1, d - 1] = bad
    got = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    seen = torch.zeros(n, 2 * group, d, dtype=torch.bool, device=DEV)
    seen[n - 1 - n // 2:, group:, 5] = True
    seen[n - 1 - n // 2:, group:, d - 1] = True
    assert torch.equal(got[~seen], clean[~seen]) and not bool(torch.isfinite(got[seen].float()).any())
    V[key, 1] = 0.0
    clean = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    K[key, 1, 3] = math.nan
    got = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    rows = torch.zeros(n, 2 * group, dtype=torch.bool, device=DEV)
    rows[n - 1 - n // 2:, group:] = True
    assert torch.equal(got[~rows], clean[~rows]) and bool(torch.isnan(got[rows].float()).all())
    K[key, 1, 3] = 0.0
    clean = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    Q[n // 2, group, 7] = bad
    got = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    rows[:] = False
    rows[n // 2, group] = True
    assert torch.equal(got[~rows], clean[~rows]) and bool(torch.isnan(got[rows].float()).all())


@pytest.mark.parametrize("d,n,m", [(64, 1, 3000), (128, 1, 3000), (128, 200, 200), (64, 50, 6000)])
def test_a_constant_value_comes_back(d, n, m):
    """Weights are divided by the sum of what they were rounded to: values that are all alike are the result, but for sums in fp32."""
    Q, K, V = inputs(n, m, 4, 2, d, 3)
    V[:] = 1.7109375
    got = attend(Q, K, V, 0.2, True, whole([0, n]), whole([0, m]), None, n, m)
    assert bool((got == 1.7109375).all())


def test_rows_of_no_sequence_stay():
    Q, K, V = inputs(300, 300, 4, 2, 64, 1)
    out = torch.full((300, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    at = whole([10, 40, 200])
    attend(Q, K, V, 0.1, True, at, at, None, 160, 160, out)
    assert bool((out[:10] == 7).all()) and bool((out[200:] == 7).all()) and not bool((out[10:200] == 7).any())
    want, off = O.attention(Q[10:], K[10:], V[10:], 0.1, True, [(30, 30), (160, 160)], [0, 30])
    near(out[10:200], want[:190], off[:190])


@pytest.mark.parametrize("heads,kv_heads,d,n,m,max_q,max_kv", [(4, 2, 64, 50, 700, 33, 600), (4, 2, 128, 300, 300, 290, 299), (8, 2, 128, 6, 5000, 4, 4100), (2, 2, 64, 1, 9, 1, 4)])
def test_longer_than_stated(heads, kv_heads, d, n, m, max_q, max_kv):
    Q, K, V = inputs(n, m, heads, kv_heads, d, 8)
    for causal in (True, False):
        got = attend(Q, K, V, 0.1, causal, whole([0, n]), whole([0, m]), None, max_q, max_kv)
        want, off = O.attention(Q, K, V, 0.1, causal, [(n, m)], [0], max_q, max_kv)
        near(got[:max_q], want[:max_q], off[:max_q])
        assert bool((got[max_q:] == 7).all())


def test_starts_and_lengths_outside_of_the_tensors_are_cut():
    Q, K, V = inputs(100, 120, 2, 2, 64, 4)
    got = attend(Q, K, V, 0.1, True, whole([-5, 40, 1000]), whole([-3, 100]), whole([60, 1 << 30]), 100, 120)
    want, off = O.attention(Q, K, V, 0.1, True, [(40, 60), (60, 20)], [0, 100])
    near(got, want, off)
    got = attend(Q, K, V, 0.1, False, whole([0, 50, 100]), whole([500, 30]), whole([10, -4]), 100, 120)
    assert bool((got == 0).all())
    got = attend(Q, K, V, 0.1, False, whole([0, 50, 100]), whole([30, -(1 << 31), 1 << 30]), None, 100, 120)
    assert bool((got[:50] == 0).all())
    want, off = O.attention(Q[50:], K, V, 0.1, False, [(50, 120)], [0])
    near(got[50:], want, off)


@pytest.mark.parametrize("d,n,m", [(64, 1, 40000), (128, 2, 70000)])
def test_long(d, n, m):
    Q, K, V = inputs(n, m, 8, 2, d, 6)
    got = attend(Q, K, V, 1 / math.sqrt(d), True, whole([0, n]), whole([0, m]), None, n, m)
    near(got, *O.attention(Q, K, V, 1 / math.sqrt(d), True, [(n, m)], [0]))


@pytest.mark.parametrize("n", [1, 140])
def test_offsets_past_32_bits(n):
    """Keys of a sequence that begin 2^32 bytes behind the tensor's start, rows far apart."""
    d, m, stride = 128, 1200, 1 << 21
    base = torch.empty((m + 1100) * stride, dtype=torch.bfloat16, device=DEV)
    K = base.as_strided((m + 1100, 1, d), (stride, d, 1))
    V = base[d:].as_strided((m + 1100, 1, d), (stride, d, 1))
    g = torch.Generator(DEV).manual_seed(2)
    for t in (K, V):
        t.copy_(torch.randn(m + 1100, 1, d, device=DEV, generator=g).to(torch.bfloat16))
    Q = torch.randn(n, 4, d, device=DEV, generator=g).to(torch.bfloat16)
    got = attend(Q, K, V, 0.1, True, whole([0, n]), whole([1100]), whole([m]), n, m)
    near(got, *O.attention(Q, K[1100:].contiguous(), V[1100:].contiguous(), 0.1, True, [(n, m)], [0]))


def test_the_same_call_gives_the_same_bits():
    for n, m in ((1, 9000), (60, 9000), (700, 700)):
        Q, K, V = inputs(n, m, 8, 2, 128, 2)
        a, b = (attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m) for _ in range(2))
        assert torch.equal(a, b)


def test_another_stream_and_a_captured_call_with_other_lengths():
    """Lengths are read on the device: a captured call is replayed with others."""
    Q, K, V = inputs(4, 4 * 900, 8, 2, 128, 7)
    starts, first, lens = whole([0, 1, 2, 3, 4]), whole([0, 900, 1800, 2700]), whole([900, 1, 30, 700])
    ws, out = workspace(4, 4, 1, 900, 8, 2, 128), torch.empty(4, 8, 128, dtype=torch.bfloat16, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = attend(Q, K, V, 0.1, True, starts, first, lens, 1, 900)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    q.qvggt_init()
    with torch.cuda.graph(graph):
        q.qvggt_attention(Q, K, V, 0.1, True, starts, first, lens, 1, 900, out, ws)
    graph.replay()
    assert torch.equal(out, other)
    for now in ([900, 1, 30, 700], [5, 900, 0, 64], [1, 1, 1, 1], [899, 333, 900, 2]):
        lens.copy_(whole(now))
        Q.copy_(Q.flip(0))
        eager = attend(Q, K, V, 0.1, True, starts, first, lens, 1, 900)
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(out, eager)
        near(out, *O.attention(Q, K, V, 0.1, True, [(1, n) for n in now], [0, 900, 1800, 2700]))


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    """Sequences of any lengths, groups of any size, buffers and packed rows, as one call."""
    import random
    rng = random.Random(seed)
    d, group, kv_heads, causal = rng.choice((64, 128)), rng.choice((1, 2, 3, 5, 7, 8, 12)), rng.choice((1, 2, 3, 8)), rng.random() < 0.6
    seqs, top_q, top_kv = rng.choice((1, 2, 5, 9)), rng.choice((1, 1, 3, 30, 200)), rng.choice((1, 40, 300, 2000))
    lengths = [(rng.randint(0 if i else 1, top_q), rng.randint(0 if i else 1, top_kv)) for i in range(seqs)]
    q_lens, kv_lens = zip(*lengths)
    T, slack = sum(q_lens), rng.randint(0, 5)
    capacity = max(kv_lens) + slack
    packed = rng.random() < 0.5
    first = starts_of(kv_lens) if packed else [i * capacity for i in range(seqs)]
    S = first[-1] if packed else seqs * capacity
    Q, K, V = inputs(T, S, group * kv_heads, kv_heads, d, seed, rng.choice((0.3, 1.5, 6.0)))
    got = attend(Q, K, V, 0.125, causal, whole(starts_of(q_lens)), whole(first), None if packed else whole(kv_lens), max(q_lens) + rng.randint(0, 3), max(kv_lens) + rng.randint(0, 3))
    near(got, *O.attention(Q, K, V, 0.125, causal, lengths, first))


def test_without_any_keys():
    Q, K, V = inputs(40, 1, 4, 2, 64, 1)
    for n in (1, 40):
        got = attend(Q[:n], K[:0], V[:0], 0.1, True, whole([0, n]), whole([0, 0]), None, n, 0)
        assert bool((got == 0).all())
        got = attend(Q[:n], K, V, 0.1, False, whole([0, n]), whole([1]), whole([5]), n, 300)
        assert bool((got == 0).all())


def test_rows_past_2_to_the_31():
    """The most sequences that a call takes; queries and results of more than 2^31 values."""
    seqs, n, heads, d = 65535, 5, 64, 128
    T = seqs * n
    Q, K, V = (torch.zeros(T, heads, d, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    g = torch.Generator(DEV).manual_seed(1)
    for t in (Q, K, V):
        t[-4 * n:] = torch.randn(4 * n, heads, d, device=DEV, generator=g).to(torch.bfloat16)
    at = torch.arange(seqs + 1, dtype=torch.int32, device=DEV) * n
    out = torch.full_like(Q, 7.0)
    q.qvggt_attention(Q, K, V, 0.1, True, at, at, None, n, n, out, workspace(T, seqs, n, n, heads, heads, d))
    near(out[-4 * n:], *O.attention(Q[-4 * n:], K[-4 * n:], V[-4 * n:], 0.1, True, [(n, n)] * 4, [0, n, 2 * n, 3 * n]))
    assert not bool(out[:-4 * n].any())
