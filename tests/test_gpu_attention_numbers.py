"""What qvggt_attention makes of queries, keys and scales at the ends of the number range: a row that sees a key has weights that add up to one, or is no number; only a row without keys is zeros.
Through every kernel: few rows and many, keys whole and in parts."""
import math

import pytest
import torch

from oracle import block as O
from tests import gpu_util as G
from tests.test_gpu_attention import attend, inputs, near, whole

pytestmark = pytest.mark.gpu
DEV = G.DEV

# query tokens, keys, query heads of a key head: few rows of one tile and of two, whole and in parts; many rows, whole and in parts
KERNELS = [(1, 1, 1), (1, 40, 4), (5, 5, 2), (9, 70, 3), (3, 9000, 2), (8, 9000, 4), (60, 60, 1), (130, 130, 2), (200, 333, 1), (60, 9000, 2)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", KERNELS)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("scale", [0.1, -0.1, 3.0])
def test_rows_of_infinite_scores_of_one_sign(d, n, m, group, bad, scale):
    """An infinity in a query whose keys all have one sign there: scores of one infinity, whichever it is, have no softmax; other rows keep their bits."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    K[:, :, 7] = K[:, :, 7].abs() + 0.5
    clean = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    near(clean, *O.attention(Q, K, V, scale, True, [(n, m)], [0]))
    rows = torch.zeros(n, 2 * group, dtype=torch.bool, device=DEV)
    for i, h in ((0, 0), (n // 2, group), (n - 1, 2 * group - 1)):
        Q[i, h, 7] = bad
        rows[i, h] = True
    got = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    assert torch.equal(got[~rows], clean[~rows])
    assert bool(torch.isnan(got[rows].float()).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", KERNELS)
def test_a_key_at_minus_infinity(d, n, m, group):
    """It has no weight beside others; a row that sees it alone is no number."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    Q[:, :, 7] = Q[:, :, 7].abs() + 0.5
    K[0, :, 7] = -math.inf
    got = attend(Q, K, V, 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    alone = m - n + 1 == 1
    if alone:
        assert bool(torch.isnan(got[0].float()).all())
    if n > alone and m > 1:
        want, off = O.attention(Q, K[1:], V[1:], 0.1, True, [(n, m - 1)], [0])
        near(got[int(alone):], want[int(alone):], off[int(alone):])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", [(3, 0, 2), (9, 4, 3), (20, 5, 1), (61, 40, 1), (300, 40, 2)])
def test_rows_that_see_no_key_are_zeros_whatever_they_are(d, n, m, group):
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    Q[:n - m, :, 7] = math.inf
    Q[n - m - 1, 0, 9] = math.nan
    got = attend(Q, K[:m], V[:m], 0.1, True, whole([0, n]), whole([0, m]), None, n, m)
    assert bool((got[:n - m] == 0).all()) and bool(torch.isfinite(got.float()).all())


def whole_scores(n, m, group, d, seed, values, only=None):
    """Queries of +-1 in one channel over keys of whole numbers there: scores without any rounding, the largest of them (several, at times) every far scale's choice."""
    g = torch.Generator(DEV).manual_seed(seed)
    Q, K, V = inputs(n, m, 2 * group, 2, d, seed)
    Q[:], K[:] = 0.0, 0.0
    Q[:, :, 3] = torch.where(torch.rand(n, 2 * group, device=DEV, generator=g) < 0.5, -1.0, 1.0).to(torch.bfloat16)
    K[:, :, 3] = torch.tensor(values, device=DEV)[torch.randint(len(values), (m, 2), device=DEV, generator=g)].to(torch.bfloat16)
    return Q, K, V


def means_of_the_largest(Q, K, V, sign, n, m):
    """(out, bound): the mean of the values of the keys with the row's largest score, weights of 1 exactly: a sum in fp32, a quotient (1 / total and a product) and the rounding of the result."""
    group = Q.shape[1] // K.shape[1]
    out, off = (torch.zeros(Q.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    for h in range(Q.shape[1]):
        x = sign * Q[:, h].double() @ K[:, h // group].double().T.contiguous()
        x = x.masked_fill(torch.arange(m, device=DEV) > m - n + torch.arange(n, device=DEV)[:, None], -math.inf)
        p = (x == x.amax(-1, keepdim=True)).double()
        p /= p.sum(-1, keepdim=True)
        v = V[:, h // group].double()
        out[:, h] = p @ v
        off[:, h] = O.rounded(out[:, h], (m + 8) * O.U * (p @ v.abs()), torch.bfloat16)
    return out, off


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", KERNELS)
@pytest.mark.parametrize("scale", [1e3, 1e7, -1e12, 1e30, -1e37, 1e38, -1e38])
@pytest.mark.parametrize("values", [[-8.0, -5.0, -2.0, 1.0, 2.0, 5.0, 8.0], [-5.0, -7.0], [5.0, 6.0, 7.0], [5.0]])
def test_far_scales_choose_the_largest_scores(d, n, m, group, scale, values):
    """Scores times the scale may lie as far out as they like, past fp32 too: weights are of differences.  (A difference of 1 is one of 1000 at least: a weight of 0.)"""
    Q, K, V = whole_scores(n, m, group, d, n + m, values)
    got = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    near(got, *means_of_the_largest(Q, K, V, math.copysign(1.0, scale), n, m))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", KERNELS)
@pytest.mark.parametrize("scale", [0.25, -0.25, 2.0])
def test_scores_far_from_zero_keep_their_differences(d, n, m, group, scale):
    """Scores of 2^20 and a few units, rising along the keys, exact in fp32: weights are those of the units.  The bound is of the units alone: weights rounded to bf16 (2^-8), an exponent of at most
    2^6 that is off by two halves of a step, sums, the result's rounding."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    Q[:], K[:] = 0.0, 0.0
    Q[:, :, 0], Q[:, :, 1] = 1024.0, 1.0
    K[:, :, 0] = 1024.0
    K[:, :, 1] = (torch.arange(m, device=DEV)[:, None] * 37 % 11 + torch.arange(m, device=DEV)[:, None] * 120 // m).to(torch.bfloat16)
    if scale < 0:
        Q[:, :, 1], K[:, :, 0] = -1.0, -1024.0
    got = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    Q[:, :, 0] = 0.0                        # a score common to all keys: the same softmax
    want, _ = O.attention(Q, K, V, scale, True, [(n, m)], [0])
    off = torch.zeros_like(want)
    for h in range(2 * group):
        x = scale * (Q[:, h].double() @ K[:, h // group].double().T.contiguous())
        x = x.masked_fill(torch.arange(m, device=DEV) > m - n + torch.arange(n, device=DEV)[:, None], -math.inf)
        p, v = torch.softmax(x, -1), V[:, h // group].double()
        spread = torch.stack([(p * (v[:, c] - want[:, h, c:c + 1]).abs()).sum(1) for c in range(d)], 1)
        off[:, h] = O.rounded(want[:, h], (2.0 ** -8 + 2 ** 7 * O.U) * 1.01 * spread + (m + 64) * O.U * (p @ v.abs() + want[:, h].abs()), torch.bfloat16)
    near(got, want, off)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", KERNELS)
def test_far_scales_of_small_queries_and_keys(d, n, m, group):
    """Powers of two in the scale for those in queries and keys: the same scores, the same bits."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    want = attend(Q, K, V, 0.125, True, whole([0, n]), whole([0, m]), None, n, m)
    K[:] = K * 2.0 ** -60
    Q[:] = Q * 2.0 ** -30
    assert torch.equal(attend(Q, K, V, 0.125 * 2.0 ** 90, True, whole([0, n]), whole([0, m]), None, n, m), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m,group", KERNELS)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("scale", [0.0, -0.0])
def test_a_scale_of_zero_makes_no_number_of_an_infinite_query(d, n, m, group, bad, scale):
    """0 times a score that is no number is none; rows of numbers are the mean of the values they see."""
    Q, K, V = inputs(n, m, 2 * group, 2, d, n + m)
    Q[n // 2, group, 7] = bad
    Q[n - 1, 0, d - 2] = bad
    got = attend(Q, K, V, scale, True, whole([0, n]), whole([0, m]), None, n, m)
    rows = torch.zeros(n, 2 * group, dtype=torch.bool, device=DEV)
    rows[n // 2, group] = rows[n - 1, 0] = True
    assert bool(torch.isnan(got[rows].float()).all())
    Q[n // 2, group, 7] = Q[n - 1, 0, d - 2] = 0.0
    want, off = O.attention(Q, K, V, 0.0, True, [(n, m)], [0])
    near(got[~rows], want[~rows], off[~rows])
