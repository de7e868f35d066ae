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
