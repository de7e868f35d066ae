"""What attention over the 4-bit key/value cache makes of keys, values and queries at the ends of the number range and beyond it: what a row does not see must not matter, whatever it is;
what it sees and is no number must show.  Bars as in test_gpu_kv4.py."""
import numpy as np
import pytest

from oracle import kv4
from tests.test_gpu_kv4 import BAR, Problem, rel

pytestmark = pytest.mark.gpu
# sizes and stated sizes (max_q, max_kv) that take each kernel: shared rows of one and two tiles, whole and in shares; own rows of one, two and four tiles, whole and in parts
KERNELS = {
    "shared": (128, 16, 4, 2, [5, 1], [60, 33], 5, 100), "shared_64": (64, 16, 2, 2, [9, 3], [60, 20], 9, 100), "shared_two_tiles": (64, 16, 2, 1, [30, 17], [60, 64], 30, 100),
    "shares": (128, 16, 4, 2, [5, 1], [1300, 33], 5, 1500), "shares_two_tiles": (128, 32, 4, 1, [12, 4], [1200, 40], 12, 1500),
    "own_64": (64, 16, 2, 2, [70, 40], [90, 64], 70, 100), "own_128": (128, 16, 2, 1, [40, 40], [77, 41], 40, 100), "own_128_two": (128, 16, 2, 2, [100, 40], [150, 47], 150000, 200),
    "own_64_four": (64, 16, 1, 1, [130, 70], [150, 70], 600000, 200), "own_64_four_parts": (64, 32, 1, 1, [257, 70], [513, 300], 500, 8192), "own_128_parts": (128, 16, 2, 1, [70, 40], [600, 300], 70, 3000),
}


def problem(name, causal=True, **kw):
    d, page, heads, kv_heads, q_lens, kv_lens, max_q, max_kv = KERNELS[name]
    p = Problem(len(name), d, page, heads, kv_heads, q_lens, kv_lens, causal=causal, spare=max_kv // page + 1, **kw)
    return p, dict(max_q=max_q, max_kv=max_kv)


def want_of_what_is_seen(p):
    """Attention of every row over the keys that it sees and no others; NaN where one of them is no number."""
    out = []
    for i, (n, k, v) in enumerate(zip(p.q_lens, p.k, p.v)):
        rows = p.turned[p.starts[i]:p.starts[i + 1]]
        for j in range(n):
            seen = min(max(len(k) - n + j + 1, 0), len(k)) if p.causal else len(k)
            bad = ~(np.isfinite(k[:seen]).all((0, 2)) & np.isfinite(v[:seen]).all((0, 2)) if seen else np.ones(p.kv_heads, bool))
            with np.errstate(all="ignore"):
                o = kv4.attention(rows[j:j + 1], k[:seen], v[:seen], p.scale, False)
            o[:, np.repeat(bad, p.heads // p.kv_heads)] = np.nan
            out.append(o)
    return np.concatenate(out)


def check(p, sizes, bar=BAR):
    """Rows of numbers as near as ever, row by row; the others NaN throughout."""
    got, want = p.run(**sizes).float().cpu().numpy().astype(np.float64), want_of_what_is_seen(p)
    none = np.isnan(want)
    assert none.any(-1).sum() == none.all(-1).sum()
    assert np.array_equal(np.isnan(got), none)
    got, want = np.where(none, 0, got), np.where(none, 0, want)
    assert rel(got, want) <= bar
    assert (np.linalg.norm(got - want, axis=-1) <= 3 * bar * (np.linalg.norm(want, axis=-1) + 0.05)).all()
    return none.all(-1)


def at_the_end(p, places, value):
    """A factor of the steps: `value` at the given places from the end of the longer sequence."""
    n = max(p)
    return lambda t: np.where((len(t) == n) & np.isin(n - t, places), value, 1.0)


@pytest.mark.parametrize("name", KERNELS)
def test_values_that_are_no_numbers_where_rows_do_not_see_them(name):
    """A step that is no number, as qvggt_kv4_append leaves it for a row that has an infinity or a NaN, in two values near the end: rows in front of them have none of it."""
    p, sizes = problem(name, v_scale=at_the_end(KERNELS[name][5], (1, 3), np.nan))
    none = check(p, sizes)
    assert none.any() and not none.all()


@pytest.mark.parametrize("place", [(1, 3), (30,)])
@pytest.mark.parametrize("name", KERNELS)
def test_keys_that_are_no_numbers(name, place):
    """The same of keys: rows that see one are no numbers, the others as ever."""
    p, sizes = problem(name, k_scale=at_the_end(KERNELS[name][5], place, np.nan))
    none = check(p, sizes)
    assert none.any() and not none.all()


@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("name", KERNELS)
def test_rows_that_see_everything(name, which):
    p, sizes = problem(name, causal=False, **{which: at_the_end(KERNELS[name][5], (20,), np.nan)})
    none = check(p, sizes)
    assert none.any() and not none.all()


@pytest.mark.parametrize("name", KERNELS)
def test_keys_of_all_sizes(name):
    """Steps from 0 to 2^8 of the ordinary one: a score's error grows with the score (2^-12 of the terms of its product), so the weights are those of scores up to some tens."""
    p, sizes = problem(name, loud=2.0 ** -7, k_scale=lambda t: np.where(t % 5 == 0, 0.0, 2.0 ** (t % 9)))
    check(p, sizes)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("name", KERNELS)
def test_queries_that_are_no_numbers(name, value, dtype):
    """One head of one token: its row is no number, its neighbours in the same tile are as ever."""
    p, sizes = problem(name, dtype=dtype)
    token = p.q_lens[0] // 2
    p.qd[token, -1, 7] = value
    got, want = p.run(**sizes).float().cpu().numpy().astype(np.float64), p.want()
    assert np.isnan(got[token, -1]).all()
    got[token, -1] = want[token, -1] = 0
    assert np.isfinite(got).all() and rel(got, want) <= BAR
    assert (np.linalg.norm(got - want, axis=-1) <= 3 * BAR * (np.linalg.norm(want, axis=-1) + 0.05)).all()
