"""What attention over the 4-bit key/value cache makes of keys, values and queries at the ends of the number range and beyond it: what a row does not see must not matter, whatever it is;
what it sees and is no number must show.  Bars as in test_gpu_kv4.py."""
import numpy as np
import pytest
import torch

import paper_2509_21302_amd as q
from oracle import kv4
from tests.test_gpu_kv4 import BAR, DEV, Problem, dev, rel, signs_of, table_of

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


@pytest.mark.gpu
@pytest.mark.parametrize("name", KERNELS)
def test_values_that_are_no_numbers_where_rows_do_not_see_them(name):
    """A step that is no number, as qvggt_kv4_append leaves it for a row that has an infinity or a NaN, in two values near the end: rows in front of them have none of it."""
    p, sizes = problem(name, v_scale=at_the_end(KERNELS[name][5], (1, 3), np.nan))
    none = check(p, sizes)
    assert none.any() and not none.all()


@pytest.mark.gpu
@pytest.mark.parametrize("place", [(1, 3), (30,)])
@pytest.mark.parametrize("name", KERNELS)
def test_keys_that_are_no_numbers(name, place):
    """The same of keys: rows that see one are no numbers, the others as ever."""
    p, sizes = problem(name, k_scale=at_the_end(KERNELS[name][5], place, np.nan))
    none = check(p, sizes)
    assert none.any() and not none.all()


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("name", KERNELS)
def test_rows_that_see_everything(name, which):
    p, sizes = problem(name, causal=False, **{which: at_the_end(KERNELS[name][5], (20,), np.nan)})
    none = check(p, sizes)
    assert none.any() and not none.all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", KERNELS)
def test_keys_of_all_sizes(name):
    """Steps from 0 to 2^8 of the ordinary one: a score's error grows with the score (2^-12 of the terms of its product), so the weights are those of scores up to some tens."""
    p, sizes = problem(name, loud=2.0 ** -7, k_scale=lambda t: np.where(t % 5 == 0, 0.0, 2.0 ** (t % 9)))
    check(p, sizes)


@pytest.mark.gpu
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


@pytest.mark.gpu
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf, 3e38])
@pytest.mark.parametrize("d,page,heads,T,pair,dtype,scattered", [(64, 16, 2, 41, 16, torch.bfloat16, False), (128, 32, 3, 41, 64, torch.float32, False),
                                                                 (64, 32, 3, 37, 0, torch.float32, True), (128, 16, 2, 37, 1, torch.bfloat16, True)])
def test_append_of_rows_that_are_no_numbers(d, page, heads, T, pair, dtype, scattered, value):
    """A key's head in one token and a value's in another (a number so large that 64 of them overflow, too): steps that are NaN and codes 0 there, every other byte as without them."""
    rng = np.random.default_rng(T)
    x = torch.from_numpy(rng.standard_normal((T, 2 * heads, d))).to(dtype)
    bad = x.clone()
    everywhere = slice(None) if value == 3e38 else slice(5, 6)
    bad[9, 1, everywhere], bad[20, heads, everywhere] = value, value
    if value == 3e38:
        signs, pair = None, 0                                # equal numbers add up in the first channel
    else:
        signs = dev(signs_of(rng, d))
    table, positions = dev(table_of(rng, 50, d if pair else 0)), dev(rng.integers(0, 50, T).astype(np.int32))
    slots = rng.permutation(6 * page)[:T] if scattered else 3 + np.arange(T)
    where = dev(slots.astype(np.int32))
    pools = []
    for rows in (x, bad):
        pools.append(torch.zeros(6, q.qvggt_kv4_page_bytes(page, heads, d), dtype=torch.uint8, device=DEV))
        rows = rows.to(DEV)
        q.qvggt_kv4_append(rows[:, :heads], rows[:, heads:], signs, where, pools[-1], page, rope=table, positions=positions, rope_pair=pair)
    want = pools[0].cpu().numpy().ravel()
    for t, head, which in ((9, 1, 0), (20, 0, 1)):
        kv4.store(want, page, heads, d, int(slots[t]), head, which, np.zeros(d, int), np.float32(np.nan))
    assert np.array_equal(pools[1].cpu().numpy().ravel(), want)
    K, V = (torch.zeros(T, heads, d, device=DEV) for _ in range(2))
    q.qvggt_kv4_read(pools[1], page, signs, where, K, V)
    for out, t, head in ((K, 9, 1), (V, 20, 0)):
        assert bool(out[t, head].isnan().all()) and int(out.isnan().sum()) == d
    # rows that see them: head 1 from token 9 on, head 0 from token 20 on
    if not scattered and value != 3e38:
        table_of_pages = torch.arange(6, device=DEV, dtype=torch.int32)[None]
        starts, lens = dev(np.array([0, T], np.int32)), dev(np.array([T + 3], np.int32))
        queries = torch.randn(T, heads, d, device=DEV)
        out = torch.zeros(T, heads, d, dtype=torch.bfloat16, device=DEV)
        q.qvggt_kv4_attention(queries, signs, 0.1, True, pools[1], page, heads, table_of_pages, starts, lens, T, T + 3, out, None)
        first = torch.full((heads,), T)
        first[1], first[0] = 9, 20
        none = torch.arange(T)[:, None] >= first[None]
        assert torch.equal(out.isnan().all(2).cpu(), none) and torch.equal(out.isnan().any(2).cpu(), none)


@pytest.mark.gpu
@pytest.mark.parametrize("d,heads,kv_heads,q_lens,kv_lens", [(128, 16, 2, [1] * 32, [300] * 32), (64, 8, 2, [4] * 32, [250] * 32), (64, 2, 2, [300], [400]), (128, 2, 1, [256], [300])])
def test_results_are_not_too_small(d, heads, kv_heads, q_lens, kv_lens):
    """Every rounding is to nearest, so errors do not add up to a factor: what results are along the right ones.  512 rows or more of 64 or 128 values, each over hundreds of keys of like
    weight: the rounding to bf16 is 8e-4 of a value rms, 8e-4 sqrt(3 / 32768) = 8e-6 along all of them; a weight's to fp16 1.4e-4, 1.4e-4 / sqrt(50 * 512) = 1e-6.  The bar is five times
    both.  Weights cut off at fp16's last bit would take 2^-12 or more."""
    p = Problem(len(q_lens), d, 16, heads, kv_heads, q_lens, kv_lens, causal=False)
    got, want = p.run().double().cpu().numpy().ravel(), p.want().ravel()
    assert abs((got @ want) / (want @ want) - 1) <= 5e-5


@pytest.mark.gpu
@pytest.mark.parametrize("power", [20, 40, 110])
@pytest.mark.parametrize("name", KERNELS)
def test_values_of_another_size_where_rows_do_not_see_them(name, power):
    """Two values near the end whose steps are 2^power of the others': rows in front of them are as exact as ever (weights of neighbouring rows are scaled each by its own)."""
    p, sizes = problem(name, v_scale=at_the_end(KERNELS[name][5], (1, 3), 2.0 ** power))
    check(p, sizes)


def sharp_bound(turned, keys, values, scale):
    """(the result of one row, how far off each of its channels may be); turned and keys in the turned basis, where products are taken.  A channel of the query is an fp16 number, off by 2^-11
    of itself at most, so score j is off by D_j = 2^-11 times the sum of the magnitudes of its product's terms.  With o the result, weights times e^+-D_j change it by
    sum_j p_j (e^D_j - 1) |v_j - o| over the new sum of weights, which is e^-max D at least.  A weight times its step is an fp16 number too, 2^-11 of it, beside a sum of weights that is
    not: 2^-11 sum_j p_j |v_j|, with the p_j that they are by then.  The result is rounded to 8 bits: 2^-8.  These sums are of the codes, whose basis the result is turned back from: a channel gets
    the 2-norm of such errors at most.  fp32 arithmetic: 2^-20 of the largest terms."""
    score = scale * keys @ turned
    weight = np.exp(score - score.max())
    weight /= weight.sum()
    o = weight @ values
    d = 2.0 ** -11 * scale * np.abs(keys) @ np.abs(turned) + 2.0 ** -20 * np.abs(score)
    moved = np.minimum(weight * np.exp(np.minimum(d + d.max(), 100.0)), 1.0)
    shift = np.minimum(weight * np.expm1(np.minimum(d, 100.0)) * np.exp(min(d.max(), 100.0)), 1.0)
    length = np.linalg.norm(values, axis=1)
    inner = shift @ np.linalg.norm(values - o, axis=1) + 2.0 ** -11 * moved @ length + 2.0 ** -20 * length.max()
    return o, inner + 2.0 ** -8 * (np.abs(o) + inner)


def fp16(x):
    return np.asarray(x, np.float16).astype(np.float64)


@pytest.mark.parametrize("loud", [3.0, 30.0, 300.0])
@pytest.mark.parametrize("d", [64, 128])
def test_the_bound_of_sharp_scores_holds_for_its_roundings(d, loud):
    """The bound against the roundings that it is for, done here (no GPU)."""
    rng = np.random.default_rng(d)
    H = kv4.hadamard(d)
    for _ in range(200):
        n = int(rng.integers(1, 90))
        k, v = (kv4.quantize(rng.standard_normal((n, d)), np.ones(d)) for _ in range(2))
        keys, values = k[0] * k[1][:, None], kv4.held(*v, np.ones(d))
        turned = loud * rng.standard_normal(d)
        o, bound = sharp_bound(turned, keys, values, d ** -0.5)
        up = 2.0 ** (13 - np.floor(np.log2(np.abs(turned).max())))
        score = d ** -0.5 * keys @ fp16(turned * up) / up
        weight = np.exp(score - score.max())
        step = v[1] / v[1].max()
        got = kv4.bf16_rne(fp16(weight * step * 128) @ v[0] @ H * v[1].max() / 128 / weight.sum())
        assert (np.abs(got - o) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("loud", [3.0, 30.0, 300.0])
@pytest.mark.parametrize("name", KERNELS)
def test_every_row_of_sharp_scores(name, loud):
    """Scores of tens to thousands, every row within its own bound."""
    p, sizes = problem(name, loud=loud)
    got = p.run(**sizes).double().cpu().numpy()
    H, group = kv4.hadamard(p.d), p.heads // p.kv_heads
    signs = p.args["signs"].cpu().numpy().astype(float)
    close = 0
    for i, (n, k, v) in enumerate(zip(p.q_lens, p.k, p.v)):
        for j in range(n):
            row, seen = p.starts[i] + j, min(max(len(k) - n + j + 1, 0), len(k))
            for h in range(p.heads if seen else 0):
                o, bound = sharp_bound(p.turned[row, h] * signs @ H, k[:seen, h // group] * signs @ H, v[:seen, h // group], p.scale)
                assert (np.abs(got[row, h] - o) <= bound).all(), (i, j, h)
                close += np.linalg.norm(bound) <= 0.2 * np.linalg.norm(o)
    if loud >= 30:
        assert close >= 0.1 * len(p.x) * p.heads             # the bound says something of a good part of the rows
