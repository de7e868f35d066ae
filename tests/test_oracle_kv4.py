"""The oracle of the 4-bit key/value cache against closed forms and its own inverse (no GPU)."""
import numpy as np
import pytest

from oracle import kv4


@pytest.mark.parametrize("d", [64, 128])
def test_hadamard_is_orthonormal_and_symmetric(d):
    H = kv4.hadamard(d)
    assert np.allclose(H @ H, np.eye(d), atol=1e-14) and np.array_equal(H, H.T)
    assert H[3, 5] == H[0, 0] * (-1) ** bin(3 & 5).count("1")


@pytest.mark.parametrize("dim,pair", [(64, 32), (64, 16), (64, 1), (32, 16), (16, 2)])
def test_turn_keeps_lengths_and_relative_positions(dim, pair):
    rng = np.random.default_rng(dim + pair)
    x, y = rng.standard_normal((2, 1, 1, 64))
    angle = np.arange(40)[:, None] * rng.uniform(0.01, 1, dim // 2)
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    at = lambda v, p: kv4.turn(v, table, np.array([p]), pair)  # noqa: E731
    assert np.allclose(np.linalg.norm(at(x, 7)), np.linalg.norm(x))
    assert np.allclose((at(x, 9) * at(y, 4)).sum(), (at(x, 25) * at(y, 20)).sum())       # the product depends on the difference of the positions
    assert np.array_equal(at(x, 7)[..., dim:], x[..., dim:]) and np.allclose(at(x, 0), x)
    # a pair by hand: channels 0 and `pair`, angle 0 of row 7
    c, s = table[7, 0], table[7, dim // 2]
    assert np.isclose(at(x, 7)[0, 0, 0], x[0, 0, 0] * c - x[0, 0, pair] * s) and np.isclose(at(x, 7)[0, 0, pair], x[0, 0, pair] * c + x[0, 0, 0] * s)


def test_quantizer_rows():
    signs = np.where(np.arange(64) % 3 == 0, -1, 1)
    codes = np.random.default_rng(0).integers(-7, 8, 64)
    codes[5] = 7
    codes2, step = kv4.quantize(kv4.held(codes, np.float64(0.5), signs), signs)          # what a row of codes stands for has these codes
    assert np.array_equal(codes, codes2) and step == 0.5
    codes0, step0 = kv4.quantize(np.zeros(64), signs)
    assert step0 == 0 and not codes0.any()
    # the error of a value is half a step at most where the rounded step is not below the row's own
    x = np.random.default_rng(1).standard_normal((50, 128))
    s = np.ones(128)
    c, st = kv4.quantize(x, s)
    assert np.abs(x @ kv4.hadamard(128) - c * st[:, None]).max() <= 0.52 * st.max() and np.abs(c).max() == 7


@pytest.mark.parametrize("d,page,heads", [(64, 16, 3), (128, 32, 2)])
def test_every_code_has_a_place_of_its_own(d, page, heads):
    places = [kv4.byte_of(page, d, t, c, v) * 2 + c % 2 for t in range(page) for c in range(d) for v in (0, 1)]
    assert sorted(places) == list(range(2 * page * d))                                   # keys and values fill a part's first page * d bytes
    pool = np.random.default_rng(0).integers(0, 256, 3 * heads * page * (d + 4)).astype(np.uint8)
    before = pool.copy()
    codes = np.random.default_rng(1).integers(-8, 8, d)
    for which in (0, 1):
        kv4.store(pool, page, heads, d, page + 5, 1, which, codes, 0.75)
        got, step = kv4.load(pool, page, heads, d, page + 5, 1, which)
        assert np.array_equal(got, codes) and step == 0.75
    assert np.count_nonzero(pool != before) <= d + 4


def test_attention_rows():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 4, 64)), rng.standard_normal((2, 2, 64)), rng.standard_normal((2, 2, 64))
    out = kv4.attention(q, k, v, 0.1, True)
    assert not out[0].any()                                                              # three queries on two keys: the first sees none
    assert np.allclose(out[1], np.repeat(v[0], 2, 0))                                    # the second sees one
    w = np.exp(0.1 * q[2, 3] @ k[:, 1].T)
    assert np.allclose(out[2, 3], w @ v[:, 1] / w.sum()) and np.allclose(kv4.attention(q, k, v, 0.1, False)[2], out[2])
    assert not kv4.attention(q, k[:0], v[:0], 0.1, False).any()
