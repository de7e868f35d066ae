"""GPU parity of qvggt_heads_norm_rope and qvggt_residual_norm with oracle/block.py (float64), value by value within the bound that the oracle derives."""
import math

import pytest
import torch

import paper_2509_21302_amd as q
from oracle import block as O
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
DEV = G.DEV
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def near(got, want, off):
    worst = ((got.double() - want).abs() / off).max() if got.numel() else torch.zeros(())
    assert float(worst) <= 1.0, float(worst)


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def table_of(rows, dim, g):
    angle = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * torch.rand(dim // 2, device=DEV, generator=g, dtype=torch.float64)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


@pytest.mark.parametrize("T,heads,kv_heads,d,dtype,kind,axes,dim,pair,lanes", [
    (1, 32, 8, 128, "bf16", "rms", 1, 128, 64, None), (1, 1, 1, 64, "f32", "layer", 1, 64, 32, None), (77, 16, 16, 64, "bf16", "layer", 2, 64, 16, None),
    (5, 3, 1, 128, "f32", "rms", 3, 128, 64, "turns"), (33, 20, 5, 64, "bf16", "none", 2, 64, 8, "any"), (9, 17, 16, 128, "bf16", "layer", 4, 128, 32, "any"),
    (4, 7, 7, 64, "f32", "rms", 3, 48, 8, None), (130, 1, 9, 128, "bf16", "none", 1, 64, 1, None), (6, 40, 2, 128, "f32", "layer", 2, 128, 2, "turns"),
    (7, 33, 33, 64, "bf16", "rms", 3, 32, 4, "any"), (3, 140, 20, 64, "bf16", "rms", 1, 0, 0, None), (12, 2, 2, 128, "bf16", "layer", 2, 96, 16, None), (8, 5, 4, 128, "f32", "none", 4, 16, 8, None)])
@pytest.mark.parametrize("gains", [True, False])
def test_heads(T, heads, kv_heads, d, dtype, kind, axes, dim, pair, lanes, gains):
    g = gen(T + d + heads)
    fused = (torch.randn(T, heads + 2 * kv_heads, d, device=DEV, generator=g) * 3 + 1).to(TYPES[dtype])
    Q, K = fused[:, :heads], fused[:, heads:heads + kv_heads]
    vec = [1 + 0.3 * torch.randn(d, device=DEV, generator=g) if gains else None for _ in range(4)]
    rope = table_of(60, dim, g) if dim else None
    positions = torch.randint(-3, 64, (axes, T), device=DEV, generator=g).int()               # outside of the table too
    pair_axis = None if lanes is None else (torch.arange(dim // 2, device=DEV) % axes if lanes == "turns" else torch.randint(0, axes + 2, (dim // 2,), device=DEV, generator=g)).to(torch.uint8)
    before = fused.clone()
    outs = [torch.full((T, n + 1, d), 7.0, dtype=fused.dtype, device=DEV) for n in (heads, kv_heads)]
    call = lambda a, b: q.qvggt_heads_norm_rope(Q, K, a, b, norm=kind, eps=1e-5, q_gain=vec[0], q_bias=vec[1], k_gain=vec[2], k_bias=vec[3], rope=rope,  # noqa: E731
                                                positions=positions if axes > 1 or T % 2 else positions[0], rope_pair=pair, pair_axis=pair_axis)
    call(outs[0][:, 1:], outs[1][:, :-1])
    assert torch.equal(fused, before) and bool((outs[0][:, 0] == 7).all()) and bool((outs[1][:, -1] == 7).all())
    for x, y, gain, bias in ((Q, outs[0][:, 1:], vec[0], vec[1]), (K, outs[1][:, :-1], vec[2], vec[3])):
        near(y, *O.heads_norm_rope(x, kind, 1e-5, gain, bias, rope, positions, pair, pair_axis))
    call(Q, K)                                                                                # in place
    assert torch.equal(Q, outs[0][:, 1:]) and torch.equal(K, outs[1][:, :-1]) and torch.equal(fused[:, heads + kv_heads:], before[:, heads + kv_heads:])


def test_heads_of_one_kind_and_of_none():
    g = gen(3)
    x = torch.randn(50, 6, 64, device=DEV, generator=g).to(torch.bfloat16)
    y, z = torch.empty_like(x), torch.empty_like(x)
    q.qvggt_heads_norm_rope(x, None, y, None, norm="rms")
    q.qvggt_heads_norm_rope(None, x, None, z, norm="rms")
    assert torch.equal(y, z)
    near(y, *O.heads_norm_rope(x, "rms", 1e-6, None, None, None, None, 0))
    q.qvggt_heads_norm_rope(x[:0], x[:0], y[:0], z[:0], norm="rms")


def test_heads_match_the_rotation_of_the_cache():
    """The same table, positions and pairs as qvggt_kv4_append takes: one axis, no norm, against the oracle's rotation of the cache."""
    from oracle import kv4
    g = gen(4)
    for d, dim, pair in ((64, 64, 16), (128, 64, 1), (128, 128, 64)):
        x, rope = torch.randn(40, 3, d, device=DEV, generator=g), table_of(50, dim, g)
        at = torch.randint(0, 50, (40,), device=DEV, generator=g).int()
        y = torch.empty_like(x)
        q.qvggt_heads_norm_rope(x, None, y, None, rope=rope, positions=at, rope_pair=pair)
        want = torch.from_numpy(kv4.turn(x.cpu().numpy(), rope.cpu().numpy(), at.cpu().numpy(), pair))
        assert float((y.cpu().double() - want).abs().max()) <= 4 * O.U * 2 * float(x.abs().max())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_head_that_is_no_number_stays_alone(bad):
    g = gen(5)
    for d in (64, 128):
        x = torch.randn(9, 20, d, device=DEV, generator=g).to(torch.bfloat16)
        rope, at = table_of(50, d, g), torch.arange(9, device=DEV).int()
        a, b = torch.empty_like(x), torch.empty_like(x)
        q.qvggt_heads_norm_rope(x, None, a, None, norm="layer", rope=rope, positions=at, rope_pair=d // 2)
        x[4, 11, 3] = bad
        q.qvggt_heads_norm_rope(x, None, b, None, norm="layer", rope=rope, positions=at, rope_pair=d // 2)
        hit = torch.zeros(9, 20, dtype=torch.bool, device=DEV)
        hit[4, 11] = True
        assert torch.equal(a[~hit], b[~hit]) and bool(torch.isnan(b[4, 11].float()).all())


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_heads_of_tiny_and_large_values(kind):
    """Variances from 2^-120 (below what the instruction for the root takes) to 2^100."""
    g = gen(6)
    x = torch.randn(60, 4, 64, device=DEV, generator=g) * 2.0 ** torch.linspace(-60, 50, 60, device=DEV)[:, None, None]
    y = torch.empty_like(x)
    q.qvggt_heads_norm_rope(x, None, y, None, norm=kind, eps=0.0)
    near(y, *O.heads_norm_rope(x, kind, 0.0, None, None, None, None, 0))
    same = torch.full((2, 1, 64), 0.75, device=DEV)                    # no variance: the bias
    y = torch.empty_like(same)
    q.qvggt_heads_norm_rope(same, None, y, None, norm="layer", eps=1e-6, q_bias=torch.arange(64, device=DEV).float())
    assert torch.equal(y, torch.arange(64, device=DEV).float().expand(2, 1, 64))


def case(M, C, x, y, h, seed, rows, cond="bf16"):
    g = gen(seed)
    randn = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    vec = lambda: randn(C) * 0.3 + 1  # noqa: E731
    parts = (0.5 * randn(max(rows, 1), 3 * C)).to(TYPES[cond])
    return dict(x=(2 * randn(M, C) + 0.5).to(TYPES[x]), y=randn(M, C).to(TYPES[y]), post_gain=vec(), post_bias=vec(), scale=vec(), gain=vec(), bias=vec(), gate=parts[:, :C],
                mod_scale=parts[:, C:2 * C], mod_shift=parts[:, 2 * C:], row_of=torch.randint(-1, rows + 1, (M,), device=DEV, generator=g).int() if rows > 1 else None, h_dtype=TYPES[h])


FULL = ("post_gain", "post_bias", "scale", "gain", "bias", "gate", "mod_scale", "mod_shift")


def update(c, post, kind, use, eps=1e-6, x_out=None, h=None):
    args = {n: c[n] if n in use else None for n in FULL}
    row_of = c["row_of"] if any(n in use for n in ("gate", "mod_scale", "mod_shift")) else None
    x_out = torch.full_like(c["x"], 7.0) if x_out is None else x_out
    h = torch.full(c["x"].shape, 7.0, dtype=c["h_dtype"], device=DEV) if h is None else h
    x, y = c["x"].clone(), None if c["y"] is None else c["y"].clone()
    q.qvggt_residual_norm(c["x"], c["y"], x_out, h, post_norm=post, norm=kind, row_of=row_of, eps=eps, **args)
    want = O.residual_norm(x, y, x.dtype, h.dtype, post, args["post_gain"], args["post_bias"], args["scale"], args["gate"], kind, args["gain"], args["bias"], args["mod_scale"],
                           args["mod_shift"], row_of, eps)
    near(x_out, *want[0])
    near(h, *want[1])
    return x_out, h


@pytest.mark.parametrize("M,C,x,y,h,post,kind,rows,use", [
    (1, 2048, "bf16", "bf16", "bf16", "none", "layer", 1, ("scale", "gain", "bias")), (37, 1024, "bf16", "bf16", "bf16", "none", "layer", 1, ("scale", "gain", "bias")),
    (19, 2560, "f32", "bf16", "bf16", "rms", "rms", 5, FULL), (3, 8, "f32", "f32", "f32", "layer", "layer", 1, FULL), (5, 8192, "bf16", "f32", "f32", "layer", "rms", 3, FULL),
    (67, 64, "bf16", "bf16", "bf16", "rms", "layer", 7, FULL), (130, 136, "f32", "bf16", "f32", "none", "rms", 1, ("gate", "gain")), (33, 256, "bf16", "bf16", "f32", "none", "none", 2, ("gate",)),
    (9, 264, "f32", "f32", "bf16", "layer", "none", 1, ("post_gain", "bias")), (11, 520, "bf16", "f32", "bf16", "none", "rms", 1, ()), (6, 1032, "f32", "bf16", "f32", "rms", "layer", 6, FULL),
    (7, 4096, "bf16", "bf16", "bf16", "none", "layer", 1, ("scale", "gain", "bias")), (4, 5128, "f32", "f32", "f32", "rms", "rms", 1, ("mod_scale", "mod_shift")),
    (1000, 120, "bf16", "bf16", "bf16", "none", "rms", 1, ("gain",)), (2, 2056, "bf16", "bf16", "f32", "layer", "layer", 2, FULL)])
def test_residual(M, C, x, y, h, post, kind, rows, use):
    c = case(M, C, x, y, h, M + C, rows, "f32" if M % 2 else "bf16")
    x_out, h_out = update(c, post, kind, use)
    # in place, of the same types
    keep = {n: None if t is None else t.clone() for n, t in c.items() if n in ("x", "y")}
    other = update(c, post, kind, use, x_out=c["x"], h=c["y"] if c["y"].dtype == c["h_dtype"] else None)
    assert torch.equal(other[0], x_out) and torch.equal(other[1], h_out)
    c.update(keep)
    # one output at a time
    row_of = c["row_of"] if any(n in use for n in ("gate", "mod_scale", "mod_shift")) else None
    args = dict({n: c[n] if n in use else None for n in FULL}, post_norm=post, norm=kind, row_of=row_of)
    a, b = torch.empty_like(x_out), torch.empty_like(h_out)
    q.qvggt_residual_norm(c["x"], c["y"], a, None, **args)
    q.qvggt_residual_norm(c["x"], c["y"], None, b, **args)
    assert torch.equal(a, x_out) and torch.equal(b, h_out)


def test_residual_without_an_update_is_a_norm():
    c = case(40, 768, "bf16", "bf16", "bf16", 2, 1)
    c["y"] = None
    x_out, _ = update(c, "rms", "layer", ("gain", "bias", "gate", "scale"))
    assert torch.equal(x_out, c["x"])


def test_residual_rows_of_their_own_condition():
    c = case(30, 512, "bf16", "bf16", "f32", 3, 30)
    c["row_of"] = None
    update(c, "none", "layer", ("gate", "mod_scale", "mod_shift"))


@pytest.mark.parametrize("C", [128, 1000, 4104])
def test_residual_no_numbers_stay_in_their_row(C):
    c = case(20, C, "bf16", "bf16", "bf16", 4, 1)
    outs = []
    for bad in (None, math.nan, math.inf):
        if bad is not None:
            c["y"][7, C - 1] = bad
        x_out, h = torch.empty_like(c["x"]), torch.empty_like(c["x"])
        q.qvggt_residual_norm(c["x"], c["y"], x_out, h, post_norm="rms", norm="layer")
        outs.append((x_out, h))
    rows = torch.arange(20, device=DEV) != 7
    for x_out, h in outs[1:]:
        assert torch.equal(x_out[rows], outs[0][0][rows]) and torch.equal(h[rows], outs[0][1][rows]) and bool(torch.isnan(h[7].float()).all())


def test_residual_means_far_from_zero():
    """A stream whose mean is 1000 times its deviation: two passes over the row keep the variance."""
    g = gen(8)
    x, y = 1000 + torch.randn(50, 1536, device=DEV, generator=g), torch.randn(50, 1536, device=DEV, generator=g)
    c = dict(x=x, y=y, row_of=None, h_dtype=torch.float32, **{n: None for n in FULL})
    update(c, "none", "layer", ())


def test_residual_offsets_past_32_bits():
    M, C = 524300, 4096
    x = torch.zeros(M, C, dtype=torch.bfloat16, device=DEV)
    y, h = torch.zeros_like(x), torch.zeros_like(x)
    g = gen(9)
    x[-20:], y[-20:] = torch.randn(20, C, device=DEV, generator=g).to(torch.bfloat16), torch.randn(20, C, device=DEV, generator=g).to(torch.bfloat16)
    want = O.residual_norm(x[-20:], y[-20:], torch.bfloat16, torch.bfloat16, kind="layer")
    q.qvggt_residual_norm(x, y, x, h, norm="layer")
    near(x[-20:], *want[0])
    near(h[-20:], *want[1])
    assert not bool(h[:-20].any())


def test_heads_past_2_to_the_31():
    T, heads, d = 262144, 68, 128
    x = torch.zeros(T, heads, d, dtype=torch.bfloat16, device=DEV)
    g = gen(10)
    x[-3:] = torch.randn(3, heads, d, device=DEV, generator=g).to(torch.bfloat16)
    rope, at = table_of(64, d, g), (torch.arange(2 * T, device=DEV) % 64).int().view(2, T)
    want = O.heads_norm_rope(x[-3:], "rms", 1e-6, None, None, rope, at[:, -3:], 64)
    q.qvggt_heads_norm_rope(x, None, x, None, norm="rms", rope=rope, positions=at, rope_pair=64)
    near(x[-3:], *want)
    assert not bool(x[:-3].any())


@pytest.mark.parametrize("seed", range(16))
def test_random_rows(seed):
    import random
    rng = random.Random(seed)
    C, M, rows = 8 * rng.choice((1, 3, 16, 17, 31, 33, 63, 65, 100, 127, 129, 200, 257, 500, 511, 513, 777, 1023)), rng.choice((1, 2, 3, 17, 64, 300)), rng.choice((1, 2, 9))
    c = case(M, C, *(rng.choice(("bf16", "f32")) for _ in range(3)), seed, rows, rng.choice(("bf16", "f32")))
    update(c, rng.choice(("none", "rms", "layer")), rng.choice(("none", "rms", "layer")), [n for n in FULL if rng.random() < 0.6], rng.choice((1e-6, 1e-3)))


def test_residual_rows_of_several_launches():
    M, C = (1 << 26) + 37, 8
    x, y = torch.zeros(M, C, dtype=torch.bfloat16, device=DEV), torch.zeros(M, C, dtype=torch.bfloat16, device=DEV)
    g = gen(11)
    at = slice((1 << 26) - 20, M)
    x[at], y[at] = (torch.randn(57, C, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    want = O.residual_norm(x[at], y[at], torch.bfloat16, torch.bfloat16, kind="rms")
    h = torch.full_like(x, 7.0)
    q.qvggt_residual_norm(x, y, x, h, norm="rms")
    near(x[at], *want[0])
    near(h[at], *want[1])
    assert not bool(h[:(1 << 26) - 20].any())
