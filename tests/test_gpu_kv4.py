"""GPU parity of the 4-bit key/value cache (qvggt_kv4_append / _read / _attention) with oracle/kv4.py, which works in float64.

Bars, from the arithmetic:
  codes       butterflies and scaling in fp32 move z by some 1e-6 of the row's largest value, z / step by some 1e-5: a code falls on the other side of a half with a probability
              of 1e-5, a step on the other side of a bf16 tie with 1e-4.  One code off by one in 10^4, plus two; one step in 10^3, plus one, by a bf16 unit
  attention   rounding the result to bf16 costs 2^-9 of a value at most; weights in fp16, rounded towards zero, 2^-10 of a weight (half of it common to all, the rest 3e-4 rms); queries
              in fp16 2^-12 of a score's terms: below 1e-3 of a weight for scores of a few units.  Together under 3.3e-3 of the 2-norm; the bar is 4e-3
"""
import numpy as np
import pytest
import torch

import paper_2509_21302_amd as q
import synth
from oracle import kv4
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
DEV = G.DEV
BAR = 4e-3


def rel(a, b):
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300))


def bf16(x):
    """numpy -> (device bf16, the values it has as float64)"""
    bits = synth.f32_to_bf16_bits(np.asarray(x, np.float32))
    return G.to_dev(bits), (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def signs_of(rng, d):
    return np.where(rng.random(d) < 0.5, -1, 1).astype(np.int8)


def table_of(rng, rows, dim):
    if not dim:
        return None
    angle = np.arange(rows)[:, None] * rng.uniform(0.003, 1, dim // 2)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


@pytest.mark.parametrize("d,page,heads,T,dim,pair,dtype", [
    (64, 16, 1, 1, 0, 0, "bf16"), (128, 16, 8, 1, 128, 64, "bf16"), (64, 64, 16, 67, 64, 16, "bf16"), (128, 32, 3, 50, 128, 1, "f32"), (128, 1024, 2, 33, 64, 4, "bf16"),
    (64, 16, 5, 130, 32, 2, "f32"), (128, 256, 1, 19, 32, 16, "bf16"), (64, 128, 2, 31, 64, 32, "f32"), (128, 64, 2, 40, 128, 8, "bf16"), (64, 32, 2, 40, 48, 8, "f32"),
    (64, 16, 2, 35, 64, 4, "bf16"), (128, 16, 2, 35, 128, 2, "f32")])
def test_append_and_read(d, page, heads, T, dim, pair, dtype):
    rng = np.random.default_rng(d + T)
    signs, table, positions = signs_of(rng, d), table_of(rng, 50, dim), rng.integers(0, 50, T).astype(np.int32)
    x = rng.standard_normal((T, 3 * heads, d)) * np.where(rng.random(d) < 0.05, 12, 1)
    xd, x = bf16(x) if dtype == "bf16" else (dev(x.astype(np.float32)), x.astype(np.float32).astype(np.float64))
    n_pages = 3 + T // page
    size = q.qvggt_kv4_page_bytes(page, heads, d)
    assert size == heads * page * (d + 4)
    slots = rng.permutation(n_pages * page)[:T].astype(np.int32) if T % 2 else (5 + np.arange(T)).astype(np.int32)
    if T > 30:
        slots[3], slots[7], slots[T - 1] = -1, n_pages * page, 2 ** 31 - 1            # no place in the pool: left out
    stored = (slots >= 0) & (slots < n_pages * page)
    before = rng.integers(0, 256, n_pages * size).astype(np.uint8)
    cache = dev(before).view(n_pages, size)
    q.qvggt_kv4_append(xd[:, heads:2 * heads], xd[:, 2 * heads:], dev(signs), dev(slots), cache, page, rope=dev(table), positions=dev(positions), rope_pair=pair)
    got = cache.cpu().numpy().ravel()
    want = before.copy()
    k, v = kv4.turn(x[:, heads:2 * heads], table, positions, pair), x[:, 2 * heads:]
    sides = [kv4.quantize(y, signs.astype(float)) for y in (k, v)]
    off = steps_off = 0
    held = np.zeros((2, T, heads, d))
    for t in np.nonzero(stored)[0]:
        for h in range(heads):
            for which, (codes, steps) in enumerate(sides):
                c, s = kv4.load(got, page, heads, d, int(slots[t]), h, which)
                held[which, t, h] = kv4.held(c, s, signs)
                assert abs(s - steps[t, h]) <= 2.0 ** -7 * steps[t, h]
                steps_off += s != steps[t, h]
                if s == steps[t, h]:
                    assert np.abs(c - codes[t, h]).max() <= 1
                    off += np.count_nonzero(c != codes[t, h])
                kv4.store(want, page, heads, d, int(slots[t]), h, which, c, s)
    assert off <= 2 + 1e-4 * 2 * T * heads * d and steps_off <= 1 + 2e-3 * T * heads
    assert np.array_equal(got, want)                                                     # nothing else was written
    for out in (torch.bfloat16, torch.float32):
        K, V = (torch.full((T, heads, d), float("nan"), dtype=out, device=DEV) for _ in range(2))
        q.qvggt_kv4_read(cache, page, dev(signs), dev(slots), K, V)
        for t, w in ((K, held[0]), (V, held[1])):
            assert np.abs(t.float().cpu().numpy() - w).max() <= np.abs(w).max() * (2.0 ** -8 if out == torch.bfloat16 else 2e-6)
            assert not t[torch.from_numpy(~stored)].any()
        only = torch.empty_like(V)
        q.qvggt_kv4_read(cache, page, dev(signs), dev(slots), None, only)
        assert torch.equal(only, V)


def test_append_rows_that_are_exact():
    """Rows whose turned values are integers times a power of two, as many as there are kinds: zeros, tiny, huge, one loud channel, a tie of a code."""
    d, page = 64, 16
    rng = np.random.default_rng(3)
    codes = rng.integers(-7, 8, (40, 1, d))
    codes[:, 0, 7] = 7
    z = codes.astype(np.float64)
    z[1, 0, 9] = 2.5                    # ties go to the even code
    z[2, 0, 9] = -3.5
    scale = np.ones(40)
    scale[3:6] = 2.0 ** -100, 2.0 ** 100, 2.0 ** -60
    z[6] = 0.0
    scale[7] = 2.0 ** -130              # a step below the smallest normal number counts as 0
    x = (z * 8) @ (kv4.hadamard(d) * 8) * (scale / 64)[:, None, None]
    xs = x.astype(np.float32)
    assert np.array_equal(xs.astype(np.float64), x)
    cache = torch.zeros(4, q.qvggt_kv4_page_bytes(page, 1, d), dtype=torch.uint8, device=DEV)
    slots = dev(np.arange(40, dtype=np.int32))
    q.qvggt_kv4_append(dev(xs), dev(-xs), None, slots, cache, page)
    got = cache.cpu().numpy().ravel()
    for t in range(40):
        for which in (0, 1):
            c, s = kv4.load(got, page, 1, d, t, 0, which)
            live = t not in (6, 7)
            assert s == (scale[t] if live else 0.0)
            assert np.array_equal(c, (1 - 2 * which) * np.rint(z[t, 0]).astype(int) if live else np.zeros(d, int))


class Problem:
    """Sequences in a pool whose other bytes are no numbers: every query and key of a batch, on both sides."""

    def __init__(self, seed, d, page, heads, kv_heads, q_lens, kv_lens, dim=0, pair=0, causal=True, dtype="bf16", loud=1.0, k_scale=None, v_scale=None, spare=2):
        rng = np.random.default_rng(seed)
        self.d, self.page, self.heads, self.kv_heads, self.causal, self.pair = d, page, heads, kv_heads, causal, pair
        self.q_lens, self.kv_lens, T = list(q_lens), list(kv_lens), sum(q_lens)
        signs = signs_of(rng, d)
        self.width = max(1, max(-(-m // page) for m in kv_lens)) + spare
        n_pages = sum(-(-m // page) for m in kv_lens) + 3
        size = q.qvggt_kv4_page_bytes(page, kv_heads, d)
        pool = np.full(n_pages * size, 255, np.uint8)
        order, used = rng.permutation(n_pages), 0
        table = rng.integers(-2 ** 31, 2 ** 31 - 1, (len(kv_lens), self.width)).astype(np.int32)
        self.k, self.v = [], []
        for i, m in enumerate(kv_lens):
            mine = order[used:used + -(-m // page)]
            used += len(mine)
            table[i, :len(mine)] = mine
            sides = []
            for which, scale in ((0, k_scale), (1, v_scale)):
                codes, steps = kv4.quantize(rng.standard_normal((m, kv_heads, d)), np.ones(d)) if m else (np.zeros((0, kv_heads, d), int), np.zeros((0, kv_heads)))
                if scale is not None and m:
                    steps = kv4.bf16_rne(steps * scale(np.arange(m))[:, None])
                for t in range(m):
                    for h in range(kv_heads):
                        kv4.store(pool, page, kv_heads, d, int(mine[t // page]) * page + t % page, h, which, codes[t, h], steps[t, h])
                sides.append(kv4.held(codes, steps, signs))
            self.k.append(sides[0])
            self.v.append(sides[1])
        x = loud * rng.standard_normal((T, heads + 2, d))
        qd, x = bf16(x) if dtype == "bf16" else (dev(x.astype(np.float32)), x.astype(np.float32).astype(np.float64))
        self.x, self.qd = x[:, :heads], qd[:, :heads]
        rope, positions = table_of(rng, 70, dim), rng.integers(0, 70, T).astype(np.int32)
        self.scale = 1 / np.sqrt(d)
        self.turned = kv4.turn(self.x, rope, positions, pair)
        starts = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        self.starts = starts
        self.args = dict(signs=dev(signs), cache=dev(pool).view(n_pages, size), page_table=dev(table), q_starts=dev(starts), kv_lens=dev(np.array(kv_lens, np.int32)))
        self.more = dict(rope=dev(rope), positions=dev(positions), rope_pair=pair)

    def want(self):
        return np.concatenate([kv4.attention(self.turned[self.starts[i]:self.starts[i + 1]], k, v, self.scale, self.causal) for i, (k, v) in enumerate(zip(self.k, self.v))])

    def run(self, max_q=None, max_kv=None, out=None, workspace=None, stream=None):
        T, a = len(self.x), self.args
        max_q, max_kv = max_q or max(max(self.q_lens), 1), max(self.kv_lens) if max_kv is None else max_kv
        if out is None:
            out = torch.full((T, self.heads, self.d), float("nan"), dtype=torch.bfloat16, device=DEV)
        if workspace is None:
            workspace = torch.full((q.qvggt_kv4_attention_workspace_bytes(T, len(self.q_lens), max_q, max_kv, self.heads, self.kv_heads, self.d),), 255, dtype=torch.uint8, device=DEV)
        q.qvggt_kv4_attention(self.qd, a["signs"], self.scale, self.causal, a["cache"], self.page, self.kv_heads, a["page_table"], a["q_starts"], a["kv_lens"],
                              max_q, max_kv, out, workspace, stream=stream, **self.more)
        return out

    def check(self, bar=BAR, **kw):
        got, want = self.run(**kw).float().cpu().numpy().astype(np.float64), self.want()
        assert np.isfinite(got).all()
        assert rel(got, want) <= bar
        dark = ~want.any(-1)
        assert not got[dark].any()                           # rows that see nothing: exactly zero
        # no row far off on its own: a bf16 unit of its values and the weights' error of its own sum
        assert (np.linalg.norm(got - want, axis=-1) <= 3 * bar * (np.linalg.norm(want, axis=-1) + 0.05)).all()
        return got


@pytest.mark.parametrize("d,page,heads,kv_heads,q_lens,kv_lens,dim,pair,causal", [
    # a token of every sequence, every end of a block, a step and a page
    (128, 16, 8, 2, [1] * 12, [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300], 128, 64, True),
    (64, 64, 4, 4, [1] * 9, [1, 63, 64, 65, 0, 95, 96, 128, 200], 64, 16, True),
    # head groups: own keys, groups of odd size, one key head for all, over 16 rows
    (64, 32, 7, 1, [1, 1, 1], [40, 1, 77], 0, 0, True), (128, 16, 40, 2, [1, 1], [70, 33], 32, 1, True), (128, 32, 64, 1, [1, 1], [50, 129], 128, 64, True),
    # a few tokens at once, rows across all kinds of tile
    (128, 16, 4, 2, [5, 2, 3, 1], [70, 2, 3, 44], 128, 64, True), (64, 16, 3, 1, [8, 7, 0, 8], [8, 60, 5, 0], 64, 32, True), (128, 128, 6, 2, [12, 9], [130, 20], 0, 0, True),
    # queries without keys in front: more queries than keys
    (64, 16, 2, 2, [9, 40], [3, 17], 0, 0, True),
    # prompts: over 64 rows, ragged, earlier keys
    (128, 16, 4, 1, [70, 33, 50], [70, 100, 61], 128, 64, True), (64, 256, 2, 2, [130, 65], [130, 300], 64, 1, True), (128, 64, 3, 3, [200], [200], 64, 8, True),
    # all keys seen, another length
    (64, 32, 4, 4, [20, 100, 3], [75, 13, 0], 0, 0, False), (128, 16, 4, 2, [150], [45], 0, 0, False), (64, 16, 2, 1, [1, 1], [33, 64], 0, 0, False)])
def test_attention(d, page, heads, kv_heads, q_lens, kv_lens, dim, pair, causal):
    Problem(len(q_lens) + d, d, page, heads, kv_heads, q_lens, kv_lens, dim, pair, causal).check()


@pytest.mark.parametrize("d", [64, 128])
def test_attention_split_over_keys(d):
    """One short row over many keys: several blocks of waves, joined; and room for longer sequences than there are."""
    p = Problem(5, d, 16, 4, 1, [1, 2], [2100, 700], d, d // 2)
    a = p.check()
    b = p.check(max_kv=p.width * 16, max_q=5)
    assert rel(a, b) <= BAR
    p = Problem(6, d, 64, 2, 2, [90, 80], [2050, 1100], 0, 0, causal=False)
    p.check()


def test_attention_of_float_queries_and_no_signs():
    p = Problem(7, 128, 16, 4, 2, [3, 20], [40, 55], 128, 64, dtype="f32")
    p.check()
    p = Problem(8, 64, 16, 4, 2, [3, 20], [40, 55], 0, 0, dtype="f32")
    signs = p.args["signs"].cpu().numpy().astype(np.float64)
    p.args["signs"] = None                                   # without signs: what was turned with them is another cache
    p.k, p.v = [k * signs for k in p.k], [v * signs for v in p.v]
    p.check()


def test_attention_of_sharp_scores():
    """Scores of hundreds: a key takes all the weight, nothing overflows."""
    # an fp16 query moves a score of 300 by 300 * 2^-12: 7 % of a weight where two keys are near each other; most rows have one key only
    p = Problem(9, 64, 16, 2, 1, [40], [60], loud=100.0)
    got, want = p.run().float().cpu().numpy(), p.want()
    assert np.isfinite(got).all()
    assert np.quantile(np.linalg.norm(got - want, axis=-1) / np.linalg.norm(want, axis=-1), 0.75) <= 1e-2
    p = Problem(10, 128, 16, 2, 1, [20], [40], loud=1e5)
    got = p.run().float().cpu().numpy()
    assert np.isfinite(got).all()


def test_attention_with_steps_of_all_sizes():
    """Values whose steps grow by 2^30 along a sequence, and fall by it: weights are scaled by the largest so far."""
    for sign in (1, -1):
        p = Problem(11, 64, 16, 2, 1, [30, 1], [400, 410], v_scale=lambda t: 2.0 ** (sign * (t / 14 - 14)))
        p.check()
    p = Problem(12, 128, 16, 4, 2, [2, 1], [90, 40], v_scale=lambda t: np.full(len(t), 2.0 ** -90))
    p.x = p.x  # (same queries)
    got, want = p.run().float().cpu().numpy().astype(np.float64) * 2.0 ** 90, p.want() * 2.0 ** 90
    assert rel(got, want) <= BAR
    # keys without any value: step 0 everywhere
    p = Problem(13, 64, 16, 2, 1, [3], [40], v_scale=lambda t: np.zeros(len(t)))
    assert not p.run().any()
    p = Problem(14, 64, 16, 2, 1, [3], [40], k_scale=lambda t: np.zeros(len(t)))
    p.check()                                                # all scores 0: the mean of the values


def test_attention_reaches_down_to_small_weights():
    """One key with a thousandth of all weight per unit and 60000 that share the rest: each of those weighs 1e-4 of it, together they are six times as much."""
    n = 60000
    p = Problem(15, 64, 1024, 1, 1, [1], [n], k_scale=lambda t: np.where(t == 100, 1.0, 0.0))
    k = p.k[0][100, 0]
    x = (k / (k @ k) * np.log(1e4) * 8)[None, None]          # scale 1/8: that key's score is log 1e4, the others' 0
    p.qd, p.x = bf16(x)
    p.turned = p.x
    p.check()


def test_attention_is_the_same_every_time():
    p = Problem(16, 128, 16, 8, 2, [1] * 6, [500, 30, 1, 0, 999, 65], 128, 64)
    first = p.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(q.qvggt_kv4_attention_workspace_bytes(6, 6, 1, 999, 8, 2, 128), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(first)
    for stream in (None, side):
        out.fill_(7.0)
        side.wait_stream(torch.cuda.current_stream())
        p.run(out=out, workspace=ws, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))
    # a later call of another problem in the same workspace leaves nothing behind
    Problem(17, 128, 16, 8, 2, [1], [700], 128, 64).run(workspace=ws)
    p.run(out=out, workspace=ws)
    assert torch.equal(out.view(torch.int16), first.view(torch.int16))


def test_append_and_attention_in_a_graph():
    """A step of decoding recorded once and replayed with other contents of its buffers, eager work in between."""
    d, page, heads, kv_heads, B = 64, 16, 4, 2, 3
    rng = np.random.default_rng(18)
    signs, table = dev(signs_of(rng, d)), dev(table_of(rng, 300, d))
    size = q.qvggt_kv4_page_bytes(page, kv_heads, d)
    caches = [torch.zeros(B * 8, size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    pages = torch.arange(B * 8, dtype=torch.int32, device=DEV).view(B, 8)
    rows = torch.empty(B, heads + 2 * kv_heads, d, dtype=torch.bfloat16, device=DEV)
    lens, slots, at = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(3))
    starts = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    outs = [torch.empty(B, heads, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ws = torch.empty(max(16, q.qvggt_kv4_attention_workspace_bytes(B, B, 1, 128, heads, kv_heads, d)), dtype=torch.uint8, device=DEV)

    def step(which):
        q.qvggt_kv4_append(rows[:, heads:heads + kv_heads], rows[:, heads + kv_heads:], signs, slots, caches[which], page, rope=table, positions=at, rope_pair=d // 2)
        q.qvggt_kv4_attention(rows[:, :heads], signs, 0.125, True, caches[which], page, kv_heads, pages, starts, lens, 1, 128, outs[which], ws, rope=table, positions=at,
                              rope_pair=d // 2)

    q.qvggt_init()
    step(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for c in caches:
        c.zero_()
    for i in range(40):
        n = torch.tensor([i, i // 2, min(3 * i, 120)], dtype=torch.int32)
        rows.copy_(torch.from_numpy(rng.standard_normal(rows.shape)).to(torch.bfloat16))
        lens.copy_(n + 1)
        at.copy_(n)
        slots.copy_(pages.cpu()[torch.arange(B), n // page] * page + n % page)
        step(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0], caches[1]) and outs[0].any(), i


def test_offsets_past_32_bits():
    """Pages in the first and last part of a pool of more than 2^32 bytes."""
    d, page, heads = 128, 64, 2
    size = q.qvggt_kv4_page_bytes(page, heads, d)
    n_pages = (2 ** 32 + 2 ** 29) // size
    cache = torch.empty(n_pages, size, dtype=torch.uint8, device=DEV)
    p = Problem(19, d, page, 4, heads, [3], [4 * page - 5], d, d // 2)
    mine = p.args["page_table"].cpu().numpy()[0, :4]
    places = np.array([0, n_pages - 1, n_pages // 2, n_pages - 7], np.int32)
    assert size * (n_pages - 7) > 2 ** 32
    for a, b in zip(mine, places):
        cache[int(b)] = p.args["cache"][int(a)]
    p.args["cache"], table = cache, p.args["page_table"].clone()
    table[0, :4] = dev(places)
    p.args["page_table"] = table
    p.check()
    slots = (places * page + 3).astype(np.int64)
    assert slots.max() < 2 ** 31
    x = torch.randn(4, 2 * heads, d, device=DEV).to(torch.bfloat16)
    q.qvggt_kv4_append(x[:, :heads], x[:, heads:], None, dev(slots.astype(np.int32)), cache, page)
    K, V = (torch.empty(4, heads, d, dtype=torch.float32, device=DEV) for _ in range(2))
    q.qvggt_kv4_read(cache, page, None, dev(slots.astype(np.int32)), K, V)
    for got, from_ in ((K, x[:, :heads]), (V, x[:, heads:])):
        err = (got - from_.float()).norm() / from_.float().norm()
        assert 0.02 < err < 0.2                              # 4 bits of a normal row: a step is about 0.4 of its deviation
    del cache


def test_refusals_leave_the_outputs_alone():
    p = Problem(20, 64, 16, 2, 1, [2], [20])
    out = torch.full((2, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(q.QvggtError) as e:
        p.run(out=out, max_kv=16 * p.width + 1)
    assert e.value.status == 2
    p2 = Problem(21, 64, 16, 2, 1, [2], [5000])
    with pytest.raises(q.QvggtError) as e:
        p2.run(out=out, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    assert e.value.status == 5
    with pytest.raises(ValueError):
        p.run(out=out.float())
    good = p.args["kv_lens"]
    p.args["kv_lens"] = good.long()
    with pytest.raises(ValueError):
        p.run(out=out)
    p.args["kv_lens"] = good
    with pytest.raises(ValueError):
        q.qvggt_kv4_append(out.transpose(0, 1), out, None, good, p.args["cache"], 16)
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("d,kv_heads,group,causal", [(64, 2, 1, False), (128, 1, 3, True)])
def test_attention_of_sequences_in_any_order_of_their_lengths(d, kv_heads, group, causal):
    """More sequences than a wave has lanes, lengths that rise, fall, repeat and are zero: every sequence gets its own rows, and those alone."""
    rng = np.random.default_rng(d)
    kv_lens = [0, 0, 40, 40, 40] + list(range(1, 31)) + list(range(90, 60, -1)) + [int(n) for n in rng.integers(0, 60, 5)]
    q_lens = [72 // group] + [int(n) for n in rng.integers(0, 4, len(kv_lens) - 1)]
    assert len(kv_lens) == 70
    Problem(d, d, 16, kv_heads * group, kv_heads, q_lens, kv_lens, causal=causal).check()
