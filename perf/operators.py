"""The operators of a 4-bit key/value cache: the calls a user makes of them, over the range of sizes they are made with, and their plain forms.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a user's program holds before the call
    run(state)          one pass: the framework's entry points where `own` is true, elementary float32 torch operations where it is not
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   what run() returns, from the definitions in 64 bits

Kinds of case:

    append      keys and values of new tokens are rotated by position, turned by a Hadamard matrix, rounded to 4 bits and stored in pages
                (`qvggt_kv4_append`); what the pages then hold is read back (`qvggt_kv4_read`)
    attend      attention of new queries over the pages (`qvggt_kv4_attention`): single tokens, a few tokens, prompts, and queries that
                see the whole of another sequence's states

Definitions, for a key or value x of a head (d channels), signs s, the orthonormal Sylvester-Hadamard matrix H of d channels:

    rotation    pairs (c, c + pair) inside consecutive groups of 2 * pair of the first rope_dim channels, pair number p of the row
                `positions[t]` of the table: (a, b) -> (a cos_p - b sin_p, b cos_p + a sin_p).  Keys and queries only
    cache       z = (s * x) H,  step = bf16(max |z| / 7),  code = clamp(rne(z / step), -8, 7);  what it stands for is s * (step * code) H
    attention   softmax over the visible keys of scale * <q, k>, times the values, with the keys and values that the cache stands for.  Query i of a
                sequence's n sees keys 0 .. len - n + i where it is causal, all `len` of them otherwise; one that sees none gives zeros

A page holds `page` tokens of every head; a head's part is page * (d + 4) bytes: the keys' codes (token after token, d / 2 bytes: channel
2 j in the low half of byte j, 2 j + 1 in the high half), the values' codes (blocks of 16 tokens, in each [4 groups of 4 tokens][16][d / 32][4 tokens]
bytes, channel pair p at [p / (d / 32)][p % (d / 32)]), the steps (a pair of bf16 per token, key's and value's).  Codes are kept as code + 8.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
FRAME = 1374            # tokens of a frame: 37 x 37 patches and 5 special tokens
MOST_PAIRS = 12289 * 12289 * 32 * 128      # query tokens x keys x heads x channels of the largest listed case
MOST_CACHE = 48 * 16384 * 16 * 64          # values of keys that a drawn case keeps in its pages, padded to its longest sequence


def listed():
    return [
        # one token of one sequence: the smallest call there is, once a layer for every token that a single user is answered with
        dict(name="append_one", kind="append", tokens=1, padding=0, heads=8, d=128, page=16, dtype="bf16", rope_dim=128, pair=64),
        # a token of each of 256 sequences, the last slots of the batch empty
        dict(name="append_batch", kind="append", tokens=256, padding=9, heads=8, d=128, page=16, dtype="bf16", rope_dim=128, pair=64),
        # one frame of a 1024-wide backbone, its rotation by row and column
        dict(name="append_frame", kind="append", tokens=FRAME, padding=0, heads=16, d=64, page=64, dtype="bf16", rope_dim=64, pair=16),
        # prompts in float32, neighbouring channels rotated together, half of them
        dict(name="append_prompts_f32", kind="append", tokens=16411, padding=0, heads=8, d=128, page=16, dtype="f32", rope_dim=64, pair=1),
        # a single user early in an answer: latency
        dict(name="decode_short", kind="attend", seqs=1, max_q=1, max_kv=777, heads=32, kv_heads=8, d=128, page=16, causal=True, rope_dim=128, pair=64, empty=0),
        # a single user with a long document
        dict(name="decode_long", kind="attend", seqs=1, max_q=1, max_kv=131071, heads=32, kv_heads=8, d=128, page=16, causal=True, rope_dim=128, pair=64, empty=0),
        # a serving batch of sequences of many lengths
        dict(name="decode_batch", kind="attend", seqs=64, max_q=1, max_kv=8192, heads=32, kv_heads=8, d=128, page=16, causal=True, rope_dim=128, pair=64, empty=2),
        # every head with keys of its own, 64 channels
        dict(name="decode_own_heads", kind="attend", seqs=48, max_q=1, max_kv=16384, heads=16, kv_heads=16, d=64, page=64, causal=True, rope_dim=64, pair=32, empty=0),
        # prompts of several users that continue what their pages hold
        dict(name="prompts_ragged", kind="attend", seqs=6, max_q=1801, max_kv=5003, heads=32, kv_heads=8, d=128, page=16, causal=True, rope_dim=128, pair=64, empty=0),
        # a new frame that looks at itself and 49 earlier ones
        dict(name="frame_over_50", kind="attend", seqs=1, max_q=FRAME, max_kv=50 * FRAME, heads=16, kv_heads=16, d=64, page=64, causal=False, rope_dim=64, pair=16, empty=0),
        # one long prompt
        dict(name="prompt_long", kind="attend", seqs=1, max_q=12289, max_kv=12289, heads=32, kv_heads=8, d=128, page=64, causal=True, rope_dim=128, pair=64, empty=0),
        # queries that see an encoder's states of another length; one sequence has none
        dict(name="cross", kind="attend", seqs=12, max_q=448, max_kv=1500, heads=20, kv_heads=20, d=64, page=32, causal=False, rope_dim=0, pair=0, empty=1),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _rotation(rng, d):
    dim = rng.choice((d, d, d, d // 2, 0))
    return dict(rope_dim=dim, pair=rng.choice((1, dim // 4, dim // 2, dim // 2)) if dim else 0)


def draw(rng):
    d, page = rng.choice((64, 128)), rng.choice((16, 16, 32, 64, 256))
    if rng.random() < 0.3:
        tokens = _spread(rng, 1, 16411)
        return dict(kind="append", tokens=tokens, padding=rng.choice((0, 0, tokens // 16)), heads=rng.choice((1, 2, 4, 8, 16)), d=d, page=page,
                    dtype=rng.choice(("bf16", "bf16", "f32")), **_rotation(rng, d))
    shape = rng.choice(("one", "one", "few", "prompt", "prompt", "cross"))
    group, kv_heads = rng.choice((1, 2, 4, 7, 8, 16)), rng.choice((1, 2, 4, 8, 8, 16))
    kv_heads = min(kv_heads, 64 // group)
    if shape in ("one", "few"):
        seqs, max_q = _spread(rng, 1, 128), 1 if shape == "one" else _spread(rng, 2, 16)
        max_kv = _spread(rng, max_q, max(max_q, min(131071, MOST_CACHE // (seqs * kv_heads * d))))
    else:
        seqs, max_q = _spread(rng, 1, 16), _spread(rng, 17, 8191)
        most = min(65535, MOST_PAIRS // (seqs * group * kv_heads * d * max_q), MOST_CACHE // (seqs * kv_heads * d))
        if most < 64:
            seqs, max_q = 1, min(max_q, 2047)
            most = min(65535, MOST_PAIRS // (group * kv_heads * d * max_q))
        max_kv = _spread(rng, min(max_q, most) if shape == "prompt" else 16, most)
    return dict(kind="attend", seqs=seqs, max_q=max_q, max_kv=max_kv, heads=group * kv_heads, kv_heads=kv_heads, d=d, page=page, causal=shape != "cross",
                empty=rng.choice((0, 0, 1)) if seqs > 2 else 0, **(_rotation(rng, d) if shape != "cross" else dict(rope_dim=0, pair=0)))


# ---------------------------------------------------------------------------------------------------------------- inputs
def _lengths(c):
    """(queries, keys) of every sequence: the longest first, the others anywhere below, `empty` ones without keys at the end."""
    rng = random.Random(c["seqs"] * 7919 + c["max_q"] * 31 + c["max_kv"])
    q, kv = [], []
    for i in range(c["seqs"]):
        n = c["max_q"] if i == 0 else rng.randint((c["max_q"] + 1) // 2, c["max_q"])
        m = 0 if i >= c["seqs"] - c["empty"] else c["max_kv"] if i == 0 else rng.randint(1, c["max_kv"])
        q.append(n)
        kv.append(max(m, n) if c["causal"] and m and c["max_kv"] >= n else m)
    return q, kv


def _table(c, rows):
    """Cosines and sines [rows, rope_dim]: by position, or for a frame's patches by row and column in one half of the channels each."""
    n = c["rope_dim"] // 2
    if not n:
        return None
    at = torch.arange(rows, device=DEV, dtype=torch.float64)
    if c["pair"] == c["rope_dim"] // 4 and c["pair"] > 1:
        turn = 100.0 ** (-torch.arange(n // 2, device=DEV, dtype=torch.float64) / (n // 2))
        angle = torch.cat([(at // 37)[:, None] * turn, (at % 37)[:, None] * turn], 1)
    else:
        angle = at[:, None] * 10000.0 ** (-torch.arange(n, device=DEV, dtype=torch.float64) / n)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _signs(d, gen):
    return (torch.randint(0, 2, (d,), device=DEV, generator=gen) * 2 - 1).to(torch.int8)


def prepare(c, seed):
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    d, page = c["d"], c["page"]
    randn = lambda *s: torch.randn(*s, device=DEV, generator=gen)  # noqa: E731
    s = dict(c, signs=_signs(d, gen))
    if c["kind"] == "append":
        T, h = c["tokens"], c["heads"]
        # keys have a few channels that are large in every token; keys and values lie behind queries in the rows of one fused product
        loud = 1 + 9 * (torch.rand(h, d, device=DEV, generator=gen) < 0.04)
        fused = randn(T, 3 * h, d)
        fused[:, h:2 * h] *= loud
        fused = fused.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        rows = 1 + max(T, 2048)
        n_pages = 2 + 2 * -(-T // page)
        # runs of tokens that follow one another in pages that do not; page 0 is nobody's
        order = 1 + torch.randperm(n_pages - 1, device=DEV, generator=gen)
        first = int(torch.randint(0, page, (1,), generator=torch.Generator().manual_seed(seed)))
        at = first + torch.arange(T, device=DEV)
        slots = order[at // page] * page + at % page
        slots[T - c["padding"]:] = -1
        s.update(k=fused[:, h:2 * h], v=fused[:, 2 * h:], rope=_table(c, rows), slots=slots.int(), positions=((at * 5) % rows).int(),
                 cache=torch.randint(0, 256, (n_pages, h * page * (d + 4)), dtype=torch.uint8, device=DEV, generator=gen))
        s.update(k_out=torch.empty(T, h, d, dtype=torch.bfloat16, device=DEV), v_out=torch.empty(T, h, d, dtype=torch.bfloat16, device=DEV))
        return s
    h = c["kv_heads"]
    q_lens, kv_lens = _lengths(c)
    T, width = sum(q_lens), -(-c["max_kv"] // page)
    n_pages = 1 + sum(-(-n // page) for n in kv_lens)
    starts = [0]
    for n in q_lens:
        starts.append(starts[-1] + n)
    # the pages: rounded normal keys and values; what lies behind a sequence's end, and page 0, is whatever was there (all ones: no number)
    cache = torch.full((n_pages, h, page * (d + 4)), 255, dtype=torch.uint8, device=DEV)
    order = 1 + torch.randperm(n_pages - 1, device=DEV, generator=gen).int()
    table = torch.full((c["seqs"], width), -1, dtype=torch.int32, device=DEV)
    used = 0
    for i, n in enumerate(kv_lens):
        m = -(-n // page)
        mine = order[used:used + m]
        table[i, :m] = mine
        used += m
        for lo in range(0, m, max(1, (1 << 26) // (h * page * d))):       # some millions of values at a time
            some = mine[lo:lo + max(1, (1 << 26) // (h * page * d))].long()
            part = torch.empty(len(some), h, page * (d + 4), dtype=torch.uint8, device=DEV)
            views = _views(part, page, d)
            steps = torch.empty(len(some), h, page, 2, dtype=torch.bfloat16, device=DEV)
            for which in (0, 1):
                z = randn(len(some), h, page, d)
                step = (z.abs().amax(-1) / 7).to(torch.bfloat16)
                u = ((z / step.float()[..., None]).round_().clamp_(-8, 7) + 8).to(torch.uint8)
                b = u[..., 0::2] | u[..., 1::2] << 4
                if which == 0:
                    views[0].copy_(b)
                else:
                    views[1].copy_(b.view(len(some), h, page // 16, 4, 4, 16, d // 32).permute(0, 1, 2, 3, 5, 6, 4))
                steps[..., which] = step
            left = n - lo * page                                         # tokens of the sequence from here on
            dead = (torch.arange(len(some) * page, device=DEV) >= left).view(len(some), 1, page, 1)
            steps = torch.where(dead, torch.full((), float("nan"), dtype=torch.bfloat16, device=DEV), steps)
            views[2].copy_(steps)
            cache[some] = part
    # queries: a third again as long as the keys, so that some keys count more than others
    q = (1.4 * randn(T, c["heads"] + 2 * h, d)).to(torch.bfloat16)[:, :c["heads"]]
    rows = max(1 + max(c["max_kv"], c["max_q"]), FRAME)
    begin = torch.tensor(starts[:-1], device=DEV).repeat_interleave(torch.tensor(q_lens, device=DEV))
    ahead = torch.tensor([max(0, m - n) for n, m in zip(q_lens, kv_lens)], device=DEV).repeat_interleave(torch.tensor(q_lens, device=DEV))
    positions = torch.arange(T, device=DEV) - begin + ahead
    s.update(q=q, rope=_table(c, rows), positions=positions.int(), scale=1 / math.sqrt(d), cache=cache.view(n_pages, -1), table=table,
             starts=torch.tensor(starts, dtype=torch.int32, device=DEV), lens=torch.tensor(kv_lens, dtype=torch.int32, device=DEV), T=T,
             out=torch.empty(T, c["heads"], d, dtype=torch.bfloat16, device=DEV))
    return s


def work(c):
    d, page = c["d"], c["page"]
    if c["kind"] == "append":
        T, h, size = c["tokens"], c["heads"], 2 if c["dtype"] == "bf16" else 4
        # keys and values in, pages out; pages in, keys and values out; the rotation's table rows, positions, slots
        moved = T * h * (2 * d * size + d + 4) + T * h * (d + 4 + 2 * d * 2) + T * (4 * c["rope_dim"] + 12)
        return {"bytes": moved, "flops": T * h * (4 * d * int(math.log2(d)) + 3 * c["rope_dim"] + 8 * d)}
    q_lens, kv_lens = _lengths(c)
    T = sum(q_lens)
    pairs = 0
    for n, m in zip(q_lens, kv_lens):
        pairs += sum(max(0, m - n + i + 1) for i in range(n)) if c["causal"] else n * m
    moved = 2 * T * c["heads"] * d * 2 + sum(kv_lens) * c["kv_heads"] * (d + 4) + T * (4 * c["rope_dim"] + 4)
    return {"bytes": moved, "flops": 4 * pairs * c["heads"] * d + 1}


# ---------------------------------------------------------------------------------------------------------------- the plain form
def _views(cache, page, d):
    """Keys' bytes [n, heads, page, d / 2], values' bytes [n, heads, page / 16, 4, 16, d / 32, 4], steps [n, heads, page, 2] of pages [n, heads, bytes]."""
    k = cache[:, :, :page * d // 2].unflatten(2, (page, d // 2))
    v = cache[:, :, page * d // 2:page * d].unflatten(2, (page // 16, 4, 16, d // 32, 4))
    return k, v, cache[:, :, page * d:].view(torch.bfloat16).unflatten(2, (page, 2))


def _hadamard(d):
    i = torch.arange(d, device=DEV)
    x = i[:, None] & i[None, :]
    x = x ^ x >> 4
    x = x ^ x >> 2
    x = (x ^ x >> 1) & 1
    return (1 - 2 * x).float() / math.sqrt(d)


def _turn(x, s):
    """The rotation by position of x [T, heads, d]."""
    if s["rope"] is None:
        return x
    dim, pair = s["rope_dim"], s["pair"]
    cos, sin = s["rope"][s["positions"].long()].view(-1, 1, 2, dim // (2 * pair), pair).unbind(2)
    a, b = x[..., :dim].unflatten(2, (dim // (2 * pair), 2, pair)).unbind(3)
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2), x[..., dim:]], 2)


def _bytes_of(x, s):
    """(codes in bytes [T, heads, d / 2], steps [T, heads]) of x [T, heads, d]."""
    z = (x * s["signs"].float()) @ _hadamard(s["d"])
    step = (z.abs().amax(-1) / 7).to(torch.bfloat16)
    u = torch.where(step[..., None] > 0, (z / step.float()[..., None]).round().clamp(-8, 7), 0.0).to(torch.int16) + 8
    return (u[..., 0::2] | u[..., 1::2] << 4).to(torch.uint8), step


def _values(b, step):
    """step * code of bytes [..., d / 2] and steps [...]."""
    u = torch.stack([b & 15, b >> 4], -1).flatten(-2)
    return (u.float() - 8) * step.float()[..., None]


def _plain_append(s):
    d, page, h = s["d"], s["page"], s["heads"]
    k, v, steps = _views(s["cache"].view(-1, h, page * (d + 4)), page, d)
    stored = (s["slots"] >= 0)[:, None, None]
    slot = s["slots"].long().clamp(min=0)                      # page 0 is nobody's
    n, t = slot // page, slot % page
    kb, ks = _bytes_of(_turn(s["k"].float(), s), s)
    vb, vs = _bytes_of(s["v"].float(), s)
    k[n, :, t] = kb
    v[n, :, t // 16, t % 16 // 4, :, :, t % 4] = vb.unflatten(2, (16, d // 32))
    steps[n, :, t] = torch.stack([ks, vs], -1)
    back = lambda b, step: torch.where(stored, _values(b, step) @ _hadamard(d) * s["signs"].float(), 0.0).to(torch.bfloat16)  # noqa: E731
    return {"k": back(k[n, :, t], steps[n, :, t, 0]), "v": back(v[n, :, t // 16, t % 16 // 4, :, :, t % 4].flatten(2), steps[n, :, t, 1])}


def _plain_attend(s):
    d, page, h, g, B = s["d"], s["page"], s["kv_heads"], s["heads"] // s["kv_heads"], s["seqs"]
    pages = s["cache"].view(-1, h, page * (d + 4))[s["table"].long().clamp(min=0)].flatten(0, 1)
    k, v, steps = _views(pages, page, d)
    L = s["table"].shape[1] * page
    at = torch.arange(L, device=DEV)
    there = at < s["lens"][:, None]                                                          # [B, L]
    by_head = lambda x: x.unflatten(0, (B, -1)).transpose(1, 2).flatten(2, 3)  # noqa: E731    [B, h, L, ...]
    steps = torch.where(there[:, None, :, None], by_head(steps).float(), 0.0)
    k = _values(by_head(k), steps[..., 0])
    v = _values(by_head(v.permute(0, 1, 2, 3, 6, 4, 5).flatten(2, 4).flatten(3)), steps[..., 1])
    # queries by sequence [B, h, n g, d], padded to the longest
    n = s["max_q"]
    row = s["starts"][:-1, None].long() + torch.arange(n, device=DEV)
    count = s["starts"].diff()
    q = (_turn(s["q"].float(), s) * s["signs"].float() @ _hadamard(d))[row.clamp(max=s["T"] - 1)]
    q = q.unflatten(2, (h, g)).permute(0, 2, 1, 3, 4).flatten(2, 3) * s["scale"]
    x = q @ k.transpose(2, 3).contiguous()                                                   # [B, h, n g, L]
    seen = there[:, None, :].expand(B, n, L)
    if s["causal"]:
        seen = seen & (at <= (s["lens"] - count)[:, None, None] + torch.arange(n, device=DEV)[:, None])
    x = x.unflatten(2, (n, g)).masked_fill_(~seen[:, None, :, None, :], -math.inf).flatten(2, 3)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    o = x @ v / torch.where(total > 0, total, 1.0)
    o = (o @ _hadamard(d) * s["signs"].float()).unflatten(2, (n, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    # back to rows [T, heads, d]
    which = torch.repeat_interleave(torch.arange(B, device=DEV), count, output_size=s["T"])
    return o[which, torch.arange(s["T"], device=DEV) - s["starts"].long()[which]].to(torch.bfloat16)


def run(s):
    if not own:
        return _plain_append(s) if s["kind"] == "append" else _plain_attend(s)
    import paper_2509_21302_amd as q
    if s["kind"] == "append":
        q.qvggt_kv4_append(s["k"], s["v"], s["signs"], s["slots"], s["cache"], s["page"], rope=s["rope"], positions=s["positions"], rope_pair=s["pair"])
        q.qvggt_kv4_read(s["cache"], s["page"], s["signs"], s["slots"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if "workspace" not in s:         # a program allocates it once for its sizes
        need = q.qvggt_kv4_attention_workspace_bytes(s["T"], s["seqs"], s["max_q"], s["max_kv"], s["heads"], s["kv_heads"], s["d"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    q.qvggt_kv4_attention(s["q"], s["signs"], s["scale"], s["causal"], s["cache"], s["page"], s["kv_heads"], s["table"], s["starts"], s["lens"],
                          s["max_q"], s["max_kv"], s["out"], s["workspace"], rope=s["rope"], positions=s["positions"], rope_pair=s["pair"])
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------- 64 bits
def _sylvester(d):
    H = torch.ones(1, 1, dtype=torch.float64, device=DEV)
    while len(H) < d:
        H = torch.cat([torch.cat([H, H], 1), torch.cat([H, -H], 1)], 0)
    return H / math.sqrt(d)


def _turned64(x, s):
    """The rotation as a complex product, pair after pair of channels."""
    x = x.double().clone()
    if s["rope"] is None:
        return x
    dim, pair = s["rope_dim"], s["pair"]
    row = s["rope"].double()[s["positions"].long()]
    for first in range(0, dim, 2 * pair):
        p = slice(first // 2, first // 2 + pair)
        z = torch.complex(x[..., first:first + pair], x[..., first + pair:first + 2 * pair])
        z = z * torch.complex(row[:, p], row[:, dim // 2:][:, p])[:, None]
        x[..., first:first + pair], x[..., first + pair:first + 2 * pair] = z.real, z.imag
    return x


def _cached64(c, s, i, n, head, keys):
    """Keys or values [n, d] of a sequence's head, byte by byte where the layout has them."""
    d, page = c["d"], c["page"]
    t = torch.arange(n, device=DEV)
    base = (s["table"][i].long()[t // page] * c["kv_heads"] + head) * page * (d + 4)
    o, j = t % page, torch.arange(d, device=DEV)
    flat, p, R = s["cache"].view(-1), j // 2, d // 32
    if keys:
        at = (o * (d // 2))[:, None] + p
    else:
        at = page * d // 2 + (o // 16 * 8 * d)[:, None] + ((o % 16 // 4 * 16)[:, None] + p // R) * R * 4 + p % R * 4 + (o % 4)[:, None]
    u = flat[base[:, None] + at] >> (j % 2 * 4).to(torch.uint8) & 15
    word = base + page * d + 4 * o + (0 if keys else 2)
    step = (flat[word + 1].int() << 24 | flat[word].int() << 16).view(torch.float32).double()
    return (u.double() - 8) * step[:, None]


def exact(c, seed):
    s = prepare(c, seed)
    d = c["d"]
    H, sign = _sylvester(d), s["signs"].double()
    if c["kind"] == "append":
        def held(x):
            z = (x.double() * sign) @ H
            step = (z.abs().amax(-1, keepdim=True) / 7).to(torch.bfloat16).double()
            x = torch.round(z / step).clamp(-8, 7) * step
            return torch.where((s["slots"] >= 0)[:, None, None], (x @ H) * sign, 0.0)
        return {"k": held(_turned64(s["k"], s)), "v": held(s["v"])}
    q_lens, kv_lens = _lengths(c)
    q = (_turned64(s["q"], s) * sign) @ H
    out = torch.zeros(s["T"], c["heads"], d, dtype=torch.float64, device=DEV)
    g, row = c["heads"] // c["kv_heads"], 0
    for i, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for head in range(c["kv_heads"] if m else 0):
            k, v = _cached64(c, s, i, m, head, True), _cached64(c, s, i, m, head, False)
            for lo in range(0, n, 4096):
                mine = q[row + lo:row + min(n, lo + 4096), head * g:(head + 1) * g]
                x = s["scale"] * (mine.reshape(-1, d) @ k.T).view(len(mine), g, m)
                if c["causal"]:
                    at = m - n + lo + torch.arange(len(mine), device=DEV)
                    x = x.masked_fill((torch.arange(m, device=DEV) > at[:, None])[:, None], -math.inf)
                p = torch.nan_to_num(torch.softmax(x, -1))
                out[row + lo:row + lo + len(mine), head * g:(head + 1) * g] = (p.view(-1, m) @ v @ H * sign).view(len(mine), g, d)
        row += n
    return out
