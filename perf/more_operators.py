"""The operators around a block's quantized layers: the calls a user makes of them, over the range of sizes they are made with, and their plain forms.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a user's program holds before the call
    run(state)          one pass: the framework's entry points where `own` is true, elementary float32 torch operations where it is not
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   what run() returns, from the definitions in 64 bits

Kinds of case:

    heads       heads of queries and keys, as they lie in the rows of a fused product, are normalised and rotated by positions with several axes
                (`qvggt_heads_norm_rope`)
    attend      attention of packed sequences over bf16 keys and values (`qvggt_attention`): single tokens and chunks over the buffers that hold their
                sequences, whole prompts, frames
    residual    what a block's output does to the residual stream, and the norm in front of the next block (`qvggt_residual_norm`)

Definitions:

    norm        layer: (x - mean) / sqrt(variance + eps), rms: x / sqrt(mean of squares + eps), none: x; then times a gain and plus a bias where they are given
    rotation    pairs (c, c + pair) inside consecutive groups of 2 * pair of the first rope_dim channels; pair number p turns by the row positions[axis_p, t] of the
                table: (a, b) -> (a cos_p - b sin_p, b cos_p + a sin_p), with axis_p = pair_axis[p], or p * axes // pairs where there is no such list
    heads       rotation(norm(x)) of every head, queries and keys with gains and biases of their own
    attention   softmax over the visible keys of scale * <q, k>, times the values.  Query i of a sequence's n sees keys 0 .. len - n + i where it is causal, all `len` of them
                otherwise; one that sees none gives zeros
    residual    x' = x + scale * gate[r] * norm_post(y),    h = norm_pre(x') * (1 + mod_scale[r]) + mod_shift[r],    r the token's row of the condition;
                what is not given is left out.  h is of x' before it is rounded
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
FRAME = 1374            # tokens of a frame: 37 x 37 patches and 5 special tokens
MOST_PAIRS = 10 * FRAME * 10 * FRAME * 16 * 64        # query tokens x keys x heads x channels of the case with the most scores
MOST_KEYS = 48 * 8192 * 8 * 128                       # values of the keys of a drawn case, padded to its longest sequence
MOST_VALUES = 100 * FRAME * 1024                      # values of a drawn residual stream


def listed():
    return [
        # one token of one sequence, before its keys go into a cache: the smallest call there is
        dict(name="heads_one", kind="heads", tokens=1, heads=32, kv_heads=8, d=128, dtype="bf16", norm="rms", gains=True, axes=1, rope_dim=128, pair=64, lanes="", apart=True),
        # ten frames of a 1024-wide backbone, rotated by row and column of their patches, special tokens at position 0
        dict(name="heads_frames", kind="heads", tokens=10 * FRAME, heads=16, kv_heads=16, d=64, dtype="bf16", norm="layer", gains=True, axes=2, rope_dim=64, pair=16, lanes="", apart=True),
        # a video's tokens with positions in time, height and width, whose pairs take turns
        dict(name="heads_video_f32", kind="heads", tokens=16411, heads=32, kv_heads=8, d=128, dtype="f32", norm="rms", gains=True, axes=3, rope_dim=128, pair=64, lanes="turns", apart=True),
        # a single user early in an answer: latency
        dict(name="attend_one", kind="attend", form="buffer", seqs=1, max_q=1, max_kv=601, heads=32, kv_heads=8, d=128, causal=True, empty=0),
        # a serving batch of sequences of many lengths, a token each
        dict(name="attend_tokens", kind="attend", form="buffer", seqs=48, max_q=1, max_kv=8192, heads=32, kv_heads=8, d=128, causal=True, empty=1),
        # chunks of new tokens over what the sequences hold already
        dict(name="attend_chunks", kind="attend", form="buffer", seqs=8, max_q=61, max_kv=16384, heads=32, kv_heads=8, d=128, causal=True, empty=0),
        # prompts of several users, behind one another
        dict(name="attend_prompts", kind="attend", form="packed", seqs=7, max_q=3001, max_kv=3001, heads=32, kv_heads=8, d=128, causal=True, empty=0),
        # one long prompt
        dict(name="attend_prompt_long", kind="attend", form="packed", seqs=1, max_q=11003, max_kv=11003, heads=32, kv_heads=8, d=128, causal=True, empty=0),
        # all tokens of ten frames look at one another
        dict(name="attend_global", kind="attend", form="packed", seqs=1, max_q=10 * FRAME, max_kv=10 * FRAME, heads=16, kv_heads=16, d=64, causal=False, empty=0),
        # a camera token's row through a block: latency
        dict(name="residual_one", kind="residual", tokens=1, width=2048, x="bf16", y="bf16", h="bf16", post="none", scale=True, pre="layer", gains=True, gate=False, mod=False, rows=0),
        # a hundred frames: the output of a block scaled into the residual stream, the next one's norm
        dict(name="residual_frames", kind="residual", tokens=100 * FRAME, width=1024, x="bf16", y="bf16", h="bf16", post="none", scale=True, pre="layer", gains=True, gate=False, mod=False, rows=0),
        # norms on both sides of a block, gate, scale and shift of every sequence's condition, a float32 residual stream
        dict(name="residual_gated", kind="residual", tokens=8191, width=2560, x="f32", y="bf16", h="bf16", post="rms", scale=False, pre="rms", gains=True, gate=True, mod=True, rows=11),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_heads(rng):
    d, kv_heads = rng.choice((64, 128)), rng.choice((1, 2, 4, 8, 16, 20))
    heads = kv_heads * rng.choice((1, 1, 2, 4, 7))
    dim, axes = rng.choice((d, d, d // 2, 0)), rng.choice((1, 2, 3))
    pair = rng.choice((1, dim // 4, dim // 2)) if dim else 0
    return dict(kind="heads", tokens=_spread(rng, 1, min(16411, 16411 * 40 * 128 // (d * (heads + kv_heads)))), heads=heads, kv_heads=kv_heads, d=d, dtype=rng.choice(("bf16", "bf16", "f32")),
                norm=rng.choice(("layer", "rms", "rms", "none") if dim else ("layer", "rms")), gains=rng.random() < 0.8, axes=axes, rope_dim=dim, pair=pair,
                lanes=rng.choice(("", "turns", "sections")), apart=rng.random() < 0.7)


def _draw_residual(rng):
    width = 8 * _spread(rng, 8, 1024) if rng.random() < 0.5 else rng.choice((768, 1024, 1280, 2048, 4096, 5120, 8192))
    gate, mod, post = rng.random() < 0.4, rng.random() < 0.4, rng.choice(("none", "none", "rms", "layer"))
    types = [rng.choice(("bf16", "bf16", "f32")) for _ in range(3)]
    tokens = _spread(rng, 1, MOST_VALUES // width * 2 // sum(1 + (t == "f32") for t in types))
    return dict(kind="residual", tokens=tokens, width=width, x=types[0], y=types[1], h=types[2], post=post, scale=rng.random() < 0.6, pre=rng.choice(("layer", "layer", "rms", "none")),
                gains=rng.random() < 0.8, gate=gate, mod=mod, rows=rng.choice((1, min(tokens, 5), min(tokens, 64))) if gate or mod else 0)


def _draw_attend(rng):
    d, shape = rng.choice((64, 128)), rng.choice(("tokens", "tokens", "chunks", "prompts", "prompts", "cross"))
    group, kv_heads = rng.choice((1, 2, 4, 7, 8, 16)), rng.choice((1, 2, 4, 8, 8, 16))
    kv_heads = min(kv_heads, 64 // group)
    each = kv_heads * d
    if shape in ("tokens", "chunks"):
        seqs = _spread(rng, 1, 96)
        max_q = 1 if shape == "tokens" else _spread(rng, 2, 128)
        most = min(131071, MOST_KEYS // (seqs * each), MOST_PAIRS // (seqs * group * each * max_q))
        max_kv = _spread(rng, min(max_q, most), most)
        form, causal = "buffer", True
    elif shape == "prompts":
        seqs = _spread(rng, 1, 24)
        max_q = max_kv = _spread(rng, 17, max(17, min(10 * FRAME, int(math.sqrt(MOST_PAIRS / (seqs * group * each))))))
        form, causal = "packed", rng.random() < 0.7
    else:
        seqs = _spread(rng, 1, 24)
        max_q = _spread(rng, 17, 2047)
        max_kv = _spread(rng, 16, max(17, min(32767, MOST_PAIRS // (seqs * group * each * max_q), MOST_KEYS // (seqs * each))))
        form, causal = "apart", rng.random() < 0.3
    return dict(kind="attend", form=form, seqs=seqs, max_q=max_q, max_kv=max_kv, heads=group * kv_heads, kv_heads=kv_heads, d=d, causal=causal,
                empty=rng.choice((0, 0, 1)) if seqs > 2 and form != "packed" else 0)


def draw(rng):
    return rng.choice((_draw_heads, _draw_residual, _draw_attend, _draw_attend))(rng)


# ---------------------------------------------------------------------------------------------------------------- inputs
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _lengths(c):
    """(queries, keys) of every sequence: the longest first, the others anywhere below, `empty` ones without keys at the end."""
    rng = random.Random(c["seqs"] * 7919 + c["max_q"] * 31 + c["max_kv"])
    q, kv = [], []
    for i in range(c["seqs"]):
        n = c["max_q"] if i == 0 else rng.randint((c["max_q"] + 1) // 2, c["max_q"])
        m = 0 if i >= c["seqs"] - c["empty"] else c["max_kv"] if i == 0 else rng.randint(1, c["max_kv"])
        q.append(n)
        kv.append(n if c["form"] == "packed" else max(m, n) if m and c["form"] == "buffer" and c["max_kv"] >= n else m)
    return q, kv


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _table(c, rows):
    """Cosines and sines [rows, rope_dim] by position."""
    n = c["rope_dim"] // 2
    if not n:
        return None
    base, turns = (100.0, n // c["axes"]) if c["axes"] == 2 else (10000.0, n)
    at = torch.arange(rows, device=DEV, dtype=torch.float64)
    angle = at[:, None] * base ** (-(torch.arange(n, device=DEV, dtype=torch.float64) % turns) / turns)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _positions(c):
    """int32 [axes, tokens], and the rows of the table."""
    t = torch.arange(c["tokens"], device=DEV)
    if c["axes"] == 1:
        rows = max(c["tokens"], 4096)
        return ((t * 5) % rows)[None].int(), rows
    place = (t % FRAME - 5).clamp(min=-1)                            # a frame's special tokens stand at row and column 0, its patches from 1 on
    high, wide = torch.where(place < 0, 0, place // 37 + 1), torch.where(place < 0, 0, place % 37 + 1)
    return torch.stack([high, wide] if c["axes"] == 2 else [t // FRAME, high, wide]).int(), max(64, c["tokens"] // FRAME + 1)


def _axes(c):
    """The axis of every pair: None for equal sections, axes that take turns, or sections of unequal lengths, the last axis's first."""
    n, axes = c["rope_dim"] // 2, c["axes"]
    if not n or not c["lanes"]:
        return None
    p = torch.arange(n, device=DEV)
    return (p % axes if c["lanes"] == "turns" else ((p + n // 8) * axes // (n + n // 8)).flip(0)).to(torch.uint8)


def prepare(c, seed):
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device=DEV, generator=gen)  # noqa: E731
    s = dict(c)
    if c["kind"] == "heads":
        T, h, m, d, t = c["tokens"], c["heads"], c["kv_heads"], c["d"], TYPES[c["dtype"]]
        # a few channels are large in every token
        fused = randn(T, h + 2 * m, d)
        fused *= 1 + 9 * (torch.rand(h + 2 * m, d, device=DEV, generator=gen) < 0.04)
        fused = fused.to(t)
        positions, rows = _positions(c)
        s.update(q=fused[:, :h], k=fused[:, h:h + m], positions=positions, rope=_table(c, rows), pair_axis=_axes(c), eps=1e-6)
        for name in ("q", "k"):
            s[name + "_gain"] = 1 + 0.2 * randn(d) if c["gains"] else None
            s[name + "_bias"] = 0.1 * randn(d) if c["gains"] and c["norm"] == "layer" else None
        if c["apart"]:
            s.update(q_out=torch.empty(T, h, d, dtype=t, device=DEV), k_out=torch.empty(T, m, d, dtype=t, device=DEV))
        else:                               # rows of a fused buffer as well
            both = torch.zeros(T, h + m, d, dtype=t, device=DEV)
            s.update(q_out=both[:, :h], k_out=both[:, h:])
        return s
    if c["kind"] == "residual":
        T, w = c["tokens"], c["width"]
        s.update(x=(3 * randn(T, w) + 0.5).to(TYPES[c["x"]]), y=randn(T, w).to(TYPES[c["y"]]), eps=1e-6, x_out=torch.empty(T, w, dtype=TYPES[c["x"]], device=DEV),
                 h_out=torch.empty(T, w, dtype=TYPES[c["h"]], device=DEV))
        s["channel_scale"] = 0.3 * randn(w) if c["scale"] else None
        for name in ("post", "pre"):
            s[name + "_gain"] = 1 + 0.2 * randn(w) if c["gains"] and c[name] != "none" else None
            s[name + "_bias"] = 0.1 * randn(w) if c["gains"] and c[name] == "layer" else None
        # gate, scale and shift are parts of the rows of one product
        parts = (0.5 * randn(max(1, c["rows"]), 3 * w)).to(torch.bfloat16)
        s["gate_rows"] = parts[:, :w] if c["gate"] else None
        s["mod_scale"], s["mod_shift"] = (parts[:, w:2 * w], parts[:, 2 * w:]) if c["mod"] else (None, None)
        s["row_of"] = (torch.arange(T, device=DEV) * c["rows"] // T).int() if c["rows"] > 1 else None
        return s
    h, m, d = c["heads"], c["kv_heads"], c["d"]
    q_lens, kv_lens = _lengths(c)
    T, starts = sum(q_lens), _starts(q_lens)
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    s.update(T=T, starts=whole(starts), scale=1 / math.sqrt(d), lens=None, out=torch.zeros(T, h, d, dtype=torch.bfloat16, device=DEV))
    # queries half as long again as the keys, so that some keys count more than others
    if c["form"] == "packed":
        fused = randn(T, h + 2 * m, d)
        fused[:, :h] *= 1.5
        fused = fused.to(torch.bfloat16)
        s.update(q=fused[:, :h], k=fused[:, h:h + m], v=fused[:, h + m:], kv_starts=s["starts"])
        return s
    s["q"] = (1.5 * randn(T, h + 2 * m, d)).to(torch.bfloat16)[:, :h]
    if c["form"] == "apart":
        S, s["kv_starts"] = sum(kv_lens), whole(_starts(kv_lens))
    else:                                   # a buffer of every sequence's longest length; what lies behind its end is whatever was there
        capacity = c["max_kv"] + 3
        S, s["kv_starts"], s["lens"] = c["seqs"] * capacity, whole([i * capacity for i in range(c["seqs"])]), whole(kv_lens)
    for name in ("k", "v"):
        s[name] = torch.empty(max(1, S), m, d, dtype=torch.bfloat16, device=DEV)
        for lo in range(0, S, 1 << 16):
            s[name][lo:lo + (1 << 16)] = randn(min(S - lo, 1 << 16), m, d).to(torch.bfloat16)
        if s["lens"] is not None:
            at = torch.arange(S, device=DEV)
            s[name][at % capacity >= s["lens"].long()[at // capacity]] = math.nan
    return s


def work(c):
    size = {"bf16": 2, "f32": 4}
    if c["kind"] == "heads":
        values = c["tokens"] * (c["heads"] + c["kv_heads"]) * c["d"]
        rows = _positions_count(c)
        return {"bytes": 2 * values * size[c["dtype"]] + c["tokens"] * 4 * c["axes"] + rows * 4 * c["rope_dim"] + 1, "flops": values * 10}
    if c["kind"] == "residual":
        values = c["tokens"] * c["width"]
        return {"bytes": values * (2 * size[c["x"]] + size[c["y"]] + size[c["h"]]) + c["width"] * (4 * 5 + 6 * c["rows"]), "flops": values * 20}
    d = c["d"]
    q_lens, kv_lens = _lengths(c)
    pairs, keys = 0, 0
    for n, m in zip(q_lens, kv_lens):
        pairs += sum(max(0, m - n + i + 1) for i in range(n)) if c["causal"] else n * m
        keys += m
    return {"bytes": 2 * sum(q_lens) * c["heads"] * d * 2 + 2 * keys * c["kv_heads"] * d * 2 + 8 * c["seqs"], "flops": 4 * pairs * c["heads"] * d + 1}


def _positions_count(c):
    """Rows of the table that a case's positions name."""
    if not c["rope_dim"]:
        return 0
    return c["tokens"] if c["axes"] == 1 else min(c["tokens"], 38 if c["axes"] == 2 else max(38, c["tokens"] // FRAME + 1))


# ---------------------------------------------------------------------------------------------------------------- the plain form
def _norm(x, kind, eps, gain, bias):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    if kind != "none":
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if gain is not None:
        x = x * gain
    return x if bias is None else x + bias


def _turn(x, s):
    """The rotation of x [T, heads, d] by the positions of its tokens."""
    if s["rope"] is None:
        return x
    dim, pair = s["rope_dim"], s["pair"]
    n = dim // 2
    p = torch.arange(n, device=DEV)
    axis = p * s["axes"] // n if s["pair_axis"] is None else s["pair_axis"].long()
    row = s["positions"].long()[axis].T                                                     # [T, pairs]
    cos, sin = (s["rope"][row, p + at].view(-1, 1, n // pair, pair) for at in (0, n))
    a, b = x[..., :dim].unflatten(2, (n // pair, 2, pair)).unbind(3)
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2), x[..., dim:]], 2)


def _plain_heads(s):
    t = TYPES[s["dtype"]]
    return {n: _turn(_norm(s[n].float(), s["norm"], s["eps"], s[n + "_gain"], s[n + "_bias"]), s).to(t) for n in ("q", "k")}


def _plain_residual(s):
    u = _norm(s["y"].float(), s["post"], s["eps"], s["post_gain"], s["post_bias"])
    if s["channel_scale"] is not None:
        u = u * s["channel_scale"]
    of = lambda rows: rows.float() if s["row_of"] is None else rows.float()[s["row_of"].long()]  # noqa: E731
    if s["gate_rows"] is not None:
        u = u * of(s["gate_rows"])
    x = s["x"].float() + u
    h = _norm(x, s["pre"], s["eps"], s["pre_gain"], s["pre_bias"])
    if s["mod"]:
        h = h * (1 + of(s["mod_scale"])) + of(s["mod_shift"])
    return {"x": x.to(s["x_out"].dtype), "h": h.to(s["h_out"].dtype)}


def _plain_attend(s):
    h, g, d, B = s["kv_heads"], s["heads"] // s["kv_heads"], s["d"], s["seqs"]
    n, L = s["max_q"], s["max_kv"]
    count, lens = s["starts"].diff(), s["lens"] if s["lens"] is not None else s["kv_starts"].diff()
    at = torch.arange(L, device=DEV)
    there = at < lens[:, None]                                                               # [B, L]
    rows = torch.where(there, s["kv_starts"][:B, None].long() + at, 0)
    # keys and values by sequence and head [B, h, L, d], zeros behind a sequence's end
    k, v = (torch.where(there[:, None, :, None], s[name][rows].transpose(1, 2).float(), 0.0) for name in ("k", "v"))
    # queries by sequence [B, h, n g, d], padded to the longest
    row = s["starts"][:-1, None].long() + torch.arange(n, device=DEV)
    q = s["q"][row.clamp(max=s["T"] - 1)].float().unflatten(2, (h, g)).permute(0, 2, 1, 3, 4).flatten(2, 3) * s["scale"]
    x = q @ k.transpose(2, 3).contiguous()                                                   # [B, h, n g, L]
    seen = there[:, None, :].expand(B, n, L)
    if s["causal"]:
        seen = seen & (at <= (lens - count)[:, None, None] + torch.arange(n, device=DEV)[:, None])
    x = x.unflatten(2, (n, g)).masked_fill_(~seen[:, None, :, None, :], -math.inf).flatten(2, 3)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ v / torch.where(total > 0, total, 1.0)).unflatten(2, (n, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    # back to rows [T, heads, d]
    which = torch.repeat_interleave(torch.arange(B, device=DEV), count, output_size=s["T"])
    return o[which, torch.arange(s["T"], device=DEV) - s["starts"].long()[which]].to(torch.bfloat16)


def run(s):
    if not own:
        return {"heads": _plain_heads, "residual": _plain_residual, "attend": _plain_attend}[s["kind"]](s)
    import paper_2509_21302_amd as q
    if s["kind"] == "heads":
        q.qvggt_heads_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], norm=s["norm"], eps=s["eps"], q_gain=s["q_gain"], q_bias=s["q_bias"], k_gain=s["k_gain"], k_bias=s["k_bias"],
                                rope=s["rope"], positions=s["positions"], rope_pair=s["pair"], pair_axis=s["pair_axis"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if s["kind"] == "residual":
        q.qvggt_residual_norm(s["x"], s["y"], s["x_out"], s["h_out"], post_norm=s["post"], post_gain=s["post_gain"], post_bias=s["post_bias"], scale=s["channel_scale"], gate=s["gate_rows"],
                              norm=s["pre"], gain=s["pre_gain"], bias=s["pre_bias"], mod_scale=s["mod_scale"], mod_shift=s["mod_shift"], row_of=s["row_of"], eps=s["eps"])
        return {"x": s["x_out"], "h": s["h_out"]}
    if "workspace" not in s:         # a program allocates it once for its sizes
        need = q.qvggt_attention_workspace_bytes(s["T"], s["seqs"], s["max_q"], s["max_kv"], s["heads"], s["kv_heads"], s["d"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    q.qvggt_attention(s["q"], s["k"], s["v"], s["scale"], s["causal"], s["starts"], s["kv_starts"], s["lens"], s["max_q"], s["max_kv"], s["out"], s["workspace"])
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------- 64 bits
def _normed64(x, kind, eps, gain, bias):
    x = x.double()
    if kind != "none":
        mean = x.sum(-1, keepdim=True) / x.shape[-1] if kind == "layer" else 0.0
        variance = ((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1]
        x = (x - mean) * (variance + eps) ** -0.5
    if gain is not None:
        x = x * gain.double()
    if bias is not None:
        x = x + bias.double()
    return x


def _turned64(x, s):
    """The rotation as a complex product, pair after pair of channels."""
    if s["rope"] is None:
        return x
    x, n, pair = x.clone(), s["rope_dim"] // 2, s["pair"]
    for p in range(n):
        axis = p * s["axes"] // n if s["pair_axis"] is None else int(s["pair_axis"][p])
        row = s["rope"].double()[s["positions"][axis].long()]
        c = p // pair * 2 * pair + p % pair
        z = torch.complex(x[..., c], x[..., c + pair]) * torch.complex(row[:, p], row[:, n + p])[:, None]
        x[..., c], x[..., c + pair] = z.real, z.imag
    return x


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "heads":
        return {n: _turned64(_normed64(s[n], c["norm"], s["eps"], s[n + "_gain"], s[n + "_bias"]), s) for n in ("q", "k")}
    if c["kind"] == "residual":
        xs, hs = [], []
        for lo in range(0, c["tokens"], 1 << 15):
            part = slice(lo, lo + (1 << 15))
            x = _normed64(s["y"][part], c["post"], s["eps"], s["post_gain"], s["post_bias"])
            r = torch.zeros(len(x), dtype=torch.int64, device=DEV) if s["row_of"] is None else s["row_of"][part].long()
            for factor in (s["channel_scale"], None if s["gate_rows"] is None else s["gate_rows"].double()[r]):
                x = x if factor is None else x * factor.double()
            x = x + s["x"][part].double()
            h = _normed64(x, c["pre"], s["eps"], s["pre_gain"], s["pre_bias"])
            if c["mod"]:
                h = h + h * s["mod_scale"].double()[r] + s["mod_shift"].double()[r]
            xs.append(x)
            hs.append(h)
        return {"x": torch.cat(xs), "h": torch.cat(hs)}
    d, g = c["d"], c["heads"] // c["kv_heads"]
    q_lens, kv_lens = _lengths(c)
    out = torch.zeros(s["T"], c["heads"], d, dtype=torch.float64, device=DEV)
    row, first = 0, s["kv_starts"].tolist()
    for i, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for head in range(c["kv_heads"] if m else 0):
            k, v = (s[name][first[i]:first[i] + m, head].double() for name in ("k", "v"))
            for lo in range(0, n, 4096):
                mine = s["q"][row + lo:row + min(n, lo + 4096), head * g:(head + 1) * g].double()
                x = s["scale"] * (mine.reshape(-1, d) @ k.T).view(len(mine), g, m)
                if c["causal"]:
                    at = m - n + lo + torch.arange(len(mine), device=DEV)
                    x = x.masked_fill((torch.arange(m, device=DEV) > at[:, None])[:, None], -math.inf)
                p = torch.nan_to_num(torch.softmax(x, -1))
                out[row + lo:row + lo + len(mine), head * g:(head + 1) * g] = (p.view(-1, m) @ v).view(len(mine), g, d)
        row += n
    return out
