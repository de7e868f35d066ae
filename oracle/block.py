"""Oracle of the operators around a block's layers (include/qvggt.h: qvggt_heads_norm_rope, qvggt_attention, qvggt_residual_norm), float64 torch on any device, written from the definitions
there.  Each comes with a bound, value by value, on what arithmetic of the stated precisions may be off by (u = 2^-24 is half a step of fp32, 2^-8 of bf16, relative):

    a sum of n terms in fp32, in any order          n u  sum |terms|
    1 / sqrt, exp2                                  2 u  of themselves (instructions of one unit in the last place)
    rounding of a result                            half a step of its type
"""
import math

import torch

U = 2.0 ** -24
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def norm(x, kind, eps, gain=None, bias=None, off=None):
    """(values, bound) of a norm over the last axis of float64 x, each value of which is off by `off` at most."""
    n = x.shape[-1]
    off = torch.zeros_like(x) if off is None else off
    if kind != "none":
        if kind == "layer":
            mean = x.mean(-1, keepdim=True)
            off = off + off.mean(-1, keepdim=True) + n * U * x.abs().mean(-1, keepdim=True)
            x = x - mean
            off = off + U * x.abs()
        v = (x * x).mean(-1, keepdim=True) + eps
        f = v.rsqrt()
        # the root of the mean square moves by the root of the mean square of what its terms are off by, at most
        share = (off * off).mean(-1, keepdim=True).sqrt() * f + (n / 2 + 8) * U
        y = x * f
        off = off * f + y.abs() * share
        off, x = off * (1 + share), y
    for factor in (gain,):
        if factor is not None:
            x, off = x * factor.double(), (off + 2 * U * x.abs()) * factor.double().abs()
    if bias is not None:
        x = x + bias.double()
        off = off + 2 * U * (x.abs() + bias.double().abs())
    return x, off + 2 * U * x.abs()


def rounded(x, off, dtype):
    """The bound with the rounding to a type."""
    return off + STEP[dtype] * (x.abs() + off) + 1e-37


def turn(x, off, table, positions, pair, pair_axis=None):
    """(values, bound) of x [T, heads, d] turned by table [rows, dim] and positions [axes, T]."""
    if table is None:
        return x, off
    n, axes = table.shape[1] // 2, positions.shape[0]
    x, off = x.clone(), off.clone()
    for p in range(n):
        axis = min(p * axes // n if pair_axis is None else int(pair_axis[p]), axes - 1)
        row = table[positions[axis].long().clamp(0, table.shape[0] - 1)].double()
        cos, sin, c = row[:, None, p], row[:, None, n + p], p // pair * 2 * pair + p % pair
        a, b, da, db = x[..., c].clone(), x[..., c + pair].clone(), off[..., c].clone(), off[..., c + pair].clone()
        x[..., c], x[..., c + pair] = a * cos - b * sin, b * cos + a * sin
        off[..., c] = da * cos.abs() + db * sin.abs() + 3 * U * ((a * cos).abs() + (b * sin).abs())
        off[..., c + pair] = db * cos.abs() + da * sin.abs() + 3 * U * ((b * cos).abs() + (a * sin).abs())
    return x, off


def heads_norm_rope(x, kind, eps, gain, bias, table, positions, pair, pair_axis=None):
    y, off = turn(*norm(x.double(), kind, eps, gain, bias), table, positions, pair, pair_axis)
    return y, rounded(y, off, x.dtype)


def residual_norm(x, y, x_dtype, h_dtype, post="none", post_gain=None, post_bias=None, scale=None, gate=None, kind="none", gain=None, bias=None, mod_scale=None, mod_shift=None, row_of=None,
                  eps=1e-6):
    """((x', bound), (h, bound))."""
    M = x.shape[0]
    if row_of is None:
        of = lambda t: t.double().expand(M, -1)  # noqa: E731
    else:
        of = lambda t: t.double()[row_of.long().clamp(0, t.shape[0] - 1)]  # noqa: E731
    s, off = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    if y is not None:
        u, off = norm(y.double(), post, eps, post_gain, post_bias)
        for factor in (scale, None if gate is None else of(gate)):
            if factor is not None:
                u, off = u * factor.double(), (off + 2 * U * u.abs()) * factor.double().abs()
        s = s + u
        off = off + 2 * U * s.abs()
    h, h_off = norm(s, kind, eps, gain, bias, off)
    if mod_scale is not None:
        h_off = h_off * (1 + of(mod_scale)).abs() + 2 * U * (h.abs() + (h * of(mod_scale)).abs())
        h = h * (1 + of(mod_scale))
    if mod_shift is not None:
        h = h + of(mod_shift)
        h_off = h_off + 2 * U * (h.abs() + of(mod_shift).abs())
    return (s, rounded(s, off, x_dtype)), (h, rounded(h, h_off, h_dtype))


def attention(q, k, v, scale, causal, lengths, starts, max_q=None, max_kv=None):
    """(out, bound) [T, heads, d]; lengths: (queries, keys) of every sequence, queries one after another from row 0, keys from row starts[b].

    Weights are rounded to bf16 in the product and in the sum that divides it, so a weight's 2^-8 counts by how far its value is from the result; a score's error (sums of d products, three
    roundings around the exponent) is one of its weight, and counts the same way.
    """
    T, heads, d = q.shape
    group = heads // k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    off = torch.full_like(out, 1e-37)          # (rows that see nothing are zeros)
    row = 0
    for (n, m), first in zip(lengths, starts):
        answered = n if max_q is None else min(n, max_q)
        looked = m if max_kv is None else min(m, max_kv)
        for h in range(heads if looked else 0):
            mine = q[row:row + answered, h].double()
            kk, vv = (t[first:first + looked, h // group].double() for t in (k, v))
            for lo in range(0, answered, 1024):
                some = mine[lo:lo + 1024]
                x, terms = scale * (some @ kk.T), abs(scale) * (some.abs() @ kk.abs().T)
                if causal:
                    hidden = torch.arange(looked, device=q.device) > m - n + lo + torch.arange(len(some), device=q.device)[:, None]
                    x, terms = x.masked_fill(hidden, -math.inf), terms.masked_fill(hidden, 0.0)
                # a row that sees no key is zeros, one whose scores are all -infinity no number
                sees = torch.ones_like(x, dtype=torch.bool) if not causal else ~hidden
                p = torch.where(sees.any(-1, keepdim=True), torch.softmax(x, -1), 0.0)
                o = p @ vv
                e = (d + 8) * U * terms.amax(-1, keepdim=True) * 2 + 8 * U
                # sum p |v - o|, a channel at a time where that is much
                if p.numel() * d <= 1 << 24:
                    spread = (p[:, :, None] * (vv[None] - o[:, None]).abs()).sum(1)
                else:
                    spread = torch.stack([(p * (vv[:, c] - o[:, c:c + 1]).abs()).sum(1) for c in range(d)], 1)
                sums = (looked + 64) * U * (p @ vv.abs() + o.abs())
                at = slice(row + lo, row + lo + len(some))
                out[at, h] = o
                off[at, h] = rounded(o, (2.0 ** -8 + e) * 1.01 * spread + sums, torch.bfloat16)
        row += n
    return out, off
