"""Oracle of the 4-bit key/value cache (include/qvggt.h, the qvggt_kv4_* entry points), float64 numpy, written from the definitions there: rotation by position, the
per-token quantizer in Hadamard space, the bytes of a page, attention over what the pages stand for."""
import numpy as np


def hadamard(d):
    """Orthonormal Sylvester-Hadamard matrix."""
    H = np.ones((1, 1))
    while H.shape[0] < d:
        H = np.block([[H, H], [H, -H]])
    return H / np.sqrt(d)


def turn(x, table, positions, pair):
    """x [T, heads, d] rotated by the rows `positions` of table [rows, dim] (cosines, then sines)."""
    x = np.array(x, np.float64)
    if table is None:
        return x
    dim = table.shape[1]
    out = x.copy()
    for c in range(dim):
        if c & pair:
            continue
        p = (c // (2 * pair)) * pair + c % pair
        cos, sin = (table[np.clip(positions, 0, len(table) - 1), p + k * dim // 2].astype(np.float64)[:, None] for k in (0, 1))
        a, b = x[..., c], x[..., c + pair]
        out[..., c], out[..., c + pair] = a * cos - b * sin, b * cos + a * sin
    return out


def bf16_rne(x):
    """float64 -> the nearest bf16 number, as float64; through float32, which is what a kernel has."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7fff + (b >> 16 & 1)) & 0xffff0000
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


def quantize(x, signs):
    """(codes int, steps) of x [..., d]: z = (s x) H, step = bf16(max |z| / 7), rne(z / step); step NaN and codes 0 where z is not finite."""
    with np.errstate(invalid="ignore"):
        z = (x * signs) @ hadamard(x.shape[-1])
    finite = np.isfinite(z).all(-1)
    z = np.where(finite[..., None], z, 0.0)
    step = np.where(finite, bf16_rne(np.abs(z).max(-1) / 7), np.nan)
    step = np.where(step < 2.0 ** -126, 0.0, step)
    codes = np.rint(np.divide(z, step[..., None], out=np.zeros_like(z), where=step[..., None] > 0)).clip(-8, 7)
    return codes.astype(np.int64), step


def held(codes, steps, signs):
    """What codes [..., d] and steps stand for."""
    return (codes * steps[..., None]) @ hadamard(codes.shape[-1]) * signs


def byte_of(page_tokens, d, t, channel, value):
    """Byte of a head's part of a page that has a channel's code of token t; channel's parity says which half."""
    p = channel // 2
    if not value:
        return t * (d // 2) + p
    w = d // 32
    return page_tokens * d // 2 + (t // 16) * 8 * d + (((t % 16) // 4 * 16 + p // w) * w + p % w) * 4 + t % 4


def store(pool, page_tokens, heads, d, slot, head, which, codes, step):
    """Codes and step of one token, head and kind (0 key, 1 value) into pool (uint8, flat)."""
    base = ((slot // page_tokens) * heads + head) * page_tokens * (d + 4)
    t = slot % page_tokens
    c = np.arange(0, d, 2)
    at = base + byte_of(page_tokens, d, t, c, which)
    pool[at] = (codes[0::2] + 8) | (codes[1::2] + 8) << 4
    word = np.asarray(step, np.float32).view(np.uint32) >> 16
    at = base + page_tokens * d + 4 * t + 2 * which
    pool[at], pool[at + 1] = word & 255, word >> 8


def load(pool, page_tokens, heads, d, slot, head, which):
    """(codes, step) of one token, head and kind."""
    base = ((slot // page_tokens) * heads + head) * page_tokens * (d + 4)
    t = slot % page_tokens
    c = np.arange(d)
    codes = (pool[base + byte_of(page_tokens, d, t, c, which)] >> (c % 2 * 4) & 15).astype(np.int64) - 8
    at = base + page_tokens * d + 4 * t + 2 * which
    return codes, (np.uint32(pool[at]) << np.uint32(16) | np.uint32(pool[at + 1]) << np.uint32(24)).view(np.float32).astype(np.float64)


def attention(q, k, v, scale, causal):
    """One sequence: q [n, heads, d], k and v [m, kv_heads, d] -> [n, heads, d]; zeros where nothing is seen."""
    n, heads, d = q.shape
    m, kv_heads = k.shape[:2]
    out = np.zeros((n, heads, d))
    for h in range(heads if m else 0):
        x = scale * q[:, h] @ k[:, h * kv_heads // heads].T
        if causal:
            x = np.where(np.arange(m) <= m - n + np.arange(n)[:, None], x, -np.inf)
        top = x.max(1, keepdims=True)
        p = np.exp(x - np.where(np.isfinite(top), top, 0.0))
        total = p.sum(1, keepdims=True)
        out[:, h] = np.divide(p, total, out=np.zeros_like(p), where=total > 0) @ v[:, h * kv_heads // heads]
    return out
