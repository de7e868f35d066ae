"""Attention of a transformer block over a stream of frames, all of it on codes: the qkv and output layers as 4-bit layers, the keys and values of the frames seen so far in a 4-bit
cache, a new frame looking at itself and all of them, rotated by row and column of its patches.

    python examples/streaming_attention.py [--frames 8] [--side 37] [--width 1024] [--heads 16]

Prints for every frame the time of its block (layers, append, attention), and how far its attention over the 4-bit cache is from the attention of the same queries, keys and values in
float32.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_21302_amd as q  # noqa: E402


def patch_table(side, d, device):
    """Cosines and sines of patch row * side + column: the first half of the channels turns by the row, the second by the column, d / 4 pairs each."""
    at = torch.arange(side * side, device=device)
    turn = 100.0 ** (-torch.arange(d // 4, device=device) / (d // 4))
    angle = torch.cat([(at // side)[:, None] * turn, (at % side)[:, None] * turn], 1)
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()


class Block:
    """qkv layer, cache, attention, output layer."""

    def __init__(self, width, heads, frames, side, page_tokens=64, device="cuda", seed=0):
        g = torch.Generator(device).manual_seed(seed)
        signs = lambda n: (torch.randint(0, 2, (n,), device=device, generator=g) * 2 - 1).to(torch.int8)  # noqa: E731
        self.heads, self.d, self.tokens = heads, width // heads, side * side
        self.w_qkv, self.w_out = (torch.randn(n * width, width, device=device, generator=g).mul_(1 / math.sqrt(width)).to(torch.bfloat16) for n in (3, 1))
        self.qkv = q.DsfqLinear(self.w_qkv, None, signs(width), calibration=torch.randn(512, width, device=device, generator=g).to(torch.bfloat16))
        self.out = q.DsfqLinear(self.w_out, None, signs(width), calibration=torch.randn(512, width, device=device, generator=g).to(torch.bfloat16))
        pages = -(-frames * self.tokens // page_tokens)
        self.rope = patch_table(side, self.d, device)
        self.cache = q.Kv4Cache(pages, page_tokens, heads, self.d, signs(self.d), self.rope, self.d // 4, device)
        self.table = torch.randperm(pages, device=device, generator=g).int()[None].contiguous()
        self.positions = torch.arange(self.tokens, device=device, dtype=torch.int32)
        self.starts = torch.tensor([0, self.tokens], device=device, dtype=torch.int32)
        self.seen = 0

    def __call__(self, x):
        """A frame's tokens [tokens, width] bf16 -> [tokens, width] bf16; the frame joins the cache."""
        return self.out(self.attention(x).view(x.shape))

    def rows(self, x):
        """Queries, keys and values of a frame's tokens, [tokens, 3 heads, d], behind one another in every row: the entry points take them as they lie."""
        return self.qkv(x).view(-1, 3 * self.heads, self.d)

    def slots(self, first, count):
        at = first + torch.arange(count, device=self.table.device)
        return self.table[0, at // self.cache.page_tokens] * self.cache.page_tokens + (at % self.cache.page_tokens).int()

    def attention(self, x):
        h, rows = self.heads, self.rows(x)
        self.cache.append(rows[:, h:2 * h], rows[:, 2 * h:], self.slots(self.seen, self.tokens), self.positions)
        self.seen += self.tokens
        lens = torch.full((1,), self.seen, device=x.device, dtype=torch.int32)
        return self.cache.attend(rows[:, :h], self.table, self.starts, lens, self.tokens, self.seen, self.positions, causal=False)

    def turned(self, x):
        """The rotation by row and column of x [tokens, heads, d], in float32."""
        cos, sin = (t.transpose(1, 2) for t in self.rope.view(-1, 2, 2, 1, self.d // 4).unbind(1))         # [tokens, 1, 2 halves, d / 4]
        a, b = x.float().unflatten(2, (2, 2, self.d // 4)).unbind(3)
        return torch.stack([a * cos - b * sin, b * cos + a * sin], 3).flatten(2)


def plain_attention(queries, keys, values):
    """[n, heads, d] over [m, heads, d], in float32."""
    o = torch.empty_like(queries)
    for i in range(queries.shape[1]):
        o[:, i] = torch.softmax(queries[:, i] @ keys[:, i].T / math.sqrt(queries.shape[2]), 1) @ values[:, i]
    return o


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("frames", 8), ("side", 37), ("width", 1024), ("heads", 16)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    block, g = Block(a.width, a.heads, a.frames, a.side), torch.Generator("cuda").manual_seed(1)
    h, keys, values, errors = a.heads, [], [], []
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for i in range(a.frames):
        x = torch.randn(a.side * a.side, a.width, device="cuda", generator=g).to(torch.bfloat16)
        rows = block.rows(x)
        keys.append(block.turned(rows[:, h:2 * h]))
        values.append(rows[:, 2 * h:].float())
        want = plain_attention(block.turned(rows[:, :h]), torch.cat(keys), torch.cat(values))
        begin.record()
        got = block.attention(x)
        y = block.out(got.view(x.shape))
        end.record()
        errors.append(float((got.float() - want).norm() / want.norm()))
        print(f"frame {i + 1}: {begin.elapsed_time(end) * 1e3:7.1f} us, attention {errors[-1]:.3f} from float32, {tuple(y.shape)}", flush=True)
    return errors


if __name__ == "__main__":
    main()
