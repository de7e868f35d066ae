"""A small convenience object around the qvggt_kv4_* entry points: a pool of pages that holds keys and values in 4 bits, appended to and attended over.

It only allocates device tensors with torch and calls the entry points; which page belongs to which sequence is the caller's to keep.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import binding as q


class Kv4Cache:
    """num_pages pages of page_tokens tokens (a power of two, 16 .. 1024) of `heads` key/value heads of head_dim (64 or 128) channels.

    signs: int8 [head_dim] of +-1, or None; rope: f32 [rows, rope_dim] cosines and sines by position, or None, with rope_pair the distance of the channels that turn together
    (include/qvggt.h).  A cache keeps one workspace, as a layer does: attend() calls of one cache follow each other on one stream, from one thread at a time.  A larger call replaces it; one
    that a captured call was given stays the cache's, since every replay writes into it.
    """

    def __init__(self, num_pages: int, page_tokens: int, heads: int, head_dim: int, signs: Optional[torch.Tensor] = None, rope: Optional[torch.Tensor] = None, rope_pair: int = 0,
                 device="cuda"):
        size = q.qvggt_kv4_page_bytes(page_tokens, heads, head_dim)
        if size == 0:
            raise q.QvggtError(q.ERR_SHAPE, "Kv4Cache")
        self.page_tokens, self.heads, self.head_dim = page_tokens, heads, head_dim
        self.signs, self.rope, self.rope_pair = signs, rope, rope_pair
        self.pages = torch.empty(num_pages, size, dtype=torch.uint8, device=device)
        self._ws = None
        self._captured = []         # workspaces that captured calls write into

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None) -> None:
        """Keys (turned by their positions) and values [T, heads, head_dim] into slots int32 [T]: page * page_tokens + offset; -1 leaves a token out."""
        q.qvggt_kv4_append(k, v, self.signs, slots, self.pages, self.page_tokens, rope=self.rope, positions=positions, rope_pair=self.rope_pair)

    def attend(self, queries: torch.Tensor, page_table: torch.Tensor, q_starts: torch.Tensor, kv_lens: torch.Tensor, max_q: int, max_kv: int,
               positions: Optional[torch.Tensor] = None, causal: bool = True, scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of queries [T, q_heads, head_dim] of several sequences over the keys and values in their pages; bf16, written into `out` when given."""
        T, heads, d = queries.shape
        need = q.qvggt_kv4_attention_workspace_bytes(T, page_table.shape[0], max_q, max_kv, heads, self.heads, d)
        ws = self._ws
        if need and (ws is None or ws.numel() < need):
            ws = self._ws = torch.empty(need, dtype=torch.uint8, device=queries.device)
        if need and q.capturing(queries) and not any(ws is kept for kept in self._captured):
            self._captured.append(ws)
        if out is None:
            out = torch.empty(T, heads, d, dtype=torch.bfloat16, device=queries.device)
        q.qvggt_kv4_attention(queries, self.signs, 1 / math.sqrt(d) if scale is None else float(scale), causal, self.pages, self.page_tokens, self.heads, page_table, q_starts, kv_lens,
                              max_q, max_kv, out, ws, rope=self.rope, positions=positions, rope_pair=self.rope_pair)
        return out

    def read(self, slots: torch.Tensor, dtype=torch.bfloat16):
        """The keys and values that slots hold, [T, heads, head_dim] each; zeros for slots outside the pool."""
        k, v = (torch.empty(slots.numel(), self.heads, self.head_dim, dtype=dtype, device=slots.device) for _ in range(2))
        q.qvggt_kv4_read(self.pages, self.page_tokens, self.signs, slots, k, v)
        return k, v
