"""The frame-global attention layer for frames that keep arriving.

The global layer of the paper runs over all frames at once.  Where they come one after another, a layer keeps the keys and values
of the tokens that it has seen (after merging: of the rows that stand for them) and lets the rows of every new chunk attend to
all of them; a frame's rows come out as if the layer had been run over everything up to that frame.
"""
from __future__ import annotations

import torch

from .binding import LiteVGGT
from .kv_cache import KVCache


class StreamingGlobalAttention:
    """One attention layer over one growing sequence: QKV projection, K and V into the cache, attention over everything so far,
    output projection.

    ``ctx`` lends its matrix products (any context on the device; its own frame count does not matter).  The cache holds
    ``capacity`` tokens in pages, as bfloat16 or as E4M3 codes (about half the memory and, over long sequences, half the
    traffic).  ``window`` keeps at least the last that many tokens: whole pages in front of them are given back and used again.
    """

    def __init__(self, ctx: LiteVGGT, capacity: int, dtype: str = "bf16", page_size: int = 64, window: int | None = None):
        if capacity < 1 or (window is not None and not 1 <= window <= capacity):
            raise ValueError(f"capacity must be positive and hold the window, got {capacity} and {window}")
        self.ctx = ctx
        self.heads, self.head_dim = ctx.cfg.heads, ctx.dim // ctx.cfg.heads
        # (whole pages are given back, so what is kept of a window begins somewhere in its first page: one more than it fills)
        n_pages = -(-capacity // page_size) + (window is not None)
        self.cache = KVCache.empty(n_pages, page_size, self.heads, self.head_dim, dtype, ctx.device.index)
        self.window = window
        self.free = list(range(n_pages))
        self.pages: list[int] = []  # of the tokens held, oldest first
        self.length = 0             # tokens held

    def reset(self):
        """Forget everything; the next rows begin a sequence."""
        self.free += self.pages
        self.pages, self.length = [], 0

    def step(self, x: torch.Tensor, w_qkv, b_qkv, w_o, b_o, frame_rows: int = 0) -> torch.Tensor:
        """The layer's output for the new rows ``x`` [rows, dim], which join the sequence.  ``frame_rows`` > 0: the rows are
        frames of that many, and a frame does not see those behind it; 0: they all see one another.  If it raises before the rows'
        K and V are stored, the layer is as it was; what raises behind that leaves them in the sequence."""
        self._check(x, w_qkv, b_qkv, w_o, b_o)
        rows, size = x.shape[0], self.cache.page_size
        spare = 0
        if self.window is not None:
            # what stays in front of the new rows is the window's, less a page at most
            spare = max(0, self.length + rows - max(self.window, rows)) // size
            spare = min(spare, self.length // size)
        held, free, left = self.pages[spare:], self.free + self.pages[:spare], self.length - spare * size
        need = -(-(left + rows) // size) - len(held)
        if need > len(free):
            raise ValueError(f"{left} tokens held and {rows} new ones need {need} pages, {len(free)} are free")
        pages, free, length = held + free[len(free) - need:], free[:len(free) - need], left + rows
        qkv = self.ctx.linear(x, w_qkv, b_qkv)
        q, k, v = (t.unflatten(1, (self.heads, self.head_dim)) for t in qkv.split(self.ctx.dim, 1))
        batch = self.cache.batch([rows], [length], [pages], causal_block=frame_rows)
        self.cache.append(batch, k, v)
        self.pages, self.free, self.length = pages, free, length
        out = self.cache.attend(batch, q)
        return self.ctx.linear(out.flatten(1), w_o, b_o)

    def _check(self, x, w_qkv, b_qkv, w_o, b_o):
        """The matrix product is told sizes and trusts every extent; all operands are looked at before the sequence changes."""
        d = self.ctx.dim
        if x.dim() != 2 or x.shape[0] < 1:
            raise ValueError(f"x must be [rows, {d}] with at least one row, got {tuple(x.shape)}")
        for name, t, shape in (("x", x, (x.shape[0], d)), ("w_qkv", w_qkv, (3 * d, d)), ("b_qkv", b_qkv, (3 * d,)), ("w_o", w_o, (d, d)), ("b_o", b_o, (d,))):
            if t is None and name.startswith("b_"):
                continue
            if t is None or t.shape != shape:
                raise ValueError(f"{name} must be {list(shape)}, got {None if t is None else tuple(t.shape)}")
            if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.device != self.ctx.device:
                raise ValueError(f"{name} must be a contiguous bfloat16 tensor on {self.ctx.device}, got {t.dtype} on {t.device}")
