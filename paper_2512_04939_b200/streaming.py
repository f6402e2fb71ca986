"""The frame-global attention layer for frames that keep arriving.

The global layer of the paper runs over all frames at once.  Where they come one after another, a layer keeps the keys and values
of the tokens that it has seen (after merging: of the rows that stand for them) and lets the rows of every new chunk attend to
all of them; a frame's rows come out as if the layer had been run over everything up to that frame.
"""
from __future__ import annotations

import torch

from .binding import LiteVGGT
from .kv_cache import NO_QUERIES, KVCache
from .rotary import RotaryAxes


class StreamingGlobalAttention:
    """One attention layer over one growing sequence: QKV projection, K and V into the cache, attention over everything so far,
    output projection.

    ``ctx`` lends its matrix products (any context on the device; its own frame count does not matter).  The cache holds
    ``capacity`` tokens in pages, as bfloat16, as E4M3 codes ("e4m3", about half the memory and, over long sequences, half the
    traffic) or in 4 bits ("e2m1", about a quarter).  ``window`` keeps at least the last that many tokens: whole pages in front of them
    are given back and used again.  ``keep`` is for streams that have no end, but whose past matters: when new rows do not fit, every head
    keeps that many of its tokens, those that have drawn most of the attention so far (the tallies fade by ``decay`` a step), the
    ``first`` first ones and the ``recent`` last ones among them whatever they drew; ``kept`` then says which ones of those held before,
    int32 [keep, heads].  ``rotary`` turns queries and keys by the positions that a step is given.
    """

    def __init__(self, ctx: LiteVGGT, capacity: int, dtype: str = "bf16", page_size: int = 64, window: int | None = None,
                 keep: int | None = None, first: int = 0, recent: int = 0, decay: float = 1.0, rotary: RotaryAxes | None = None):
        if capacity < 1 or (window is not None and not 1 <= window <= capacity):
            raise ValueError(f"capacity must be positive and hold the window, got {capacity} and {window}")
        if keep is None and (first or recent or decay != 1.0):
            raise ValueError("first, recent and decay go with keep")
        if keep is not None and (window is not None or not 1 <= keep < capacity or min(first, recent) < 0 or first + recent > keep
                                 or not 0.0 <= decay <= 1.0):
            raise ValueError(f"keep must be less than the capacity, hold first and recent and go without a window, and decay lie in [0, 1], got "
                             f"keep {keep}, capacity {capacity}, first {first}, recent {recent}, window {window}, decay {decay}")
        if rotary is not None and rotary.head_dim != ctx.dim // ctx.cfg.heads:
            raise ValueError(f"the rotation is for heads of {rotary.head_dim}, the layer's have {ctx.dim // ctx.cfg.heads}")
        self.ctx = ctx
        self.heads, self.head_dim = ctx.cfg.heads, ctx.dim // ctx.cfg.heads
        # (whole pages are given back, so what is kept of a window begins somewhere in its first page: one more than it fills)
        n_pages = -(-capacity // page_size) + (window is not None)
        if keep is not None:  # what is kept moves to pages that nothing is read from
            n_pages += -(-keep // page_size)
        tallies = {} if keep is None else {"weights": True}
        self.cache = KVCache.empty(n_pages, page_size, self.heads, self.head_dim, dtype, ctx.device.index, **tallies)
        self.window = window
        self.capacity, self.keep, self.first, self.recent, self.decay, self.rotary = capacity, keep, first, recent, decay, rotary
        self.kept = None
        self.free = list(range(n_pages))
        self.pages: list[int] = []  # of the tokens held, oldest first
        self.length = 0             # tokens held

    def reset(self):
        """Forget everything; the next rows begin a sequence."""
        self.free += self.pages
        self.pages, self.length, self.kept = [], 0, None

    def step(self, x: torch.Tensor, w_qkv, b_qkv, w_o, b_o, frame_rows: int = 0, positions: torch.Tensor | None = None) -> torch.Tensor:
        """The layer's output for the new rows ``x`` [rows, dim], which join the sequence.  ``frame_rows`` > 0: the rows are
        frames of that many, and a frame does not see those behind it; 0: they all see one another.  If it raises before the rows'
        K and V are stored, the layer is as it was; what raises behind that leaves them in the sequence.  ``positions`` int32 [axes, rows]:
        where the rows stand, with a ``rotary``."""
        self._check(x, w_qkv, b_qkv, w_o, b_o)
        if (positions is None) != (self.rotary is None):
            raise ValueError("positions go with a rotary")
        rows, size = x.shape[0], self.cache.page_size
        spare = 0
        if self.window is not None:
            # what stays in front of the new rows is the window's, less a page at most
            spare = max(0, self.length + rows - max(self.window, rows)) // size
            spare = min(spare, self.length // size)
        held, free, left = self.pages[spare:], self.free + self.pages[:spare], self.length - spare * size
        kept, full = self.kept, self.keep is not None and self.length + rows > self.capacity
        if full:
            if self.keep + rows > self.capacity:
                raise ValueError(f"{rows} new rows do not fit beside the {self.keep} tokens that are kept of {self.capacity}")
            n = -(-self.keep // size)
            held, free, left = self.free[len(self.free) - n:], self.free[:len(self.free) - n] + self.pages, self.keep
        need = -(-(left + rows) // size) - len(held)
        if need > len(free):
            raise ValueError(f"{left} tokens held and {rows} new ones need {need} pages, {len(free)} are free")
        pages, free, length = held + free[len(free) - need:], free[:len(free) - need], left + rows
        qkv = self.ctx.linear(x, w_qkv, b_qkv)
        q, k, v = (t.unflatten(1, (self.heads, self.head_dim)) for t in qkv.split(self.ctx.dim, 1))
        if self.rotary is not None:
            self.rotary.rotate(positions, q, k, out=(q, k))
        if full:  # (the pages that are read are as they were, and the sequence's until the rows are stored)
            source, target = self.cache.batch([0], [self.length], [self.pages]), self.cache.batch([left], [left], [held], NO_QUERIES)
            kept = self.cache.evict(source, target, self.first, self.recent)
        batch = self.cache.batch([rows], [length], [pages], causal_block=frame_rows)
        self.cache.append(batch, k, v)
        self.pages, self.free, self.length, self.kept = pages, free, length, kept
        if self.keep is None:
            out = self.cache.attend(batch, q)
        else:
            out, lse = self.cache.attend(batch, q, lse=True)
            self.cache.weigh(batch, q, lse, decay=self.decay)
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
