"""A paged K/V cache and the attention that reads it, for frames that keep arriving.

    cache = KVCache.empty(pages, page_size, kv_heads, head_dim, dtype="e4m3")
    batch = cache.batch(rows=[1041], lengths=[52050], pages=[page_ids])    # once per step: the same for every call on this cache
    cache.append(batch, k, v)                                              # the last 1041 tokens of the sequence
    out = cache.attend(batch, q)                                           # over all 52050

Which pages a sequence owns is the caller's business; the library checks that they exist - in the pool of the cache that plans the
batch, and no other cache takes it.  Shapes, types, strides and
devices are checked here, everything else in the C library.
"""
from __future__ import annotations

import ctypes as C
import math

import numpy as np
import torch

from .binding import KVConfig, _check, load_library

_DTYPES = {"bf16": (0, torch.bfloat16), "e4m3": (1, torch.float8_e4m3fn)}


def _whole(name: str, numbers) -> np.ndarray:
    """One whole number after another, as 64-bit ones."""
    given = np.asarray(numbers)
    with np.errstate(invalid="ignore"):
        whole = given.astype(np.int64)
    if given.ndim != 1 or not np.array_equal(given, whole):
        raise ValueError(f"{name} must be whole numbers in one dimension")
    return whole


class KVBatch:
    """Rows, lengths and pages of a step's sequences, planned for one cache (see :meth:`KVCache.batch`)."""

    def __init__(self, owner: "KVCache", handle, memory: torch.Tensor, rows: int, q_heads: int, stream: int):
        self.owner = owner
        self.handle = handle
        self.memory = memory
        self.rows = rows
        self.q_heads = q_heads
        self.kv_shape = (rows, owner.kv_heads, owner.head_dim)
        self.q_shape = (rows, q_heads, owner.head_dim)
        self._stream = stream

    def __del__(self):  # pragma: no cover
        try:
            if self.handle is not None:
                self.owner.lib.litevggt_kv_batch_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


class KVCache:
    """A cache over pools of the caller's: ``k``, ``v`` [pages, kv_heads, page_size, head_dim], bfloat16, or float8_e4m3fn
    with the exponents ``k_exp``, ``v_exp`` uint8 [pages, kv_heads, page_size]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor | None = None, v_exp: torch.Tensor | None = None):
        self.lib = load_library()
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError(f"k and v must both be [pages, kv_heads, page_size, head_dim], got {tuple(k.shape)} and {tuple(v.shape)}")
        narrow = k.dtype == torch.float8_e4m3fn
        if not narrow and k.dtype != torch.bfloat16 or v.dtype != k.dtype:
            raise ValueError(f"k and v must both be bfloat16 or both float8_e4m3fn, got {k.dtype} and {v.dtype}")
        tensors = {"k": k, "v": v}
        if narrow:
            for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
                if t is None or t.dtype != torch.uint8 or t.shape != k.shape[:3]:
                    raise ValueError(f"{name} must be uint8 {tuple(k.shape[:3])} beside float8_e4m3fn pools")
                tensors[name] = t
        elif k_exp is not None or v_exp is not None:
            raise ValueError("bfloat16 pools have no exponents")
        for name, t in tensors.items():
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
            if not t.is_cuda or t.device != k.device:
                raise ValueError("every pool must live on the same CUDA device")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.device, self._index = k.device, k.get_device()
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self._scale = 1.0 / math.sqrt(self.head_dim)
        self._append, self._attend = self.lib.litevggt_kv_append, self.lib.litevggt_kv_attend
        self.status = torch.zeros(64, dtype=torch.int32, device=k.device)
        self._home = self._stream()
        cfg = KVConfig(self.pages, self.page_size, self.kv_heads, self.head_dim, 1 if narrow else 0)
        self.handle = C.c_void_p()
        _check(self.lib.litevggt_kv_create(C.byref(cfg), self.device.index, *(C.c_void_p(t.data_ptr()) if t is not None else None
                                                                             for t in (k, v, k_exp, v_exp, self.status)),
                                           C.byref(self.handle)), "kv_create")

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype: str = "bf16", device: int = 0) -> "KVCache":
        """A cache with pools of its own, not initialised."""
        if dtype not in _DTYPES:
            raise ValueError(f"dtype must be one of {sorted(_DTYPES)}, got {dtype!r}")
        where = torch.device("cuda", device)
        shape = (pages, kv_heads, page_size, head_dim)
        pools = [torch.empty(shape, dtype=_DTYPES[dtype][1], device=where) for _ in range(2)]
        if dtype == "e4m3":
            pools += [torch.empty(shape[:3], dtype=torch.uint8, device=where) for _ in range(2)]
        return cls(*pools)

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.litevggt_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ a step
    def batch(self, rows, lengths, pages, q_heads: int | None = None, causal_block: int = 0) -> KVBatch:
        """Plans a step: ``rows[i]`` rows of the packed tensors belong to sequence i, which holds ``lengths[i]`` tokens (those
        rows included, as its last) in the pages ``pages[i]`` (more than it needs may be named).  ``causal_block`` = c: a
        row sees the tokens before its sequence's rows and the blocks of c rows up to its own; 0: all of them."""
        if len(rows) != len(lengths) or len(rows) != len(pages) or len(rows) == 0:
            raise ValueError(f"rows, lengths and pages name {len(rows)}, {len(lengths)} and {len(pages)} sequences")
        n_rows, n_tokens = _whole("rows", rows), _whole("lengths", lengths)
        if min(n_rows.min(), n_tokens.min()) < 0 or max(n_rows.max(), n_tokens.max()) >= 2 ** 31:
            raise ValueError("rows and lengths must lie in [0, 2^31)")
        lists = []
        for n, ids in zip(n_tokens.tolist(), pages):
            need = -(-n // self.page_size)
            if len(ids) < need:
                raise ValueError(f"a sequence of {n} tokens needs {need} pages, got {len(ids)}")
            lists.append(np.asarray(ids[:need]))
        flat = _whole("pages", lists[0] if len(lists) == 1 else np.concatenate(lists))
        if flat.size and (flat.min() < 0 or flat.max() >= self.pages):
            raise ValueError(f"pages must lie in [0, {self.pages})")
        r32, n32, p32 = (np.ascontiguousarray(a, np.int32) for a in (n_rows, n_tokens, flat))
        q_heads = self.kv_heads if q_heads is None else q_heads
        if max(abs(q_heads), abs(causal_block)) >= 2 ** 31:  # (ctypes would pass the lower 32 bits)
            raise ValueError(f"q_heads and causal_block must be less than 2^31, got {q_heads} and {causal_block}")
        handle, n_bytes = C.c_void_p(), C.c_size_t()
        _check(self.lib.litevggt_kv_batch_create(self.handle, len(rows), r32.ctypes.data, n32.ctypes.data, p32.ctypes.data, q_heads,
                                                 causal_block, C.byref(handle), C.byref(n_bytes)), "kv_batch_create")
        with torch.cuda.device(self.device):
            memory = torch.empty(n_bytes.value, dtype=torch.uint8, device=self.device)
        stream = self._stream()
        made = KVBatch(self, handle, memory, int(n_rows.sum()), q_heads, stream)
        _check(self.lib.litevggt_kv_batch_place(handle, memory.data_ptr(), n_bytes.value, stream), "kv_batch_place")
        return made

    def append(self, batch: KVBatch, k: torch.Tensor, v: torch.Tensor) -> None:
        """Writes ``k``, ``v`` [batch.rows, kv_heads, head_dim] (bfloat16; slices of a fused projection will do) into the
        batch's sequences as their last tokens."""
        code = self._append(self.handle, batch.handle, *self._rows("k", k, batch.kv_shape), *self._rows("v", v, batch.kv_shape),
                            self._use(batch))
        if code:
            _check(code, "kv_append")

    def gather(self, batch: KVBatch) -> tuple[torch.Tensor, torch.Tensor]:
        """K and V of the batch's rows, bfloat16 [batch.rows, kv_heads, head_dim]."""
        k = torch.empty(batch.kv_shape, dtype=torch.bfloat16, device=self.device)
        v = torch.empty_like(k)
        _check(self.lib.litevggt_kv_gather(self.handle, batch.handle, k.data_ptr(), v.data_ptr(), self._use(batch)), "kv_gather")
        return k, v

    def attend(self, batch: KVBatch, q: torch.Tensor, scale: float | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
        """softmax(scale q K^T) V of the batch's rows over the tokens that they see; ``q`` bfloat16 [batch.rows, q_heads, head_dim].
        ``scale`` is 1 / sqrt(head_dim) unless given (positive, less than 1e30).  ``out``, if given, must not lie where ``q`` does.  A row that sees no token
        comes out as zero."""
        q_rows = self._rows("q", q, batch.q_shape)
        if out is None:
            out = q.new_empty(batch.q_shape)
        else:
            self._rows("out", out, batch.q_shape)
            if not out.is_contiguous():
                raise ValueError("out must be contiguous")
        code = self._attend(self.handle, batch.handle, *q_rows, self._scale if scale is None else scale, out.data_ptr(), self._use(batch))
        if code:
            _check(code, "kv_attend")
        return out

    # ------------------------------------------------------------------ checks
    def poll(self):
        """Synchronise the current stream; raise if a kernel gave up on a wait."""
        _check(self.lib.litevggt_kv_poll(self.handle, self._stream()), "kv_poll")

    def launch_count(self) -> int:
        n = C.c_int64()
        _check(self.lib.litevggt_kv_launch_count(self.handle, C.byref(n)), "kv_launch_count")
        return n.value

    def _stream(self) -> int:
        return torch._C._cuda_getCurrentRawStream(self._index)  # (a Stream object costs 3 us)

    def _use(self, batch: KVBatch) -> int:
        """The current stream.  Where the batch or the pools come from another one, their memory is in use on this one as well, and
        is not given away before its work here is done."""
        stream = self._stream()
        if stream != batch._stream or stream != self._home:
            here = torch.cuda.current_stream(self.device)
            batch.memory.record_stream(here)
            for t in (self.k, self.v, self.k_exp, self.v_exp, self.status):
                if t is not None:
                    t.record_stream(here)
        return stream

    def _rows(self, name: str, t: torch.Tensor, shape: tuple) -> tuple[int, int, int]:
        """A checked tensor's address and its strides from row to row and head to head (that of a dimension of one says nothing)."""
        if t.shape != shape:
            raise ValueError(f"{name} must be {list(shape)}, got {tuple(t.shape)}")
        if t.dtype != torch.bfloat16 or t.get_device() != self._index:
            raise ValueError(f"{name} must be bfloat16 on {self.device}, got {t.dtype} on {t.device}")
        row, head, channel = t.stride()
        row, head, address = row if shape[0] > 1 else 0, head if shape[1] > 1 else 0, t.data_ptr()
        if channel != 1 or row % 8 or head % 8 or address % 16:
            raise ValueError(f"{name}'s head_dim must be contiguous, its rows and heads 16-byte aligned, got strides {t.stride()}")
        return address, row, head
