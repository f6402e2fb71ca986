"""Queries and keys turned by their positions along several axes: time, height and width of a token of a video.

    rotary = RotaryAxes(64, sections=(16, 24, 24), bases=(10000.0, 100.0, 100.0))
    q, k = rotary.rotate(positions, q, k)              # positions int32 [3, rows]; q, k [rows, heads, 64], slices of a projection will do
    grad_q, grad_k = rotary.rotate_back(positions, grad_q, grad_k)   # the gradient

Nothing here enters an autograd graph: tensors that require a gradient are refused unless gradients are off (``torch.no_grad``, or inside the
``forward`` and ``backward`` of a ``torch.autograd.Function``, which is where ``rotate`` and ``rotate_back`` belong in training).

Shapes, types and devices are checked here, everything else in the C library.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch

from .binding import RotaryConfig, _check, load_library

_LAYOUTS = {"halves": 0, "pairs": 1, "across": 2}
_PACK = tuple(struct.Struct("@" + "qqqqqqi4x" * n).pack for n in (1, 2))  # litevggt_rotary_tensor, one and two of them
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class RotaryAxes:
    """Axis a turns ``sections[a]`` channels of a head (even numbers, together at most ``head_dim``; what lies behind them stays) by
    position * bases[a]^(-i / n) in the i-th of its n planes.  ``layout``: which channels make a plane - ``halves`` of the axis's own
    section, neighbouring ``pairs``, or halves ``across`` all sections, with one ladder of frequencies for all axes."""

    def __init__(self, head_dim: int, sections, bases, layout: str = "halves", device: int = 0):
        sections, bases = tuple(sections), tuple(bases)
        if layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}, got {layout!r}")
        if not 1 <= len(sections) <= 4 or len(bases) != len(sections):
            raise ValueError(f"one to four axes with a section and a base each, got {sections} and {bases}")
        if any(int(n) != n or not 0 <= n < 2 ** 31 for n in (head_dim, *sections)):
            raise ValueError(f"head_dim and sections must be whole numbers, got {head_dim} and {sections}")
        if not 0 <= device < torch.cuda.device_count():
            raise ValueError(f"there is no CUDA device {device}")
        self.lib = load_library()
        self.head_dim, self.sections, self.bases, self.layout = int(head_dim), tuple(int(n) for n in sections), bases, layout
        self.device = torch.device("cuda", device)
        self._index = device
        self._axes = n = len(sections)
        cfg = RotaryConfig(self.head_dim, n, (C.c_int32 * 4)(*self.sections), (C.c_double * 4)(*bases), _LAYOUTS[layout])
        self.handle = C.c_void_p()
        self._table = torch.empty(2048, dtype=torch.uint8, device=self.device)
        self._home = torch._C._cuda_getCurrentRawStream(device)
        _check(self.lib.litevggt_rotary_create(C.byref(cfg), device, self._table.data_ptr(), 2048, self._home, C.byref(self.handle)), "rotary_create")
        self._apply = self.lib.litevggt_rotary_apply

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.litevggt_rotary_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def rotate(self, positions: torch.Tensor, q: torch.Tensor, k: torch.Tensor | None = None, out=None):
        """``q`` (and ``k``) turned: [rows, heads, head_dim], bfloat16, float16 or float32, the head's channels contiguous, by ``positions``
        int32 [axes, rows].  New tensors, or those of ``out`` (one, or a pair beside a ``k``), which may be the inputs themselves."""
        return self._turn(positions, q, k, out, 0)

    def rotate_back(self, positions: torch.Tensor, q: torch.Tensor, k: torch.Tensor | None = None, out=None):
        """The reverse, and the gradient of :meth:`rotate`: from the gradients of its outputs to those of its inputs."""
        return self._turn(positions, q, k, out, 1)

    def _turn(self, positions, q, k, out, back):
        # (a small call takes as long as its checks do)
        if k is None:
            given, graph = (q,), q.requires_grad
            outs = (torch.empty_like(q),) if out is None else (out,)
        else:
            given, graph = (q, k), q.requires_grad or k.requires_grad
            outs = (torch.empty_like(q), torch.empty_like(k)) if out is None else tuple(out)
        if (graph or (out is not None and any(o.requires_grad for o in outs))) and torch.is_grad_enabled():
            raise ValueError("rotations are not recorded by autograd, and their gradient would be lost: call them under torch.no_grad() or in "
                             "a torch.autograd.Function, with rotate_back for the gradients, or detach the tensors")
        kind, rows, index = _DTYPES.get(q.dtype), q.shape[0] if q.dim() == 3 else -1, self._index
        fine = (kind is not None and len(outs) == len(given) and positions.shape == (self._axes, rows) and positions.dtype == torch.int32
                and positions.get_device() == index)
        numbers = []
        if fine:
            for t, o in zip(given, outs):
                shape, s, z = t.shape, t.stride(), o.stride()
                fine = (fine and len(shape) == 3 and shape[0] == rows and shape[1] >= 1 and shape[2] == self.head_dim and o.shape == shape
                        and t.dtype == q.dtype and o.dtype == q.dtype and t.get_device() == index and o.get_device() == index
                        and s[2] == 1 and z[2] == 1)
                if not fine:
                    break
                numbers += (t.data_ptr(), s[0], s[1], o.data_ptr(), z[0], z[1], shape[1])
        if not fine:
            self._refuse(positions, given, outs, rows)
        axis_stride, row_stride = positions.stride()
        stream = torch._C._cuda_getCurrentRawStream(index)
        if stream != self._home:  # the table is in use there as well, and is not given away before that is done
            self._table.record_stream(torch.cuda.current_stream(index))
        code = self._apply(self.handle, positions.data_ptr(), axis_stride, row_stride, rows, kind, back, _PACK[len(given) - 1](*numbers),
                           len(given), stream)
        if code:
            _check(code, "rotary_apply")
        return outs[0] if k is None else outs

    def _refuse(self, positions, given, outs, rows):
        if len(outs) != len(given):
            raise ValueError(f"out must hold {len(given)} tensors, got {len(outs)}")
        for name, t, o in zip(("q", "k"), given, outs):
            if t.dim() != 3 or t.shape[0] != rows or t.shape[1] < 1 or t.shape[2] != self.head_dim or o.shape != t.shape:
                raise ValueError(f"{name} and its output must be [{rows}, heads, {self.head_dim}], got {tuple(t.shape)} and {tuple(o.shape)}")
            if t.dtype not in _DTYPES or t.dtype != given[0].dtype or o.dtype != t.dtype:
                raise ValueError(f"q, k and their outputs must be of one type, bfloat16, float16 or float32, got {t.dtype} and {o.dtype} for {name}")
            if t.get_device() != self._index or o.get_device() != self._index:
                raise ValueError(f"{name} and its output must be on {self.device}, got {t.device} and {o.device}")
            if t.stride(2) != 1 or o.stride(2) != 1:
                raise ValueError(f"{name}'s channels must be contiguous, got strides {t.stride()} and {o.stride()}")
        raise ValueError(f"positions must be int32 [{self._axes}, {rows}] on {self.device}, got {positions.dtype} {tuple(positions.shape)} on {positions.device}")
