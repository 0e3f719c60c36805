"""Rotary positions over several axes (include/clq_rope.h) on torch tensors.

``Rope`` holds the frequencies of a head's pairs; a call turns the heads of queries and keys, which
may lie in the packed output of a QKV product, by their tokens' positions in time, height and
width.  Every step runs in libclq.so.
"""
import ctypes
import fractions
import struct

import torch

from . import clq
from .clq import _check, _dt, _elsewhere, _ptr, _stream, _with_stream
from .mx import _INT32, _on_gpu

PAIRS = {"interleaved": 0, "halves": 1}
_P, _I, _L = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_SIGS = {"clq_rope": (_I, [_P, _I, _I, _I, _I, _L, _L, _P, _I, _I, _P, _P, _I, _I, _P, _L, _L, _P])}
EXPORTS = tuple(_SIGS)
_lib = None
# pi to 60 digits: a frequency's fraction of a turn is wanted to 64 bits
_PI = fractions.Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def load():
    """libclq.so with the entry point of rotary positions."""
    global _lib
    if _lib is None:
        lib = clq.load()
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def clq_rope(x, dtype, T, H, D, token_stride, head_stride, positions, ld_positions, axes,
             host_sections, turns, pairs, inverse, out, out_token_stride, out_head_stride, stream):
    return load().clq_rope(x, dtype, T, H, D, token_stride, head_stride, positions, ld_positions,
                           axes, host_sections, turns, pairs, inverse, out, out_token_stride,
                           out_head_stride, stream)


def _turn(f):
    """The frequency f (radians a position) as a fraction of a turn, a signed 64-bit number."""
    n = round(fractions.Fraction(f) / (2 * _PI) * (1 << 64)) & ((1 << 64) - 1)
    return n - (1 << 64) if n >> 63 else n


class Rope:
    """Rotary positions of heads of ``head_dim`` values.

    ``sections``: how many values of a head belong to each axis (even numbers, one to four axes,
    at most head_dim together; the values behind them stay as they are).  Value pair i of an axis
    with d values has the frequency theta^(-2 i / d); ``freqs``: the frequencies of all pairs
    instead, in the order of the axes.  ``pairs``: "interleaved" (values 2 p, 2 p + 1) or "halves"
    (values p, P + p of P pairs in all).  The constructor copies them to ``device`` and waits: not
    under stream capture."""

    def __init__(self, head_dim, sections, theta=10000.0, pairs="interleaved", freqs=None,
                 device="cuda"):
        sections = [int(s) for s in sections]
        if not 1 <= len(sections) <= 4 or any(s < 0 or s % 2 for s in sections):
            raise ValueError("sections are one to four even numbers, got %r" % (sections,))
        if not 2 <= sum(sections) <= head_dim or head_dim > 4096:
            raise ValueError("sections of %d values do not fit a head of %d (at most 4096)"
                             % (sum(sections), head_dim))
        if pairs not in PAIRS:
            raise ValueError("pairs must be one of %s, got %r" % (sorted(PAIRS), pairs))
        if freqs is None:
            if not theta > 0:
                raise ValueError("theta must be positive, got %r" % (theta,))
            freqs = [float(theta) ** (-2.0 * i / d) for d in sections for i in range(d // 2)]
        freqs = [float(f) for f in freqs]
        if len(freqs) != sum(sections) // 2:
            raise ValueError("expected %d frequencies, got %d" % (sum(sections) // 2, len(freqs)))
        if not all(abs(f) < float("inf") for f in freqs):
            raise ValueError("frequencies must be finite")
        self.head_dim, self.sections, self.pairs, self.freqs = head_dim, sections, pairs, freqs
        self.axes = len(sections)
        self.turns = torch.tensor([_turn(f) for f in freqs], dtype=torch.int64).to(device)
        if self.turns.is_cuda:  # whichever stream uses it first
            torch.cuda.current_stream(self.turns.device).synchronize()
        # int32 pairs of each axis, as bytes: a copy of this object has them too, wherever they lie
        self.section_pairs = struct.pack("=%di" % self.axes, *(s // 2 for s in sections))
        self.layout = PAIRS[pairs]

    def __call__(self, x, positions, out=None, inverse=False, stream=None):
        """x [T, H, head_dim] fp16 / bf16 with unit stride in a head (any strides of tokens and
        heads), positions int32 [T, axes] -> x turned, [T, H, head_dim]; ``out``: written there
        (x itself: in place; heads that overlap one another, or others of x, are refused).  ``inverse`` turns back:
        the gradient of x from that of the result."""
        if stream is not None and _elsewhere(stream):
            return _with_stream(stream, self, x, positions, out, inverse)
        host = clq._host or clq._find_host()
        fn = getattr(host, "rope", None) if host else None
        if fn is not None:
            r = fn(x, positions, self.turns, self.section_pairs, self.axes, self.head_dim, self.layout,
                   int(bool(inverse)), out)
            if r is not None:
                if type(r) is int:
                    raise clq.ClqError(r, "clq_rope")
                return r
        if x.dim() != 3 or x.shape[2] != self.head_dim or x.stride(2) != 1:
            raise ValueError("x must have shape [T, H, %d] and unit stride in a head, got %s, strides %s"
                             % (self.head_dim, tuple(x.shape), x.stride()))
        T, H, D = x.shape
        if (positions.dtype != torch.int32 or tuple(positions.shape) != (T, self.axes)
                or (self.axes > 1 and positions.stride(1) != 1)):
            raise ValueError("positions must be int32 of shape (%d, %d) with unit column stride"
                             % (T, self.axes))
        ld = positions.stride(0) if T > 1 else self.axes
        if T > _INT32 or H > _INT32 or ld > _INT32:  # (ctypes would cut them)
            raise ValueError("tokens, heads and the stride of positions are 32-bit numbers, got %d, %d, %d" % (T, H, ld))
        if out is None:
            out = torch.empty((T, H, D), dtype=x.dtype, device=x.device)
        elif (out.shape != x.shape or out.dtype != x.dtype or out.stride(2) != 1
              or (T > 1 and out.stride(0) == 0) or (H > 1 and out.stride(1) == 0)):
            raise ValueError("out must be like x, with unit stride in a head and places of its own for each")
        sections = (ctypes.c_int32 * self.axes).from_buffer_copy(self.section_pairs)
        if self.turns.dtype != torch.int64 or tuple(self.turns.shape) != (sum(sections),) or not self.turns.is_contiguous():
            raise ValueError("turns must be one contiguous int64 a pair, %d of them, got %s %s"
                             % (sum(sections), self.turns.dtype, tuple(self.turns.shape)))
        _on_gpu(x, positions, out, self.turns)
        _check(clq_rope(_ptr(x), _dt(x), T, H, D, x.stride(0), x.stride(1), _ptr(positions),
                        ld, self.axes, sections, _ptr(self.turns),
                        self.layout, int(bool(inverse)), _ptr(out), out.stride(0),
                        out.stride(1), _stream(stream)), "clq_rope")
        return out
