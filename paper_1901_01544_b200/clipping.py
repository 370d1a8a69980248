"""Norms and clipping of gradient tensors on their way into the pruned all-reduce step (include/iwp_clip.h has the formulas).

Like the rest of the binding this only marshals arguments: every step runs in the library's CUDA kernels on torch's current
stream, there is no CPU fallback, and errors are `IwpError` (status codes) or `TypeError` / `ValueError` (tensors that do not
fit).  A `GradientClip` is made for the tensors that a program's gradients are kept in, holds them, and lays out once where they are; it is
used as the plans of `losses` are: one stream and one thread at a time, made before a CUDA graph is captured and kept as
long as the graph.
"""
from __future__ import annotations

import ctypes as C
import itertools
from typing import Optional, Sequence

from . import losses
from .binding import IwpError, _check
from .routing import _Here

EXPORTS = ["iwp_clip_layout", "iwp_clip_table", "iwp_clip"]

_vp, _i64, _i32, _f64 = C.c_void_p, C.c_int64, C.c_int32, C.c_double


class ClipTensor(C.Structure):
    _fields_ = [("in_", _vp), ("out", _vp), ("rows", _i64), ("cols", _i64), ("in_ld", _i64), ("out_ld", _i64), ("group", _i32), ("in_type", _i32),
                ("out_type", _i32)]


class ClipSizes(C.Structure):
    _fields_ = [("table_bytes", _i64), ("workspace_bytes", _i64), ("parts", _i64), ("warps", _i64), ("range", _i64)]


class ClipArgs(C.Structure):
    _fields_ = [
        ("table", _vp), ("parts", _i64), ("warps", _i64), ("squares", _vp), ("norms", _vp), ("factors", _vp), ("workspace", _vp),
        ("workspace_bytes", _i64), ("state", _vp), ("max_norm", _f64), ("scale", _f64), ("groups", _i32), ("write", _i32), ("have_squares", _i32),
        ("drop_nonfinite", _i32),
    ]


_ready = False


def lib() -> C.CDLL:
    global _ready
    L = losses.lib()
    if not _ready:
        L.iwp_clip_layout.argtypes = [_vp, _i64, _i32, _vp]
        L.iwp_clip_table.argtypes = [_vp, _i64, _i32, _vp, _i64]
        L.iwp_clip.argtypes = [_vp, _vp]
        _ready = True
    return L


class ClipResult:
    """norms and factors: [groups] float32; squares: [groups] float64, the sums of squares before `scale`."""

    __slots__ = ("_out", "_groups", "squares")

    def __init__(self, out, groups, squares):
        self._out, self._groups, self.squares = out, groups, squares

    @property
    def norms(self):
        return self._out[: self._groups]

    @property
    def factors(self):
        return self._out[self._groups :]


def _runs(shape, strides) -> list:
    """The tensor as matrices: (first element of each operand, rows, cols, row strides).  strides: of each operand, by dimension;
    dimensions are put in the order of the first one's strides (broadcast ones outermost) and merged where all operands allow it."""
    dims = sorted(((n, s) for n, s in zip(shape, zip(*strides)) if n != 1), key=lambda d: (d[1][0] > 0, -d[1][0]))
    merged: list = []
    for n, s in dims:
        if merged and all(a == n * b for a, b in zip(merged[-1][1], s)):
            merged[-1] = (merged[-1][0] * n, s)
        else:
            merged.append((n, s))
    one = tuple(0 for _ in strides)
    if not merged:
        return [(one, 1, 1, one)]
    if any(s != 1 for s in merged[-1][1]):
        raise ValueError("elements that follow one another in a gradient must be neighbours in memory, and in its output the same way")
    cols = merged.pop()[0]
    if not merged:
        return [(one, 1, cols, one)]
    rows, ld = merged.pop()
    outer = 1
    for n, _ in merged:
        outer *= n
    if outer > 65536:
        raise ValueError("a gradient of too many strided dimensions: make it contiguous")
    return [(tuple(sum(i * s[o] for i, (_, s) in zip(at, merged)) for o in range(len(strides))), rows, cols, ld)
            for at in itertools.product(*(range(n) for n, _ in merged))]


def _spans(entries, field: str, sizes) -> list:
    """(first byte, end) of every run of memory of these entries; of whole matrices where rows are many."""
    out = []
    for e in entries:
        at, ld, size = getattr(e, field), getattr(e, "in_ld" if field == "in_" else "out_ld"), sizes[e.in_type if field == "in_" else e.out_type]
        if e.rows == 1 or ld <= e.cols:
            out.append((at, at + ((e.rows - 1) * ld + e.cols) * size))
        else:
            out += [(at + r * ld * size, at + (r * ld + e.cols) * size) for r in range(e.rows)]
    return out


class GradientClip(_Here):
    """Norms and clipping of `tensors` (float32, bfloat16, float16, in any mixture), in groups with a norm each.

    into: tensors of the same shapes that the clipped gradients are written to, of any of the three types, such as views of a
    worker's row of the pruner's gradients; None: gradients are clipped where they are.  groups: the group of each tensor, 0, 1, ...
    (all in one if None).  Tensors may be strided as long as runs of neighbouring elements remain."""

    def __init__(self, tensors: Sequence, into: Optional[Sequence] = None, groups: Optional[Sequence[int]] = None):
        L = lib()
        super().__init__()
        t = self._torch
        self._tensors = list(tensors)
        self._into = self._tensors if into is None else list(into)
        which = [0] * len(self._tensors) if groups is None else [int(g) for g in groups]
        if len(self._into) != len(self._tensors) or len(which) != len(self._tensors):
            raise ValueError("as many outputs and groups as tensors")
        self.groups = 1 + max(which, default=0)
        entries = []
        for i, (x, y, g) in enumerate(zip(self._tensors, self._into, which)):
            for name, z in ((f"tensors[{i}]", x), (f"into[{i}]", y)):
                if z.dtype not in self._codes:
                    raise TypeError(f"{name} has dtype {z.dtype}, expected one of {[str(d) for d in self._floats]}")
                if z.device != self.device or z.shape != x.shape:
                    raise ValueError(f"{name} is {tuple(z.shape)} on {z.device}, expected {tuple(x.shape)} on {self.device}")
            if x.numel() == 0:
                continue
            a, b, at_x, at_y = self._codes[x.dtype], self._codes[y.dtype], x.data_ptr(), y.data_ptr()
            if x.is_contiguous() and y.is_contiguous():
                entries.append(ClipTensor(at_x, at_y, 1, x.numel(), 0, 0, g, a, b))
                continue
            for (fx, fy), rows, cols, (lx, ly) in _runs(tuple(x.shape), (x.stride(), y.stride())):
                entries.append(ClipTensor(at_x + fx * x.element_size(), at_y + fy * y.element_size(), rows, cols, lx, ly, g, a, b))
        if any(g < 0 for g in which):
            raise ValueError("groups are 0, 1, ...")
        self._writable = self._apart(entries)
        if into is not None and not self._writable:
            raise ValueError("an output overlaps another one or a gradient")
        if not self._writable:
            for e in entries:
                e.out = None
        table = (ClipTensor * max(1, len(entries)))(*entries)
        sizes = ClipSizes()
        _check(L.iwp_clip_layout(table, len(entries), self.groups, C.byref(sizes)), "iwp_clip_layout")
        host = t.empty(sizes.table_bytes, dtype=t.uint8)
        _check(L.iwp_clip_table(table, len(entries), self.groups, host.data_ptr(), sizes.table_bytes), "iwp_clip_table")
        self._table = host.to(self.device)
        self._made.record()  # the table is there, too
        self._planned = sizes.workspace_bytes
        self._args = ClipArgs(table=self._table.data_ptr(), parts=sizes.parts, warps=sizes.warps, state=self._state_at, groups=self.groups)
        self._args_at = C.addressof(self._args)

    def _memory(self):
        return self._state, self._ws, self._table

    @staticmethod
    def _apart(entries) -> bool:
        """Whether every output is apart from all others and from all gradients but its own."""
        sizes = {losses.IWP_F32: 4, losses.IWP_BF16: 2, losses.IWP_F16: 2}
        own = [e.in_ == e.out and e.in_type == e.out_type and (e.rows == 1 or e.in_ld == e.out_ld) for e in entries]
        if any(e.rows > 1 and e.out_ld < e.cols for e in entries):
            return False
        outs = sorted(_spans(entries, "out", sizes))
        if any(a[1] > b[0] for a, b in zip(outs, outs[1:])):
            return False
        ins = _spans([e for e, o in zip(entries, own) if not o], "in_", sizes)
        both = sorted([(a, b, 1) for a, b in outs] + [(a, b, 0) for a, b in ins])
        end = [0, 0]  # of the inputs and of the outputs so far
        for a, b, kind in both:
            if a < end[1 - kind]:
                return False
            end[kind] = max(end[kind], b)
        return True

    def _run(self, max_norm, scale, write, squares, drop) -> ClipResult:
        t, dev, G, a = self._torch, self.device, self.groups, self._args
        out = t.empty(2 * G, dtype=t.float32, device=dev)
        if squares is None:
            squares = t.empty(G, dtype=t.float64, device=dev)
            a.have_squares = 0
        else:
            losses._vector(squares, "squares", G, (t.float64,), dev)
            a.have_squares = 1
        at = out.data_ptr()
        a.norms, a.factors, a.squares = at, at + 4 * G, squares.data_ptr()
        a.max_norm, a.scale, a.write, a.drop_nonfinite = max_norm, scale, write, int(drop)
        stream = self._stream()
        if self._capturing():
            self._captured = True
        if self._ws_at is None:
            self._grow(0)
            a.workspace, a.workspace_bytes = self._ws_at, self._ws_bytes
        status = self._lib.iwp_clip(self._args_at, stream)
        if status:
            raise IwpError(status, "iwp_clip")
        return ClipResult(out, G, squares)

    def norm(self, *, scale: float = 1.0) -> ClipResult:
        """The groups' norms, times |scale|; nothing is written to the tensors."""
        return self._run(float("inf"), scale, 0, None, False)

    def clip(self, max_norm: float, *, scale: float = 1.0, squares=None, drop_nonfinite: bool = False) -> ClipResult:
        """Writes every tensor times its group's factor: `scale` (the inverse of a loss's scaling, say), and as much less as
        brings a norm above max_norm down to it.

        squares: sums of squares to take instead of the tensors' own, e.g. of a `norm` on each rank, added up over the ranks.
        drop_nonfinite: a group that holds a NaN or an infinity is written as zeros (it is left unclipped otherwise)."""
        if not self._writable:
            raise ValueError("gradients that overlap one another cannot be clipped where they are")
        return self._run(max_norm, scale, 1, squares, drop_nonfinite)
