"""Losses whose gradients the pruned all-reduce step takes: output head with cross entropy, output head against a
teacher's top logits, balance loss of a router (include/iwp_loss.h has the formulas).

Like the rest of the binding this only marshals arguments: every step runs in the library's CUDA kernels on torch's
current stream, torch supplies device memory, there is no CPU fallback, and errors are `IwpError` (status codes) or
`TypeError` / `ValueError` (tensors that do not fit the call).  A plan (`HeadLoss`, `ExpertBalance`) owns the
workspace of its calls; like a `Pruner` it serves one stream and one thread at a time.  `check()` reads the status
word that kernels set, e.g. after a target outside the vocabulary.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Any, Optional

from . import binding
from .binding import IWP_ERR_INVALID, IwpError, _check

IWP_F32, IWP_BF16, IWP_F16 = 0, 1, 2
EXPORTS = ["iwp_loss_reset", "iwp_loss_status", "iwp_head_workspace", "iwp_head_loss", "iwp_balance_workspace", "iwp_balance_loss"]

_vp, _i64, _i32, _f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float


class HeadArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("vocab", _i64), ("dim", _i64), ("hidden", _vp), ("hidden_ld", _i64), ("weight", _vp), ("weight_ld", _i64),
        ("targets", _vp), ("ignore_index", _i64), ("top_ids", _vp), ("top_ids_ld", _i64), ("top_logits", _vp), ("top_logits_ld", _i64),
        ("loss", _vp), ("rows", _vp), ("lse", _vp), ("dloss", _vp), ("dloss_rows", _vp), ("dhidden", _vp), ("dhidden_ld", _i64),
        ("dweight", _vp), ("dweight_ld", _i64), ("workspace", _vp), ("workspace_bytes", _i64), ("piece_bytes", _i64),
        ("temperature", _f32), ("scale", _f32), ("dtype", _i32), ("top_k", _i32), ("ids_bytes", _i32), ("top_type", _i32),
        ("dhidden_type", _i32), ("dweight_type", _i32), ("mean", _i32), ("accumulate", _i32), ("have_lse", _i32),
    ]


class BalanceArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("logits", _vp), ("logits_ld", _i64), ("ids", _vp), ("ids_ld", _i64), ("mask", _vp), ("dloss", _vp), ("loss", _vp),
        ("counts", _vp), ("mean_prob", _vp), ("dlogits", _vp), ("dlogits_ld", _i64), ("workspace", _vp), ("workspace_bytes", _i64),
        ("coef", _f32), ("scale", _f32), ("experts", _i32), ("top_k", _i32), ("type", _i32), ("ids_bytes", _i32),
    ]


_ready = False


def lib() -> C.CDLL:
    global _ready
    L = binding.lib()
    if not _ready:
        L.iwp_loss_reset.argtypes = [_vp, _vp]
        L.iwp_loss_status.argtypes = [_vp, _vp, _vp]
        L.iwp_head_workspace.restype, L.iwp_head_workspace.argtypes = _i64, [_vp]
        L.iwp_head_loss.argtypes = [_vp, _vp]
        L.iwp_balance_workspace.restype, L.iwp_balance_workspace.argtypes = _i64, [_vp]
        L.iwp_balance_loss.argtypes = [_vp, _vp]
        _ready = True
    return L


@dataclass
class HeadResult:
    """loss: 0-d, rows and lse: [T], all float32; dhidden / dweight: None where they were not asked for."""

    loss: Any = None
    rows: Any = None
    lse: Any = None
    dhidden: Any = None
    dweight: Any = None


@dataclass
class BalanceResult:
    """loss: 0-d float32, counts: [E] int32, mean_prob: [E] float32, dlogits: [T, E] or None."""

    loss: Any = None
    counts: Any = None
    mean_prob: Any = None
    dlogits: Any = None


def _types():
    import torch

    return torch, {torch.float32: IWP_F32, torch.bfloat16: IWP_BF16, torch.float16: IWP_F16}


def _rows_of(x, name: str, shape, dtypes, device) -> int:
    """Checks a matrix (rows may be strided, columns not) and returns its row stride."""
    if x.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {x.dtype}, expected one of {[str(d) for d in dtypes]}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, expected {device}")
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(x.shape)}, expected {tuple(shape)}")
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError(f"{name}: neighbouring columns must be neighbours in memory")
    if x.shape[0] <= 1:
        return x.shape[1]
    if x.stride(0) < x.shape[1]:
        raise ValueError(f"{name}: rows overlap")
    return x.stride(0)


def _vector(x, name: str, n: int, dtypes, device) -> None:
    if x.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {x.dtype}, expected one of {[str(d) for d in dtypes]}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, expected {device}")
    if x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{name} must hold {n} contiguous elements")


class _Plan:
    def __init__(self):
        torch, self._codes = _types()
        if not torch.cuda.is_available():
            raise RuntimeError("iwp needs a CUDA device; there is no CPU fallback")
        self._torch = torch
        self.device = torch.device("cuda", torch.cuda.current_device())
        lib()
        self._ws = None

    def _stream(self) -> int:
        return self._torch.cuda.current_stream(self.device).cuda_stream

    def _grow(self, need: int) -> None:
        if need < 0:
            raise IwpError(IWP_ERR_INVALID, "workspace size")
        if self._ws is None or self._ws.numel() < need:
            status = 0 if self._ws is None else self.status()
            self._ws = self._torch.empty(need, dtype=self._torch.uint8, device=self.device)
            _check(lib().iwp_loss_reset(self._ws.data_ptr(), self._stream()), "iwp_loss_reset")
            if status:  # a set status word outlives a larger workspace
                self._ws[:4].view(self._torch.int32).fill_(status)

    def status(self) -> int:
        """The status word, after everything enqueued on the current stream."""
        if self._ws is None:
            return 0
        v = C.c_int32()
        _check(lib().iwp_loss_status(self._ws.data_ptr(), C.byref(v), self._stream()), "iwp_loss_status")
        return int(v.value)

    def check(self) -> None:
        _check(self.status(), type(self).__name__)

    def reset(self) -> None:
        if self._ws is not None:
            _check(lib().iwp_loss_reset(self._ws.data_ptr(), self._stream()), "iwp_loss_reset")


class HeadLoss(_Plan):
    """Output head [vocab, dim] with its loss; the logits are never kept.

    tokens: the most rows a call will bring (more are allowed: the workspace then grows once); top_k: the most teacher
    logits per row; piece_bytes: bound on the probabilities held at a time while gradients are formed (0 = 512 MiB)."""

    def __init__(self, tokens: int, vocab: int, dim: int, dtype=None, top_k: int = 1, piece_bytes: int = 0):
        super().__init__()
        t = self._torch
        self.vocab, self.dim, self.dtype, self.piece_bytes = int(vocab), int(dim), dtype or t.bfloat16, int(piece_bytes)
        if self.dtype not in (t.bfloat16, t.float16):
            raise TypeError("HeadLoss takes bfloat16 or float16 operands")
        a = HeadArgs(tokens=int(tokens), vocab=self.vocab, dim=self.dim, dtype=self._codes[self.dtype], top_k=int(top_k),
                     piece_bytes=self.piece_bytes)
        a.hidden_ld = a.weight_ld = (self.dim + 7) // 8 * 8
        a.dhidden = a.dweight = 256
        a.dhidden_ld = a.dweight_ld = self.dim
        a.dhidden_type = a.dweight_type = a.dtype
        if self.dim % 8:  # rows of contiguous operands do not start at multiples of 16 bytes: they will be copied
            a.hidden_ld = a.weight_ld = self.dim
        self._grow(lib().iwp_head_workspace(C.byref(a)))

    # one call of iwp_head_loss
    def _run(self, hidden, weight, a: HeadArgs, *, grad, ignore_index=0, reduction="mean", lse=None, dloss=None, scale=1.0, dhidden=None,
             dweight=None, accumulate=False, want=("hidden", "weight")) -> HeadResult:
        t, dev = self._torch, self.device
        if hidden.dim() != 2 or weight.dim() != 2:
            raise ValueError("hidden and weight are matrices")
        T, two = hidden.shape[0], (self.dtype,)
        a.tokens, a.vocab, a.dim, a.dtype, a.piece_bytes = T, self.vocab, self.dim, self._codes[self.dtype], self.piece_bytes
        a.hidden_ld = _rows_of(hidden, "hidden", (T, self.dim), two, dev)
        a.weight_ld = _rows_of(weight, "weight", (self.vocab, self.dim), two, dev)
        a.hidden, a.weight = hidden.data_ptr(), weight.data_ptr()
        if reduction not in ("mean", "sum"):
            raise ValueError("reduction is 'mean' or 'sum'")
        a.mean, a.ignore_index, a.scale = int(reduction == "mean"), int(ignore_index), float(scale)
        r = HeadResult()
        if lse is None:
            out = t.empty(2 * T + 1, dtype=t.float32, device=dev)
            r.rows, r.lse, r.loss = out[:T], out[T : 2 * T], out[2 * T]
            a.rows, a.lse, a.loss = r.rows.data_ptr(), r.lse.data_ptr(), r.loss.data_ptr()
        else:
            _vector(lse, "lse", T, (t.float32,), dev)
            r.lse, a.lse, a.have_lse = lse, lse.data_ptr(), 1
        if T == 0 and lse is None:
            a.lse = out.data_ptr()
        if grad:
            if dloss is not None:
                if dloss.dim() == 0:
                    _vector(dloss, "dloss", 1, (t.float32,), dev)
                    a.dloss = dloss.data_ptr()
                else:
                    _vector(dloss, "dloss", T, (t.float32,), dev)
                    a.dloss_rows = dloss.data_ptr()
            a.accumulate = int(accumulate)
            for name, given, shape in (("hidden", dhidden, (T, self.dim)), ("weight", dweight, (self.vocab, self.dim))):
                if name not in want:
                    continue
                if given is None:
                    if accumulate:
                        raise ValueError(f"accumulate needs d{name}")
                    given = t.empty(shape, dtype=self.dtype, device=dev)
                ld = _rows_of(given, "d" + name, shape, (self.dtype, t.float32), dev)
                setattr(a, "d" + name, given.data_ptr() or 256)  # an empty tensor has no address
                setattr(a, f"d{name}_ld", ld)
                setattr(a, f"d{name}_type", self._codes[given.dtype])
                setattr(r, "d" + name, given)
        if T == 0:
            a.hidden = a.hidden or 256
            a.targets = a.targets or (256 if not a.top_k else None)
            a.top_ids, a.top_logits = a.top_ids or 256, a.top_logits or 256
            a.lse = a.lse or 256
        L = lib()
        need = L.iwp_head_workspace(C.byref(a))
        if self._ws.numel() < need or need < 0:
            self._grow(need)
        a.workspace, a.workspace_bytes = self._ws.data_ptr(), self._ws.numel()
        _check(L.iwp_head_loss(C.byref(a), self._stream()), "iwp_head_loss")
        return r

    def _hard(self, hidden, targets) -> HeadArgs:
        _vector(targets, "targets", hidden.shape[0], (self._torch.int64,), self.device)
        return HeadArgs(targets=targets.data_ptr(), temperature=1.0)

    def _soft(self, hidden, top_ids, top_logits, temperature) -> HeadArgs:
        t = self._torch
        if top_ids.dim() != 2:
            raise ValueError("top_ids is a matrix")
        shape = (hidden.shape[0], top_ids.shape[1])
        a = HeadArgs(temperature=float(temperature), top_k=shape[1])
        a.top_ids_ld = _rows_of(top_ids, "top_ids", shape, (t.int64, t.int32), self.device)
        a.top_logits_ld = _rows_of(top_logits, "top_logits", shape, tuple(self._codes), self.device)
        a.top_ids, a.top_logits = top_ids.data_ptr(), top_logits.data_ptr()
        a.ids_bytes, a.top_type = (8 if top_ids.dtype == t.int64 else 4), self._codes[top_logits.dtype]
        return a

    def cross_entropy(self, hidden, weight, targets, *, ignore_index: int = -100, reduction: str = "mean") -> HeadResult:
        """Loss of targets[t] under softmax(hidden weight^T): loss, rows and lse."""
        return self._run(hidden, weight, self._hard(hidden, targets), grad=False, ignore_index=ignore_index, reduction=reduction)

    def cross_entropy_grad(self, hidden, weight, targets, *, ignore_index: int = -100, reduction: str = "mean", lse=None, dloss=None,
                           scale: float = 1.0, dhidden=None, dweight=None, accumulate: bool = False,
                           want=("hidden", "weight")) -> HeadResult:
        """The loss and its gradients, times `scale` and the upstream gradient `dloss` (0-d, or one value per row).

        lse: of an earlier forward pass over the same operands; the forward pass is then left out (no loss, no rows).
        dhidden / dweight: where to write (the operands' type or float32, e.g. a view of a worker's row of the
        pruner's gradients); accumulate adds to what they hold.  want: which of the two gradients."""
        return self._run(hidden, weight, self._hard(hidden, targets), grad=True, ignore_index=ignore_index, reduction=reduction, lse=lse,
                         dloss=dloss, scale=scale, dhidden=dhidden, dweight=dweight, accumulate=accumulate, want=want)

    def distill(self, hidden, weight, top_ids, top_logits, temperature: float = 1.0, *, reduction: str = "mean") -> HeadResult:
        """temperature^2 times the divergence of the student's softmax from the teacher's over its top logits."""
        return self._run(hidden, weight, self._soft(hidden, top_ids, top_logits, temperature), grad=False, reduction=reduction)

    def distill_grad(self, hidden, weight, top_ids, top_logits, temperature: float = 1.0, *, reduction: str = "mean", lse=None, dloss=None,
                     scale: float = 1.0, dhidden=None, dweight=None, accumulate: bool = False, want=("hidden", "weight")) -> HeadResult:
        """As cross_entropy_grad, against the teacher; lse is that of the logits divided by the temperature."""
        return self._run(hidden, weight, self._soft(hidden, top_ids, top_logits, temperature), grad=True, reduction=reduction, lse=lse,
                         dloss=dloss, scale=scale, dhidden=dhidden, dweight=dweight, accumulate=accumulate, want=want)


class ExpertBalance(_Plan):
    """Balance loss of a router over `experts` experts; tokens: the most rows a call will bring (more are allowed)."""

    def __init__(self, tokens: int, experts: int):
        super().__init__()
        self.experts = int(experts)
        a = BalanceArgs(tokens=int(tokens), experts=self.experts, top_k=1, type=IWP_F32)
        self._grow(lib().iwp_balance_workspace(C.byref(a)))

    def _run(self, logits, ids, mask, coef, dloss, scale, grad, dlogits) -> BalanceResult:
        t, dev, E = self._torch, self.device, self.experts
        if logits.dim() != 2 or ids.dim() != 2:
            raise ValueError("logits and ids are matrices")
        T, k = logits.shape[0], ids.shape[1]
        a = BalanceArgs(tokens=T, experts=E, top_k=k, coef=float(coef), scale=float(scale))
        a.logits_ld = _rows_of(logits, "logits", (T, E), tuple(self._codes), dev)
        a.ids_ld = _rows_of(ids, "ids", (T, k), (t.int64, t.int32), dev)
        a.logits, a.ids, a.type, a.ids_bytes = logits.data_ptr(), ids.data_ptr(), self._codes[logits.dtype], (8 if ids.dtype == t.int64 else 4)
        if mask is not None:
            _vector(mask, "mask", T, (t.bool, t.uint8), dev)
            a.mask = mask.data_ptr()
        out = t.empty(E + 1, dtype=t.float32, device=dev)
        r = BalanceResult(loss=out[E], mean_prob=out[:E], counts=t.empty(E, dtype=t.int32, device=dev))
        a.loss, a.mean_prob, a.counts = r.loss.data_ptr(), r.mean_prob.data_ptr(), r.counts.data_ptr()
        if grad:
            if dloss is not None:
                _vector(dloss, "dloss", 1, (t.float32,), dev)
                a.dloss = dloss.data_ptr()
            r.dlogits = t.empty((T, E), dtype=logits.dtype, device=dev) if dlogits is None else dlogits
            a.dlogits_ld = _rows_of(r.dlogits, "dlogits", (T, E), (logits.dtype,), dev)
            a.dlogits = r.dlogits.data_ptr()
        if T == 0:
            a.logits, a.ids = a.logits or 256, a.ids or 256
        a.workspace, a.workspace_bytes = self._ws.data_ptr(), self._ws.numel()
        _check(lib().iwp_balance_loss(C.byref(a), self._stream()), "iwp_balance_loss")
        return r

    def loss(self, logits, ids, mask=None, *, coef: float = 0.01) -> BalanceResult:
        """Loss, counts and mean probabilities of router logits [T, E] and chosen experts ids [T, k]."""
        return self._run(logits, ids, mask, coef, None, 1.0, False, None)

    def grad(self, logits, ids, mask=None, *, coef: float = 0.01, dloss=None, scale: float = 1.0, dlogits=None) -> BalanceResult:
        """The same with the gradient to the logits, times `scale` and the upstream gradient `dloss` (0-d)."""
        return self._run(logits, ids, mask, coef, dloss, scale, True, dlogits)
