"""Losses whose gradients the pruned all-reduce step takes: output head with cross entropy, output head against a
teacher's top logits, balance loss of a router (include/iwp_loss.h has the formulas).

Like the rest of the binding this only marshals arguments: every step runs in the library's CUDA kernels on torch's
current stream, torch supplies device memory, there is no CPU fallback, and errors are `IwpError` (status codes) or
`TypeError` / `ValueError` (tensors that do not fit the call).  A plan (`HeadLoss`, `ExpertBalance`) owns the
workspace of its calls; like a `Pruner` it serves one stream and one thread at a time.  `check()` reads the status
word that kernels set, e.g. after a target outside the vocabulary.

Calls may be captured in a CUDA graph (a plan is made before the capture, and kept as long as the graph, which works in
its workspace): from its first capture on, a plan keeps every workspace that it outgrows, for the graphs' sake.
"""
from __future__ import annotations

import ctypes as C

from . import binding
from .binding import IWP_ERR_CAPACITY, IWP_ERR_INVALID, IwpError, _check

IWP_F32, IWP_BF16, IWP_F16 = 0, 1, 2
LOSS_STATE = 256
EXPORTS = ["iwp_loss_reset", "iwp_loss_status", "iwp_head_workspace", "iwp_head_loss", "iwp_balance_workspace", "iwp_balance_loss"]

_vp, _i64, _i32, _f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float


class HeadArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("vocab", _i64), ("dim", _i64), ("hidden", _vp), ("hidden_ld", _i64), ("weight", _vp), ("weight_ld", _i64),
        ("targets", _vp), ("ignore_index", _i64), ("top_ids", _vp), ("top_ids_ld", _i64), ("top_logits", _vp), ("top_logits_ld", _i64),
        ("loss", _vp), ("rows", _vp), ("lse", _vp), ("dloss", _vp), ("dloss_rows", _vp), ("dhidden", _vp), ("dhidden_ld", _i64),
        ("dweight", _vp), ("dweight_ld", _i64), ("workspace", _vp), ("workspace_bytes", _i64), ("state", _vp), ("piece_bytes", _i64),
        ("temperature", _f32), ("scale", _f32), ("dtype", _i32), ("top_k", _i32), ("ids_bytes", _i32), ("top_type", _i32),
        ("dhidden_type", _i32), ("dweight_type", _i32), ("mean", _i32), ("accumulate", _i32), ("have_lse", _i32),
    ]


class BalanceArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("logits", _vp), ("logits_ld", _i64), ("ids", _vp), ("ids_ld", _i64), ("mask", _vp), ("dloss", _vp), ("loss", _vp),
        ("counts", _vp), ("mean_prob", _vp), ("dlogits", _vp), ("dlogits_ld", _i64), ("workspace", _vp), ("workspace_bytes", _i64),
        ("state", _vp),
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


class HeadResult:
    """loss: 0-d, rows and lse: [T], all float32 (None where no forward pass was made, lse then as given); dhidden /
    dweight: None where they were not asked for."""

    __slots__ = ("_out", "_lse", "_tokens", "dhidden", "dweight")

    def __init__(self, out, lse, tokens):
        self._out, self._lse, self._tokens, self.dhidden, self.dweight = out, lse, tokens, None, None

    @property
    def loss(self):
        return None if self._out is None else self._out[-1]

    @property
    def rows(self):
        return None if self._out is None else self._out[: self._tokens]

    @property
    def lse(self):
        return self._lse if self._out is None else self._out[self._tokens : -1]


class BalanceResult:
    """loss: 0-d float32, counts: [E] int32, mean_prob: [E] float32, dlogits: [T, E] or None."""

    __slots__ = ("_out", "counts", "dlogits")

    def __init__(self, out, counts, dlogits):
        self._out, self.counts, self.dlogits = out, counts, dlogits

    @property
    def loss(self):
        return self._out[-1]

    @property
    def mean_prob(self):
        return self._out[:-1]


def _types():
    import torch

    return torch, {torch.float32: IWP_F32, torch.bfloat16: IWP_BF16, torch.float16: IWP_F16}


def _bad(x, name: str, shape, dtypes, device):
    if x.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {x.dtype}, expected one of {[str(d) for d in dtypes]}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, expected {device}")
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(x.shape)}, expected {tuple(shape)}")


def _rows_of(x, name: str, shape, dtypes, device) -> int:
    """Checks a matrix (rows may be strided, columns not) and returns its row stride."""
    if x.dtype not in dtypes or x.shape != shape or x.device != device:
        _bad(x, name, shape, dtypes, device)
    ld, step = x.stride()
    rows, cols = shape
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: neighbouring columns must be neighbours in memory")
    if rows <= 1:
        return cols
    if ld < cols:
        raise ValueError(f"{name}: rows overlap")
    return ld


def _vector(x, name: str, n: int, dtypes, device) -> None:
    if x.dtype not in dtypes or x.device != device:
        _bad(x, name, x.shape, dtypes, device)
    if x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{name} must hold {n} contiguous elements")


class _Plan:
    """What plans share: the state and the workspace of their calls, and the streams these are used on."""

    _state_bytes, _reset_entry = LOSS_STATE, "iwp_loss_reset"

    def __init__(self):
        torch, self._codes = _types()
        if not torch.cuda.is_available():
            raise RuntimeError("iwp needs a CUDA device; there is no CPU fallback")
        self._torch = torch
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._lib = lib()
        self._capturing = torch._C._cuda_isCurrentStreamCapturing
        if self._capturing():
            raise RuntimeError(f"make the {type(self).__name__} before the capture: its state is zeroed once, not by every replay")
        self._ws, self._ws_at, self._ws_bytes = None, None, 0  # made by the first call
        self._planned = 0
        self._captured, self._outgrown = False, []
        self._floats = tuple(self._codes)
        self._ids = (torch.int64, torch.int32)
        self._raw_stream = torch._C._cuda_getCurrentRawStream  # current_stream() without the object around it
        self._state = torch.empty(self._state_bytes, dtype=torch.uint8, device=self.device)
        self._index = self.device.index
        self._state_at, self._last = self._state.data_ptr(), self._raw_stream(self._index)
        _check(getattr(self._lib, self._reset_entry)(self._state_at, self._last), self._reset_entry)
        self._made = torch.cuda.Event()
        self._made.record()

    def _stream(self) -> int:
        """The stream of this call."""
        s = self._raw_stream(self._index)
        if s != self._last and not self._capturing():
            # another stream than last time: behind the state's zeroing, and no memory of the plan's goes back to the
            # allocator before that stream is done with it
            now = self._torch.cuda.current_stream(self.device)
            now.wait_event(self._made)
            for x in self._memory():
                if x is not None:
                    x.record_stream(now)
            self._last = s
        return s

    def _memory(self):
        return self._state, self._ws

    def _plan(self, need: int) -> None:
        if need < 0:
            raise IwpError(IWP_ERR_INVALID, "workspace size")
        self._planned = need

    def _grow(self, need: int) -> None:
        if need < 0:
            raise IwpError(IWP_ERR_INVALID, "workspace size")
        need = max(need, self._planned)
        if self._ws_bytes < need:
            old, self._ws = self._ws, self._torch.empty(need, dtype=self._torch.uint8, device=self.device)
            self._ws_at, self._ws_bytes = self._ws.data_ptr(), need
            if self._captured and old is not None:
                self._outgrown.append(old)

    def status(self) -> int:
        """The status word, after everything enqueued on the current stream."""
        v = C.c_int32()
        _check(lib().iwp_loss_status(self._state_at, C.byref(v), self._stream()), "iwp_loss_status")
        return int(v.value)

    def check(self) -> None:
        _check(self.status(), type(self).__name__)

    def reset(self) -> None:
        _check(getattr(self._lib, self._reset_entry)(self._state_at, self._stream()), self._reset_entry)


class HeadLoss(_Plan):
    """Output head [vocab, dim] with its loss.  Forward passes keep no logits; gradients hold the probabilities of a piece of
    the vocabulary in 16 bits while they are formed, of all of it where `piece_bytes` allows.

    tokens: the most rows a call will bring; top_k: the most teacher logits per row.  The first call makes a workspace
    that serves forward passes of that size; the first gradient (or a call that needs more) makes a larger one.
    piece_bytes: bound on the probabilities held at a time (0 = 1 GiB, or 4 vocab dim bytes, what the weights and their
    gradient take, where that is more).  A plan that has formed gradients keeps a workspace of that, the partial sums
    (78 MB or more) and copies of the hidden states."""

    def __init__(self, tokens: int, vocab: int, dim: int, dtype=None, top_k: int = 1, piece_bytes: int = 0):
        super().__init__()
        t = self._torch
        self.vocab, self.dim, self.dtype, self.piece_bytes = int(vocab), int(dim), dtype or t.bfloat16, int(piece_bytes)
        if self.dtype not in (t.bfloat16, t.float16):
            raise TypeError("HeadLoss takes bfloat16 or float16 operands")
        self._code, self._two, self._out_types = self._codes[self.dtype], (self.dtype,), (self.dtype, t.float32)
        a = HeadArgs(tokens=int(tokens), vocab=self.vocab, dim=self.dim, dtype=self._codes[self.dtype], top_k=int(top_k),
                     piece_bytes=self.piece_bytes)
        a.hidden_ld = a.weight_ld = (self.dim + 7) // 8 * 8
        if self.dim % 8:  # rows of contiguous operands do not start at multiples of 16 bytes: they will be copied
            a.hidden_ld = a.weight_ld = self.dim
        self._plan(lib().iwp_head_workspace(C.byref(a)))

    # one call of iwp_head_loss
    def _run(self, hidden, weight, a: HeadArgs, *, grad, ignore_index=0, reduction="mean", lse=None, dloss=None, scale=1.0, dhidden=None,
             dweight=None, accumulate=False, want=("hidden", "weight")) -> HeadResult:
        t, dev, V, D = self._torch, self.device, self.vocab, self.dim
        if hidden.dim() != 2:
            raise ValueError("hidden is a matrix")
        T, two = hidden.shape[0], self._two
        a.tokens, a.vocab, a.dim, a.dtype, a.piece_bytes = T, V, D, self._code, self.piece_bytes
        a.hidden_ld = _rows_of(hidden, "hidden", (T, D), two, dev)
        a.weight_ld = _rows_of(weight, "weight", (V, D), two, dev)
        a.hidden, a.weight = hidden.data_ptr(), weight.data_ptr()
        if reduction == "mean":
            a.mean = 1
        elif reduction != "sum":
            raise ValueError("reduction is 'mean' or 'sum'")
        a.ignore_index = ignore_index
        if lse is None:
            out = t.empty(2 * T + 1, dtype=t.float32, device=dev)
            r = HeadResult(out, None, T)
            at = out.data_ptr()
            a.rows, a.lse, a.loss = at, at + 4 * T, at + 8 * T
        else:
            _vector(lse, "lse", T, (t.float32,), dev)
            r = HeadResult(None, lse, T)
            a.lse, a.have_lse = lse.data_ptr() or 256, 1
        if grad:
            a.scale = scale
            if dloss is not None:
                if dloss.dim() == 0:
                    _vector(dloss, "dloss", 1, (t.float32,), dev)
                    a.dloss = dloss.data_ptr()
                else:
                    _vector(dloss, "dloss", T, (t.float32,), dev)
                    a.dloss_rows = dloss.data_ptr()
            if accumulate:
                a.accumulate = 1
                if ("hidden" in want and dhidden is None) or ("weight" in want and dweight is None):
                    raise ValueError("accumulate needs the gradients to add to")
            if "hidden" in want:
                if dhidden is None:
                    dhidden, a.dhidden_ld, a.dhidden_type = t.empty(T, D, dtype=self.dtype, device=dev), D, self._code
                else:
                    a.dhidden_ld, a.dhidden_type = _rows_of(dhidden, "dhidden", (T, D), self._out_types, dev), self._codes[dhidden.dtype]
                a.dhidden = dhidden.data_ptr() or 256  # an empty tensor has no address
                r.dhidden = dhidden
            if "weight" in want:
                if dweight is None:
                    dweight, a.dweight_ld, a.dweight_type = t.empty(V, D, dtype=self.dtype, device=dev), D, self._code
                else:
                    a.dweight_ld, a.dweight_type = _rows_of(dweight, "dweight", (V, D), self._out_types, dev), self._codes[dweight.dtype]
                a.dweight = dweight.data_ptr()
                r.dweight = dweight
        if T == 0:
            a.hidden = a.hidden or 256
            if a.top_k:
                a.top_ids, a.top_logits = a.top_ids or 256, a.top_logits or 256
            else:
                a.targets = a.targets or 256
        ref, stream = C.byref(a), self._stream()
        if self._capturing():
            self._captured = True
        if self._ws_at is None:
            self._grow(self._lib.iwp_head_workspace(ref))
        a.workspace, a.workspace_bytes, a.state = self._ws_at, self._ws_bytes, self._state_at
        status = self._lib.iwp_head_loss(ref, stream)
        if status == IWP_ERR_CAPACITY:  # more tokens, or rows that have to be copied, for the first time
            self._grow(self._lib.iwp_head_workspace(ref))
            a.workspace, a.workspace_bytes = self._ws_at, self._ws_bytes
            status = self._lib.iwp_head_loss(ref, stream)
        if status:
            raise IwpError(status, "iwp_head_loss")
        return r

    def _hard(self, hidden, targets) -> HeadArgs:
        _vector(targets, "targets", hidden.shape[0], self._ids[:1], self.device)
        a = HeadArgs()
        a.targets, a.temperature = targets.data_ptr(), 1.0
        return a

    def _soft(self, hidden, top_ids, top_logits, temperature) -> HeadArgs:
        if top_ids.dim() != 2:
            raise ValueError("top_ids is a matrix")
        shape = (hidden.shape[0], top_ids.shape[1])
        a = HeadArgs()
        a.temperature, a.top_k = temperature, shape[1]
        a.top_ids_ld = _rows_of(top_ids, "top_ids", shape, self._ids, self.device)
        a.top_logits_ld = _rows_of(top_logits, "top_logits", shape, self._floats, self.device)
        a.top_ids, a.top_logits = top_ids.data_ptr(), top_logits.data_ptr()
        a.ids_bytes, a.top_type = (8 if top_ids.dtype is self._ids[0] else 4), self._codes[top_logits.dtype]
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
        self._masks = (self._torch.bool, self._torch.uint8)
        self._args = a = BalanceArgs(tokens=int(tokens), experts=self.experts, top_k=1, type=IWP_F32)  # of every call
        self._args_at = C.addressof(a)
        self._plan(lib().iwp_balance_workspace(C.byref(a)))

    def _run(self, logits, ids, mask, coef, dloss, scale, grad, dlogits) -> BalanceResult:
        t, dev, E, a = self._torch, self.device, self.experts, self._args
        if logits.dim() != 2 or ids.dim() != 2:
            raise ValueError("logits and ids are matrices")
        T, k = logits.shape[0], ids.shape[1]
        a.tokens, a.top_k, a.coef, a.scale = T, k, coef, scale
        a.logits_ld = ld = _rows_of(logits, "logits", (T, E), self._floats, dev)
        a.ids_ld = _rows_of(ids, "ids", (T, k), self._ids, dev)
        a.logits, a.ids, a.type, a.ids_bytes = logits.data_ptr(), ids.data_ptr(), self._codes[logits.dtype], (8 if ids.dtype is self._ids[0] else 4)
        if mask is None:
            a.mask = None
        else:
            _vector(mask, "mask", T, self._masks, dev)
            a.mask = mask.data_ptr()
        out = t.empty(E + 1, dtype=t.float32, device=dev)
        counts = t.empty(E, dtype=t.int32, device=dev)
        at = out.data_ptr()
        a.mean_prob, a.loss, a.counts, a.dloss = at, at + 4 * E, counts.data_ptr(), None
        if grad:
            if dloss is not None:
                _vector(dloss, "dloss", 1, self._floats[:1], dev)
                a.dloss = dloss.data_ptr()
            if dlogits is None:
                dlogits = t.empty_like(logits) if ld == E and T > 1 else t.empty(T, E, dtype=logits.dtype, device=dev)
                a.dlogits_ld = E
            else:
                a.dlogits_ld = _rows_of(dlogits, "dlogits", (T, E), (logits.dtype,), dev)
            a.dlogits = dlogits.data_ptr()
        else:
            a.dlogits = None
        if T == 0:
            a.logits, a.ids = a.logits or 256, a.ids or 256
        stream = self._stream()
        if self._ws_at is None:
            self._grow(0)
            a.workspace, a.workspace_bytes, a.state = self._ws_at, self._ws_bytes, self._state_at
        status = self._lib.iwp_balance_loss(self._args_at, stream)
        if status:
            raise IwpError(status, "iwp_balance_loss")
        return BalanceResult(out, counts, dlogits)

    def loss(self, logits, ids, mask=None, *, coef: float = 0.01) -> BalanceResult:
        """Loss, counts and mean probabilities of router logits [T, E] and chosen experts ids [T, k]."""
        return self._run(logits, ids, mask, coef, None, 1.0, False, None)

    def grad(self, logits, ids, mask=None, *, coef: float = 0.01, dloss=None, scale: float = 1.0, dlogits=None) -> BalanceResult:
        """The same with the gradient to the logits, times `scale` and the upstream gradient `dloss` (0-d)."""
        return self._run(logits, ids, mask, coef, dloss, scale, True, dlogits)


# ---- differentiable forms (once: a second derivative is refused) --------------------------------------


def _once():
    """The autograd.Function that refuses second derivatives, made on first use (importing this module does not import torch)."""
    global _refuses
    if _refuses is None:
        import torch

        class Once(torch.autograd.Function):
            """make(): gradients that depend on `inputs`.  Under create_graph a derivative of them is asked for only if
            they are differentiated again, and is refused then (they would pass for constants otherwise)."""

            @staticmethod
            def forward(ctx, make, *inputs):
                return make()

            @staticmethod
            def backward(ctx, *_):
                raise RuntimeError("these gradients come from kernels and cannot be differentiated again")

        _refuses = Once
    return _refuses


_refuses = None


def _functions():
    """autograd.Function classes around the plans, made on first use."""
    global _autograd
    if _autograd is None:
        import torch

        Once = _once()

        class Head(torch.autograd.Function):
            @staticmethod
            def forward(ctx, hidden, weight, plan, kind, args, kwargs):
                r = getattr(plan, kind)(hidden, weight, *args, **kwargs)
                tensors = [a for a in args if isinstance(a, torch.Tensor)]  # they come first
                ctx.plan, ctx.kind, ctx.rest, ctx.kwargs = plan, kind, args[len(tensors) :], kwargs
                ctx.save_for_backward(hidden, weight, r.lse, *tensors)
                return r.loss.clone()

            @staticmethod
            def backward(ctx, dloss):
                hidden, weight, lse, *tensors = ctx.saved_tensors
                want = tuple(n for n, need in zip(("hidden", "weight"), ctx.needs_input_grad) if need)
                grad = getattr(ctx.plan, ctx.kind + "_grad")

                def make():
                    r = grad(hidden, weight, *tensors, *ctx.rest, lse=lse, dloss=dloss.float(), want=want, **ctx.kwargs)
                    return r.dhidden, r.dweight

                return *Once.apply(make, hidden, weight, dloss), None, None, None, None

        class Balance(torch.autograd.Function):
            @staticmethod
            def forward(ctx, logits, plan, ids, mask, coef):
                ctx.plan, ctx.coef = plan, coef
                ctx.save_for_backward(logits, ids, mask)
                r = plan.loss(logits, ids, mask, coef=coef)
                ctx.mark_non_differentiable(r.counts)
                return r.loss.clone(), r.counts

            @staticmethod
            def backward(ctx, dloss, _):
                logits, ids, mask = ctx.saved_tensors
                make = lambda: ctx.plan.grad(logits, ids, mask, coef=ctx.coef, dloss=dloss.float()).dlogits  # noqa: E731
                return Once.apply(make, logits, dloss), None, None, None, None

        _autograd = (Head, Balance)
    return _autograd


_autograd = None


def cross_entropy(plan: HeadLoss, hidden, weight, targets, **kwargs):
    """The loss of plan.cross_entropy as a differentiable function of hidden and weight.  Only lse is kept for the
    backward pass, which forms the probabilities anew, piece by piece."""
    return _functions()[0].apply(hidden, weight, plan, "cross_entropy", (targets,), kwargs)


def distill(plan: HeadLoss, hidden, weight, top_ids, top_logits, temperature: float = 1.0, **kwargs):
    """The loss of plan.distill as a differentiable function of hidden and weight (not of the teacher's logits)."""
    return _functions()[0].apply(hidden, weight, plan, "distill", (top_ids, top_logits, temperature), kwargs)


def balance(plan: ExpertBalance, logits, ids, mask=None, coef: float = 0.01):
    """(loss, counts) of plan.loss, the loss a differentiable function of the router's logits."""
    return _functions()[1].apply(logits, plan, ids, mask, coef)
