"""A router over experts: the choice of experts with its weights and their gradient (`ExpertRouter`), and rows exchanged
between tokens and experts (`ExpertExchange`).  include/iwp_route.h has the formulas; `losses.ExpertBalance` takes the ids.

Like the rest of the binding this only marshals arguments: every step runs in the library's CUDA kernels on torch's current
stream, there is no CPU fallback, and errors are `IwpError` (status codes) or `TypeError` / `ValueError` (tensors that do not
fit the call).  Plans are used as those of `losses`: one stream and one thread at a time, made before a CUDA graph is
captured and kept as long as the graph.  The differentiable forms can be captured with their backward pass, as torch's own
operators can: nothing of an earlier eager backward graph of the same leaves may be left then.  The plans' `check` has
nothing to report: what cannot be chosen is in the outputs.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

from . import binding, losses
from .binding import IwpError
from .losses import _Plan, _rows_of, _vector

ROUTE_STATE = 256 + 4096
IWP_SOFTMAX, IWP_SIGMOID = 0, 1
EXPORTS = ["iwp_route_reset", "iwp_route", "iwp_route_grad", "iwp_order_workspace", "iwp_order", "iwp_dispatch", "iwp_combine",
           "iwp_combine_grad"]

_vp, _i64, _i32, _f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float


class RouteArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("logits", _vp), ("logits_ld", _i64), ("bias", _vp), ("mask", _vp), ("ids", _vp), ("weights", _vp), ("counts", _vp),
        ("state", _vp), ("weight_scale", _f32), ("experts", _i32), ("top_k", _i32), ("groups", _i32), ("top_groups", _i32), ("group_top", _i32),
        ("score", _i32), ("renormalize", _i32), ("type", _i32), ("ids_bytes", _i32),
    ]


class RouteGradArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("logits", _vp), ("logits_ld", _i64), ("ids", _vp), ("ids_ld", _i64), ("weights", _vp), ("weights_ld", _i64),
        ("dweights", _vp), ("dweights_ld", _i64), ("dlogits", _vp), ("dlogits_ld", _i64), ("weight_scale", _f32), ("scale", _f32),
        ("experts", _i32), ("top_k", _i32), ("score", _i32), ("renormalize", _i32), ("type", _i32), ("ids_bytes", _i32), ("accumulate", _i32),
    ]


class OrderArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("ids", _vp), ("ids_ld", _i64), ("offsets", _vp), ("slots", _vp), ("rows", _vp), ("workspace", _vp),
        ("workspace_bytes", _i64), ("experts", _i32), ("top_k", _i32), ("ids_bytes", _i32),
    ]


class ExchangeArgs(C.Structure):
    _fields_ = [
        ("tokens", _i64), ("dim", _i64), ("slots", _vp), ("offsets", _vp), ("by_token", _vp), ("by_token_ld", _i64), ("by_slot", _vp),
        ("by_slot_ld", _i64), ("weights", _vp), ("weights_ld", _i64), ("by_token_out", _vp), ("by_token_out_ld", _i64), ("by_slot_out", _vp),
        ("by_slot_out_ld", _i64), ("dweights", _vp), ("experts", _i32), ("top_k", _i32), ("type", _i32),
    ]


_ready = False


def lib() -> C.CDLL:
    global _ready
    L = losses.lib()
    if not _ready:
        L.iwp_route_reset.argtypes = [_vp, _vp]
        L.iwp_order_workspace.restype, L.iwp_order_workspace.argtypes = _i64, [_vp]
        for name in ("iwp_route", "iwp_route_grad", "iwp_order", "iwp_dispatch", "iwp_combine", "iwp_combine_grad"):
            getattr(L, name).argtypes = [_vp, _vp]
        _ready = True
    return L


class Route(NamedTuple):
    """ids: [T, k] (-1: no expert), weights: [T, k] float32, counts: [E] int32."""

    ids: object
    weights: object
    counts: object


class Order(NamedTuple):
    """offsets: [E + 1], slots: [T, k] (-1: none), rows: [T k] (token of each slot, -1 behind the last), all int32."""

    offsets: object
    slots: object
    rows: object


_UNKNOWN = (None,) * 7


class _Made(Order):
    """An order as a plan has made it: the plan, tokens and choices, the shape of the slots, where slots and offsets are, and the
    slots' version (None in inference mode).  What is made of it (`_replace`, copies) is an order like any other."""

    made = _UNKNOWN

    @classmethod
    def _make(cls, tensors):
        return Order(*tensors)

    def __reduce_ex__(self, protocol):
        return Order, tuple(self)


def _made(tensors, made) -> _Made:
    order = _Made(*tensors)
    order.made = made
    return order


class _Here(_Plan):
    """A plan whose calls are refused while another device than its own is current."""

    def __init__(self):
        super().__init__()
        self._current = self._torch._C._cuda_getDevice

    def _stream(self) -> int:
        if self._current() != self._index:
            raise ValueError(f"the plan is on {self.device}, which is not the current device")
        s = self._raw_stream(self._index)
        return s if s == self._last else super()._stream()


class ExpertRouter(_Here):
    """Chooses top_k of `experts` experts per token.

    score: "softmax" over the experts, or "sigmoid" of each logit.  groups, top_groups: the experts of the top_groups best of
    that many equal groups take part, groups scored by the sum of their group_top (1 or 2) largest values.  renormalize: the chosen scores
    are divided by their sum.  weight_scale: factor of all weights.  int64_ids: type of the ids (int32 otherwise)."""

    _state_bytes, _reset_entry = ROUTE_STATE, "iwp_route_reset"

    def __init__(self, experts: int, top_k: int, *, score: str = "softmax", groups: int = 1, top_groups: int = 1, group_top: int = 2,
                 renormalize: bool = True, weight_scale: float = 1.0, int64_ids: bool = False):
        lib()
        super().__init__()
        t = self._torch
        if score not in ("softmax", "sigmoid"):
            raise ValueError("score is 'softmax' or 'sigmoid'")
        self.experts, self.top_k, self.score, self.renormalize = int(experts), int(top_k), score, bool(renormalize)
        self._id_type = t.int64 if int64_ids else t.int32
        self._masks = (t.bool, t.uint8)
        code = IWP_SOFTMAX if score == "softmax" else IWP_SIGMOID
        self._args = a = RouteArgs(state=self._state_at, weight_scale=weight_scale, experts=self.experts, top_k=self.top_k, groups=groups,
                                   top_groups=top_groups, group_top=group_top, score=code, renormalize=self.renormalize,
                                   ids_bytes=8 if int64_ids else 4)
        self._grad_args = RouteGradArgs(weight_scale=weight_scale, experts=self.experts, top_k=self.top_k, score=code,
                                        renormalize=self.renormalize)
        self._args_at, self._grad_at = C.addressof(a), C.addressof(self._grad_args)
        a.logits = a.ids = a.weights = 256  # a call without tokens touches nothing: the plan's sizes are checked here
        a.logits_ld = self.experts
        binding._check(self._lib.iwp_route(self._args_at, self._raw_stream(self._index)), "iwp_route")

    def route(self, logits, bias=None, mask=None) -> Route:
        """Experts and weights of router logits [T, E]; bias: [E] float32, added to the scores for the choice alone; mask: [T],
        False where a token goes to no expert."""
        t, dev, a, k = self._torch, self.device, self._args, self.top_k
        if logits.dim() != 2:
            raise ValueError("logits is a matrix")
        T = logits.shape[0]
        a.logits_ld = _rows_of(logits, "logits", (T, self.experts), self._floats, dev)
        a.tokens, a.logits, a.type = T, logits.data_ptr() or 256, self._codes[logits.dtype]
        if bias is None:
            a.bias = None
        else:
            _vector(bias, "bias", self.experts, self._floats[:1], dev)
            a.bias = bias.data_ptr()
        if mask is None:
            a.mask = None
        else:
            _vector(mask, "mask", T, self._masks, dev)
            a.mask = mask.data_ptr()
        ids, weights = t.empty(T, k, dtype=self._id_type, device=dev), t.empty(T, k, dtype=t.float32, device=dev)
        counts = t.empty(self.experts, dtype=t.int32, device=dev)
        a.ids, a.weights, a.counts = ids.data_ptr() or 256, weights.data_ptr() or 256, counts.data_ptr()
        status = self._lib.iwp_route(self._args_at, self._stream())
        if status:
            raise IwpError(status, "iwp_route")
        return Route(ids, weights, counts)

    def grad(self, logits, ids, weights, dweights, *, scale: float = 1.0, dlogits=None, accumulate: bool = False):
        """The gradient [T, E] to the logits, times `scale`, for the gradient dweights to the weights of `route`.

        ids: as `route` returns them, distinct in a row.  dlogits: where to write, of the logits' type; accumulate adds to
        what it holds, such as the balance loss's gradient."""
        t, dev, a, k = self._torch, self.device, self._grad_args, self.top_k
        if logits.dim() != 2:
            raise ValueError("logits is a matrix")
        T = logits.shape[0]
        a.logits_ld = _rows_of(logits, "logits", (T, self.experts), self._floats, dev)
        a.ids_ld = _rows_of(ids, "ids", (T, k), self._ids, dev)
        a.weights_ld = _rows_of(weights, "weights", (T, k), self._floats[:1], dev)
        a.dweights_ld = _rows_of(dweights, "dweights", (T, k), self._floats[:1], dev)
        if dlogits is None:
            if accumulate:
                raise ValueError("accumulate needs the gradient to add to")
            dlogits = t.empty(T, self.experts, dtype=logits.dtype, device=dev)
            a.dlogits_ld = self.experts
        else:
            a.dlogits_ld = _rows_of(dlogits, "dlogits", (T, self.experts), (logits.dtype,), dev)
        if T == 0:
            return dlogits
        a.tokens, a.type, a.ids_bytes, a.scale, a.accumulate = T, self._codes[logits.dtype], ids.element_size(), scale, int(accumulate)
        a.logits, a.ids, a.weights, a.dweights, a.dlogits = logits.data_ptr(), ids.data_ptr(), weights.data_ptr(), dweights.data_ptr(), dlogits.data_ptr()
        status = self._lib.iwp_route_grad(self._grad_at, self._stream())
        if status:
            raise IwpError(status, "iwp_route_grad")
        return dlogits


class ExpertExchange(_Here):
    """Rows from tokens to the experts of their ids and back, sorted by expert."""

    def __init__(self, experts: int):
        lib()
        super().__init__()
        self.experts = int(experts)
        self._order_args = a = OrderArgs(experts=self.experts, top_k=1, ids_bytes=4)
        self._plan(self._lib.iwp_order_workspace(C.byref(a)))
        self._order_at = C.addressof(a)

        def entry(name):
            args = ExchangeArgs(experts=self.experts)  # of every call
            return args, C.addressof(args), getattr(self._lib, name)

        self._dispatch, self._combine, self._combine_grad = entry("iwp_dispatch"), entry("iwp_combine"), entry("iwp_combine_grad")

    def order(self, ids) -> Order:
        """Slots of the pairs (t, j) with ids [T, k]; ids outside the experts belong to none."""
        t, dev, a = self._torch, self.device, self._order_args
        if ids.dim() != 2:
            raise ValueError("ids is a matrix")
        T, k = shape = ids.shape
        a.ids_ld = _rows_of(ids, "ids", shape, self._ids, dev)
        a.tokens, a.top_k, a.ids, a.ids_bytes = T, k, ids.data_ptr() or 256, ids.element_size()
        offsets = t.empty(self.experts + 1, dtype=t.int32, device=dev)
        slots, rows = t.empty(T, k, dtype=t.int32, device=dev), t.empty(T * k, dtype=t.int32, device=dev)
        offsets_at, at = offsets.data_ptr(), slots.data_ptr()
        a.offsets, a.slots, a.rows = offsets_at, at or 256, rows.data_ptr() or 256
        stream = self._stream()
        if self._capturing():
            self._captured = True
        if self._ws_at is None:
            self._grow(0)
        a.workspace, a.workspace_bytes = self._ws_at, self._ws_bytes
        status = self._lib.iwp_order(self._order_at, stream)
        if status:
            raise IwpError(status, "iwp_order")
        order = _Made(offsets, slots, rows)
        order.made = self, T, k, shape, at, offsets_at, None if slots.is_inference() else slots._version
        return order

    def _begin(self, a: ExchangeArgs, order: Order, x, name: str):
        """T, k and the width of x, a matrix, in an exchange by `order`, and what makes a matrix that its slots are written to, of x's type."""
        shape = x.shape
        if len(shape) != 2:
            raise ValueError(f"{name} is a matrix")
        offsets, slots, _ = order
        plan, T, k, of, at, offsets_at, version = order.made if type(order) is _Made else _UNKNOWN
        new = x.new_empty
        # (an order's tensors can be written to, resized, transposed or set to other memory after it was made)
        if (plan is not self or slots.data_ptr() != at or offsets.data_ptr() != offsets_at or slots.shape != of or not slots.is_contiguous()
                or (version is not None and slots._version != version)):
            if slots.dim() != 2:
                raise ValueError("slots is a matrix")
            _vector(slots, "slots", slots.numel(), self._ids[1:], self.device)
            _vector(offsets, "offsets", self.experts + 1, self._ids[1:], self.device)
            T, k = slots.shape
            at, offsets_at = slots.data_ptr(), offsets.data_ptr()
            new = x.new_zeros  # (there may be slots that no pair has)
        D = shape[1]
        a.slots, a.offsets, a.tokens, a.top_k, a.dim = at, offsets_at, T, k, D
        return T, k, D, new

    def _end(self, a: ExchangeArgs, at: int, call, entry: str) -> None:
        if a.tokens == 0 or a.dim == 0:
            return
        status = call(at, self._stream())
        if status:
            raise IwpError(status, entry)

    def dispatch(self, x, order: Order, *, out=None):
        """Rows [T k, D] in the order of the slots: x [T, D] of each slot's token; zero behind the last slot, and where pairs were
        dropped from an order (slots set to -1, not in place in inference mode), but for rows of `out` below the last slot, which are
        left as they are."""
        a, at, call = self._dispatch
        T, k, D, new = self._begin(a, order, x, "x")
        a.by_token_ld = _rows_of(x, "x", (T, D), self._floats, self.device)
        a.by_token, a.type = x.data_ptr(), self._codes[x.dtype]
        if out is None:
            out = new(T * k, D)
            a.by_slot_out_ld = D
        else:
            a.by_slot_out_ld = _rows_of(out, "out", (T * k, D), (x.dtype,), self.device)
        a.by_slot_out = out.data_ptr()
        self._end(a, at, call, "iwp_dispatch")
        return out

    def combine(self, z, order: Order, weights=None, *, out=None):
        """Rows [T, D]: the sum of each token's rows of z [T k, D], times weights [T, k] float32 (1 if None)."""
        a, at, call = self._combine
        T, k, D, _ = self._begin(a, order, z, "z")
        a.by_slot_ld = _rows_of(z, "z", (T * k, D), self._floats, self.device)
        a.by_slot, a.type = z.data_ptr(), self._codes[z.dtype]
        if weights is None:
            a.weights = None
        else:
            a.weights_ld = _rows_of(weights, "weights", (T, k), self._floats[:1], self.device)
            a.weights = weights.data_ptr()
        if out is None:
            out = z.new_empty(T, D)
            a.by_token_out_ld = D
        else:
            a.by_token_out_ld = _rows_of(out, "out", (T, D), (z.dtype,), self.device)
        a.by_token_out = out.data_ptr()
        self._end(a, at, call, "iwp_combine")
        return out

    def dispatch_grad(self, dout, order: Order, *, out=None):
        """The gradient [T, D] to x of `dispatch`, for the gradient [T k, D] to its rows."""
        return self.combine(dout, order, None, out=out)

    def combine_grad(self, dy, z, order: Order, weights=None, *, out=None, want=("rows", "weights")):
        """The gradients ([T k, D] to z, [T, k] float32 to the weights) of `combine`; None where `want` leaves one out.  Rows of
        dropped pairs as in `dispatch`."""
        a, at, call = self._combine_grad
        T, k, D, new = self._begin(a, order, dy, "dy")
        a.by_token_ld = _rows_of(dy, "dy", (T, D), self._floats, self.device)
        a.by_token, a.type = dy.data_ptr(), self._codes[dy.dtype]
        if weights is None:
            a.weights = None
        else:
            a.weights_ld = _rows_of(weights, "weights", (T, k), self._floats[:1], self.device)
            a.weights = weights.data_ptr()
        dz = dw = a.by_slot = a.by_slot_out = a.dweights = None
        if "rows" in want:
            if out is None:
                dz = new(T * k, D)
                a.by_slot_out_ld = D
            else:
                dz = out
                a.by_slot_out_ld = _rows_of(dz, "out", (T * k, D), (dy.dtype,), self.device)
            a.by_slot_out = dz.data_ptr()
        if "weights" in want:
            a.by_slot_ld = _rows_of(z, "z", (T * k, D), (dy.dtype,), self.device)
            dw = self._torch.empty(T, k, dtype=self._torch.float32, device=self.device)
            a.by_slot, a.dweights = z.data_ptr(), dw.data_ptr()
        if D == 0 and dw is not None:
            dw.zero_()
        if dz is not None or dw is not None:
            self._end(a, at, call, "iwp_combine_grad")
        return dz, dw


# ---- differentiable forms (once: a second derivative is refused) --------------------------------------


def _functions():
    global _autograd
    if _autograd is None:
        import torch

        Once = losses._once()

        class Routing(torch.autograd.Function):
            @staticmethod
            def forward(ctx, logits, plan, bias, mask):
                r = plan.route(logits, bias, mask)
                ctx.plan = plan
                ctx.save_for_backward(logits, r.ids, r.weights)
                ctx.mark_non_differentiable(r.ids, r.counts)
                return r.weights, r.ids, r.counts

            @staticmethod
            def backward(ctx, dweights, _, __):
                logits, ids, weights = ctx.saved_tensors
                make = lambda: ctx.plan.grad(logits, ids, weights, dweights.contiguous())  # noqa: E731
                return Once.apply(make, logits, dweights), None, None, None

        class Dispatch(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, plan, order):
                ctx.plan, ctx.made = plan, getattr(order, "made", _UNKNOWN)
                ctx.save_for_backward(*order)
                return plan.dispatch(x, order)

            @staticmethod
            def backward(ctx, dout):
                order = _made(ctx.saved_tensors, ctx.made)
                return Once.apply(lambda: ctx.plan.dispatch_grad(dout.contiguous(), order), dout), None, None

        class Combine(torch.autograd.Function):
            @staticmethod
            def forward(ctx, z, weights, plan, order):
                ctx.plan, ctx.made = plan, getattr(order, "made", _UNKNOWN)
                ctx.save_for_backward(z, weights, *order)
                return plan.combine(z, order, weights)

            @staticmethod
            def backward(ctx, dy):
                z, weights, *order = ctx.saved_tensors
                want = tuple(n for n, need in zip(("rows", "weights"), ctx.needs_input_grad) if need)
                order = _made(order, ctx.made)
                make = lambda: ctx.plan.combine_grad(dy.contiguous(), z, order, weights, want=want)  # noqa: E731
                return *Once.apply(make, z, weights, dy), None, None

        _autograd = (Routing, Dispatch, Combine)
    return _autograd


_autograd = None


def route(plan: ExpertRouter, logits, bias: Optional[object] = None, mask=None) -> Route:
    """plan.route with weights that are a differentiable function of the logits."""
    weights, ids, counts = _functions()[0].apply(logits, plan, bias, mask)
    return Route(ids, weights, counts)


def dispatch(plan: ExpertExchange, x, order: Order):
    """plan.dispatch as a differentiable function of x."""
    return _functions()[1].apply(x, plan, order)


def combine(plan: ExpertExchange, z, order: Order, weights):
    """plan.combine as a differentiable function of z and the weights."""
    return _functions()[2].apply(z, weights, plan, order)
