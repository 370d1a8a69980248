"""CPU-only checks of what an exchange takes for an order: as it was made, remade by what rebuilds tuples, and changed since.
The plan is a real one without its CUDA side; the arguments that a launch would get are looked at."""
import copy
import ctypes as C
import pickle

import pytest
import torch

from paper_1901_01544_b200 import routing

T, K, E, D = 6, 3, 5, 4


class Nothing:
    """A library whose calls succeed and do nothing."""

    def iwp_order(self, args, stream):
        return 0


def plan():
    p = object.__new__(routing.ExpertExchange)
    p._torch, p.device, p.experts, p._lib = torch, torch.device("cpu"), E, Nothing()
    p._ids, p._codes = (torch.int64, torch.int32), {torch.float32: 0}
    p._floats = tuple(p._codes)
    p._order_args = routing.OrderArgs(experts=E, top_k=1, ids_bytes=4)
    p._order_at = C.addressof(p._order_args)
    p._stream, p._capturing, p._ws_at, p._ws_bytes = (lambda: 0), (lambda: False), 256, 256
    return p


def order(p):
    o = p.order(torch.zeros(T, K, dtype=torch.int32))
    with torch.no_grad():
        o.offsets.data.zero_(), o.slots.data.copy_(torch.arange(T * K).view(T, K)), o.rows.data.zero_()
    return o


def taken(p, o):
    """What a call with this order hands over: tokens, choices, and where slots and offsets are."""
    a = routing.ExchangeArgs()
    x = torch.zeros(T, D)
    assert p._begin(a, o, x, "x")[:3] == (a.tokens, a.top_k, D)
    return a.tokens, a.top_k, a.slots, a.offsets


def at(o):
    return (*o.slots.shape, o.slots.data_ptr(), o.offsets.data_ptr())


REMADE = {
    "replace nothing": lambda o: o._replace(),
    "replace slots": lambda o: o._replace(slots=torch.where(o.slots % 2 == 0, -1, o.slots)),
    "type": lambda o: type(o)(*o),
    "make": lambda o: type(o)._make(list(o)),
    "tree_map": lambda o: torch.utils._pytree.tree_map(torch.clone, o),
    "copy": copy.copy,
    "deepcopy": copy.deepcopy,
    "pickle": lambda o: pickle.loads(pickle.dumps(o)),
}


@pytest.mark.parametrize("how", REMADE)
def test_a_remade_order_is_taken_with_its_own_tensors(how):
    p = plan()
    o = order(p)
    remade = REMADE[how](o)
    assert isinstance(remade, routing.Order) and remade._fields == o._fields
    assert taken(p, remade) == at(remade) and taken(p, o) == at(o)
    if "slots" not in how:
        assert all(torch.equal(a, b) for a, b in zip(remade, o))


def test_a_remade_order_does_not_hold_its_plan():
    p = plan()
    for how in REMADE.values():
        remade = how(order(p))
        assert p not in getattr(remade, "made", ())


def test_an_order_whose_tensors_have_moved_is_taken_where_they_are():
    p = plan()
    o = order(p)
    o.slots.data = o.slots.clone()
    o.offsets.set_(o.offsets.clone())
    assert taken(p, o) == at(o)
    o.slots.resize_(2 * T, K)
    assert taken(p, o) == at(o) and o.slots.shape == (2 * T, K)
    o.slots.resize_(T - 1, K)  # (stays where it is)
    assert taken(p, o) == at(o) and o.slots.shape == (T - 1, K)


def test_an_order_that_no_longer_fits_is_refused():
    p = plan()
    a = routing.ExchangeArgs()
    x = torch.zeros(T, D)
    o = p.order(torch.zeros(K, K, dtype=torch.int32))
    o.slots.t_()  # the same memory and shape, in another order
    with pytest.raises(ValueError):
        p._begin(a, o, x, "x")
    o = order(p)
    o.offsets.set_(torch.zeros(E, dtype=torch.int32))
    with pytest.raises(ValueError):
        p._begin(a, o, x, "x")
    for bad in (dict(slots=o.slots.flatten()), dict(slots=o.slots[:, :2]), dict(offsets=o.offsets[:3])):
        with pytest.raises(ValueError):
            p._begin(a, o._replace(**bad), x, "x")
    with pytest.raises(TypeError):
        p._begin(a, o._replace(slots=o.slots.long()), x, "x")


class Rows:
    """A plan whose exchange leaves rows where they are."""

    def dispatch(self, x, order):
        return x.clone()

    def dispatch_grad(self, dout, order):
        return dout.clone()


def test_the_refusal_of_a_second_derivative_names_no_other_operator():
    x = torch.ones(T, D, requires_grad=True)
    o = routing.Order(*(torch.zeros(1, dtype=torch.int32) for _ in range(3)))
    (dx,) = torch.autograd.grad(routing.dispatch(Rows(), x, o).square().sum(), [x], create_graph=True)
    with pytest.raises(RuntimeError, match="cannot be differentiated again") as refused:
        dx.sum().backward()
    assert "loss" not in str(refused.value)


def test_what_is_written_to_is_looked_at_again():
    """Slots that no pair has any more are made zero; a plan's own order, in inference mode too, has none."""
    p = plan()
    a, x = routing.ExchangeArgs(), torch.zeros(T, D)
    for inference in (False, True):
        with torch.inference_mode(inference):
            o = p.order(torch.zeros(T, K, dtype=torch.int32))
            assert p._begin(a, o, x, "x")[3].__name__ == "new_empty"
            assert p._begin(a, o._replace(slots=o.slots.clone()), x, "x")[3].__name__ == "new_zeros"
            assert p._begin(a, routing.Order(*o), x, "x")[3].__name__ == "new_zeros"
            if not inference:
                o.slots[0, 0] = -1
                assert p._begin(a, o, x, "x")[3].__name__ == "new_zeros"


def test_a_backward_pass_knows_its_plans_order():
    p = plan()
    seen = []
    p.dispatch = lambda x, o: x.clone()

    def dispatch_grad(dout, o):
        seen.append(p._begin(routing.ExchangeArgs(), o, dout, "dout")[3].__name__)
        return dout.clone()

    p.dispatch_grad = dispatch_grad
    x = torch.ones(T, D, requires_grad=True)
    routing.dispatch(p, x, order(p)).sum().backward()
    o = order(p)
    routing.dispatch(p, x, o._replace(slots=o.slots.clone())).sum().backward()
    assert seen == ["new_empty", "new_zeros"]
