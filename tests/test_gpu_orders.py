"""An exchange by orders that were remade or changed after the plan made them."""
import copy

import pytest
import torch

from paper_1901_01544_b200 import routing

pytestmark = pytest.mark.gpu
DEV = "cuda"
T, E, K, D = 70, 9, 3, 40


def setting():
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    ex = routing.ExpertExchange(E)
    ids = torch.stack([torch.randperm(E, generator=g, device=DEV)[:K] for _ in range(T)])
    x, dy, z, w = (torch.randn(*s, generator=g, device=DEV) for s in ((T, D), (T, D), (T * K, D), (T, K)))
    return ex, ex.order(ids), x, dy, z, w


def calls(ex, o, x, dy, z, w):
    return [ex.dispatch(x, o), ex.combine(z, o, w), *ex.combine_grad(dy, z, o, w), ex.dispatch_grad(z, o)]


@pytest.mark.parametrize("remade", [lambda o: o._replace(), lambda o: type(o)(*o), copy.copy, copy.deepcopy,
                                    lambda o: torch.utils._pytree.tree_map(torch.clone, o)])
def test_remade_orders(remade):
    ex, o, *rows = setting()
    assert all(torch.equal(a, b) for a, b in zip(calls(ex, remade(o), *rows), calls(ex, o, *rows)))


def test_pairs_dropped_from_an_order():
    """Slots of -1 are nobody's: not read, not written, no gradient."""
    ex, o, x, dy, z, w = setting()
    drop = torch.rand(T, K, device=DEV) < 0.3
    less = o._replace(slots=torch.where(drop, -1, o.slots))
    keep, slots = ~drop, o.slots.long()
    there = torch.full((T * K, D), 7.0, device=DEV)
    want = there.clone()
    want[slots[keep]] = x[:, None].expand(T, K, D)[keep]
    assert torch.equal(ex.dispatch(x, less, out=there), want)
    y = ex.combine(z, less, w).double()
    parts = (w.double()[:, :, None] * z.double()[slots]).masked_fill(drop[:, :, None], 0)
    # three terms, each sum rounded (2^-24 of what it may be at most)
    assert ((y - parts.sum(1)).abs() <= 3 * 2.0**-24 * parts.abs().sum(1)).all()
    dz, dw = ex.combine_grad(dy, z, less, w, out=there.clone())
    want = there.clone()
    want[slots[keep]] = (w[:, :, None] * dy[:, None])[keep]
    assert torch.equal(dz, want) and (dw[drop] == 0).all()
    # without an output they are written to, zero
    want = torch.zeros(T * K, D, device=DEV)
    want[slots[keep]] = (w[:, :, None] * dy[:, None])[keep]
    held = torch.full((T * K, D), float("nan"), device=DEV)
    del held  # (what the next allocation may find)
    assert torch.equal(ex.combine_grad(dy, z, less, w, want=("rows",))[0], want)
    want[slots[keep]] = x[:, None].expand(T, K, D)[keep]
    held = torch.full((T * K, D), float("nan"), device=DEV)
    del held
    assert torch.equal(ex.dispatch(x, less), want)
    products = dy.double()[:, None] * z.double()[slots]
    assert ((dw.double() - products.sum(2)).abs()[keep] <= (D + 2) * 2.0**-24 * products.abs().sum(2)[keep]).all()


def test_an_order_moved_in_memory():
    ex, o, *rows = setting()
    want = calls(ex, o, *rows)
    kept = o.slots.clone(), o.offsets.clone()
    o.slots.data, o.offsets.data = kept
    assert all(torch.equal(a, b) for a, b in zip(calls(ex, o, *rows), want))
    o.slots.resize_(T + 1, K)
    with pytest.raises(ValueError):
        ex.dispatch(rows[0], o)


@pytest.mark.parametrize("E", [8, 128, 1000])
@pytest.mark.parametrize("pairs", [4095, 4096, 4097, 4110, 6144, 6147, 8190, 8193])
def test_orders_about_where_more_blocks_take_part(pairs, E):
    """One pair per token, three, and ids that belong to nobody; slots are those of a stable sort."""
    for k in (1, 3):
        ids = torch.randint(-1, E + 1, (pairs // k, k), generator=torch.Generator(device=DEV).manual_seed(pairs), device=DEV)
        o = routing.ExpertExchange(E).order(ids)
        flat = ids.flatten()
        mine = (flat >= 0) & (flat < E)
        by_slot = torch.sort(torch.where(mine, flat, E), stable=True).indices[: int(mine.sum())]
        slots = torch.full_like(flat, -1)
        slots[by_slot] = torch.arange(len(by_slot), device=DEV)
        rows = torch.full_like(flat, -1)
        rows[: len(by_slot)] = by_slot // k
        counts = torch.bincount(flat[mine], minlength=E)
        assert torch.equal(o.slots.flatten().long(), slots) and torch.equal(o.rows.long(), rows)
        assert torch.equal(o.offsets.long(), torch.cat([counts.new_zeros(1), counts.cumsum(0)]))


def test_gradients_with_pairs_dropped():
    """The differentiable forms by an order that pairs were dropped from: nothing of what memory held reaches a gradient."""
    ex, o, x, dy, z, w = setting()
    drop = torch.rand(T, K, device=DEV) < 0.3
    less = o._replace(slots=torch.where(drop, -1, o.slots))
    x, w = x.requires_grad_(), w.requires_grad_()
    gain = torch.randn(T * K, D, device=DEV).requires_grad_()
    held = [torch.full((T * K, D), float("nan"), device=DEV) for _ in range(4)]
    del held
    y = routing.combine(ex, routing.dispatch(ex, x, less) * gain, less, w)
    got = torch.autograd.grad(y, [x, w, gain], dy)
    x64, w64, g64 = (v.detach().double().requires_grad_() for v in (x, w, gain))
    want = (w64.masked_fill(drop, 0)[:, :, None] * g64[o.slots.long()] * x64[:, None]).sum(1)
    ref = torch.autograd.grad(want, [x64, w64, g64], dy.double())
    # roundings of 2^-24: two products and a sum of three terms, a product and a sum of D products, two products
    w0, d0 = w64.detach().abs().masked_fill(drop, 0)[:, :, None], dy.double().abs()[:, None]
    g0, x0 = g64.detach().abs()[o.slots.long()], x64.detach().abs()[:, None]
    size = ((w0 * d0 * g0).sum(1), (d0 * g0 * x0).sum(2), torch.zeros(T * K, D, device=DEV).double().index_copy_(0, o.slots.flatten().long(), (w0 * d0 * x0).flatten(0, 1)))
    for a, b, n, bound in zip(got, ref, (6, D + 3, 3), size):
        assert ((a.double() - b).abs() <= n * 2.0**-24 * bound).all()
    assert torch.equal(got[1] == 0, drop)


@pytest.mark.parametrize("inference", [False, True])
def test_pairs_dropped_in_place(inference):
    with torch.inference_mode(inference):
        ex, o, x, *_ = setting()
        whole = ex.dispatch(x, o)
        drop = torch.rand(T, K, device=DEV) < 0.3
        slots = o.slots.long()
        less = o if not inference else o._replace(slots=o.slots.clone())
        less.slots.masked_fill_(drop, -1)
        held = torch.full((T * K, D), float("nan"), device=DEV)
        del held
        want = whole.clone()
        want[slots[drop]] = 0
        assert torch.equal(ex.dispatch(x, less), want)
