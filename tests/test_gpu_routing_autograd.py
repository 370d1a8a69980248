"""The differentiable forms of routing and exchange refuse what they cannot answer, and are captured with their backward pass."""
import pytest
import torch

from paper_1901_01544_b200 import routing

pytestmark = pytest.mark.gpu
DEV = "cuda"
T, E, K, D = 70, 24, 3, 40


def forms():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    logits, x, z, w = (torch.randn(*s, generator=g, device=DEV).requires_grad_() for s in ((T, E), (T, D), (T * K, D), (T, K)))
    mask = torch.rand(T, generator=g, device=DEV) < 0.8
    router, exchange = routing.ExpertRouter(E, K), routing.ExpertExchange(E)
    order = exchange.order(router.route(logits.detach()).ids)
    return {
        "route": (lambda: routing.route(router, logits, None, mask).weights, [logits], [logits]),
        "dispatch": (lambda: routing.dispatch(exchange, x, order), [x], [order.slots]),
        "combine": (lambda: routing.combine(exchange, z, order, w), [z, w], [z, w, order.slots]),
    }


@pytest.mark.parametrize("form", ["route", "dispatch", "combine"])
def test_second_derivatives_are_refused(form):
    call, leaves, _ = forms()[form]
    grads = torch.autograd.grad(call().square().sum(), leaves, create_graph=True)
    plain = torch.autograd.grad(call().square().sum(), leaves)
    assert all(torch.equal(a.detach(), b) for a, b in zip(grads, plain))
    with pytest.raises(RuntimeError):
        sum(a.pow(2).sum() for a in grads).backward()


@pytest.mark.parametrize("form", ["route", "dispatch", "combine"])
def test_inputs_changed_before_the_backward_pass_are_refused(form):
    for i in range(len(forms()[form][2])):
        call, leaves, kept = forms()[form]
        out = call().square().sum()
        with torch.no_grad():
            kept[i].copy_(kept[i].flip(0))
        with pytest.raises(RuntimeError):
            out.backward()
        call().square().sum().backward()
        assert all(torch.isfinite(x.grad).all() for x in leaves)


def test_only_what_needs_a_gradient():
    call, (z, w), _ = forms()["combine"]
    (dz,) = torch.autograd.grad(call().sum(), [z])
    (dw,) = torch.autograd.grad(call().sum(), [w])
    both = torch.autograd.grad(call().sum(), [z, w])
    assert torch.equal(dz, both[0]) and torch.equal(dw, both[1])


@pytest.mark.parametrize("form", ["route", "dispatch", "combine"])
def test_captured_with_the_backward_pass(form):
    call, leaves, _ = forms()[form]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(call().square().sum(), leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
        grads = torch.autograd.grad(out.square().sum(), leaves)
    with torch.no_grad():
        for x in leaves:
            x.mul_(0.5)
    graph.replay()
    got = [out.clone(), *(d.clone() for d in grads)]
    want = call()
    want = [want, *torch.autograd.grad(want.square().sum(), leaves)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
