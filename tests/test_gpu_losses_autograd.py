"""The differentiable forms of the losses refuse what they cannot answer: second derivatives, and inputs that were changed
between the forward and the backward pass."""
import pytest
import torch
from test_gpu_losses import BF, DEV, operands

from paper_1901_01544_b200 import losses

pytestmark = pytest.mark.gpu
T, V, D, E, K = 60, 300, 32, 16, 5


def forms():
    h, w, y, g = operands(T, V, D, BF, 950)
    plan, router = losses.HeadLoss(T, V, D, BF, top_k=K), losses.ExpertBalance(T, E)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :K].contiguous()
    teacher = torch.randn(T, K, generator=g, device=DEV)
    x = torch.randn(T, E, generator=g, device=DEV)
    chosen = torch.topk(x, 2, dim=1).indices
    mask = torch.rand(T, generator=g, device=DEV) < 0.8
    h.requires_grad_(), w.requires_grad_(), x.requires_grad_()
    return {
        "cross_entropy": (lambda: losses.cross_entropy(plan, h, w, y), h, [y]),
        "distill": (lambda: losses.distill(plan, h, w, ids, teacher, 2.0), h, [ids, teacher]),
        "balance": (lambda: losses.balance(router, x, chosen, mask, 1.0)[0], x, [chosen, mask]),
    }


@pytest.mark.parametrize("form", ["cross_entropy", "distill", "balance"])
def test_second_derivatives_are_refused(form):
    call, leaf, _ = forms()[form]
    loss = call()
    (grad,) = torch.autograd.grad(loss, leaf, create_graph=True)
    plain = torch.autograd.grad(call(), leaf)[0]
    assert torch.equal(grad.detach(), plain)
    with pytest.raises(RuntimeError):  # a gradient penalty would silently be left out
        (call() + grad.float().pow(2).sum()).backward()


@pytest.mark.parametrize("form,which", [("cross_entropy", 0), ("distill", 0), ("distill", 1), ("balance", 0), ("balance", 1)])
def test_inputs_changed_before_the_backward_pass_are_refused(form, which):
    call, leaf, others = forms()[form]
    loss = call()
    others[which].copy_(others[which].flip(0))
    with pytest.raises(RuntimeError):
        loss.backward()
    call().backward()  # as they are now
    assert torch.isfinite(leaf.grad.float()).all()


def test_saved_tensor_hooks_see_every_input():
    for form, (call, _, others) in forms().items():
        seen = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append(t.data_ptr()) or t, lambda t: t):
            call().backward()
        assert all(t.data_ptr() in seen for t in others), form
