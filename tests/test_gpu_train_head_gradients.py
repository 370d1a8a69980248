"""What the example that trains a head and a router hands to the pruned step: the router's gradient, and the choices behind it."""
import pytest
import torch

from paper_1901_01544_b200 import binding, losses, routing, train_head

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, U = 2.0**-8, 2.0**-24


@pytest.mark.parametrize("workers", [1, 2])
def test_the_gates_gradient_has_both_parts(monkeypatch, workers):
    """Of the balance loss and of the head's loss through the mixture, against 64 bits, in a step whose experts differ; the gradient to
    the mixture's features is taken as the head gives it.

    Bounds: a chosen expert's upstream gradient is a product of features that bf16 has rounded once (half a step, taken twice for the
    sums in fp32 behind it); renormalized weights pass on w_j (d_j - sum_i p_i d_i).  The balance loss's part is fp32: 64 roundings."""
    T, D, E, V = 128, 64, 16, 503
    steps, calls = [], []
    real = {name: getattr(train_head, name) for name in ("mixture", "mixture_grad")}
    route = routing.ExpertRouter.route
    monkeypatch.setattr(routing.ExpertRouter, "route", lambda self, x, *a: calls.append([x.clone()]) or route(self, x, *a))
    monkeypatch.setattr(train_head, "mixture", lambda ex, x, gain, r: calls[-1].extend([x, gain.clone(), r]) or real["mixture"](ex, x, gain, r))
    monkeypatch.setattr(train_head, "mixture_grad", lambda ex, dy, gain, r, s: calls[-1].append(dy.clone()) or real["mixture_grad"](ex, dy, gain, r, s))

    class Step(binding.Pruner):
        def step(self, grads, master, update, *a, **kw):
            steps.append(grads.clone())
            out = super().step(grads, master, update, *a, **kw)
            g = torch.Generator(device=DEV).manual_seed(7)
            master[-E * D :] = torch.randn(E * D, generator=g, device=DEV)  # gains that make experts differ
            return out

    monkeypatch.setattr(binding, "Pruner", Step)
    train_head.train(steps=2, workers=workers, tokens=T, vocab=V, dim=D, experts=E, mix=True)
    assert len(steps) == 2 and len(calls) == 2 * workers
    for w, (scores, x, gain, r, dy) in enumerate(calls[workers:]):
        got = steps[1][w, V * D : V * D + E * D].view(E, D).double()
        ids, x, dy = r.ids.long(), x.double(), dy.double()
        s64 = scores.double().requires_grad_()
        weights = torch.softmax(torch.gather(s64, 1, ids), 1)
        parts = (1 + gain.double()[ids]) * x[:, None, :]
        (through,) = torch.autograd.grad((weights[:, :, None] * parts).sum(1), s64, dy)
        f = torch.bincount(ids.flatten(), minlength=E).double() / ids.numel()
        p = torch.softmax(s64, 1)
        (balance,) = torch.autograd.grad(E * (f * p.mean(0)).sum(), s64)
        want = (through + balance).T @ x
        p, weights = p.detach(), weights.detach()
        off = 2 * H * (dy.abs()[:, None, :] * parts.abs()).sum(2)
        off = weights * (off + (weights * off).sum(1, keepdim=True))
        off = torch.zeros(T, E, dtype=torch.float64, device=DEV).scatter_add_(1, ids, off)
        off += 64 * U * E / T * p * (f + (f * p).sum(1, keepdim=True))
        bound = off.T @ x.abs() + T * U * ((through + balance).abs().T @ x.abs())
        assert ((got - want).abs() <= bound).all()
        # the mixture's part could not be missing (that of the balance loss, the smaller one here, is alone in the test below)
        assert ((through.T @ x).abs() > bound).double().mean() > 0.2


def test_the_gates_gradient_without_a_mixture(monkeypatch):
    """Of the balance loss alone: 64 roundings of its terms, and a sum over the tokens, in fp32."""
    T, D, E, V = 128, 64, 16, 503
    steps, calls = [], []
    route, balance_grad, step = routing.ExpertRouter.route, losses.ExpertBalance.grad, binding.Pruner.step
    monkeypatch.setattr(routing.ExpertRouter, "route", lambda self, x, *a: calls.append([x.clone()]) or route(self, x, *a))
    monkeypatch.setattr(losses.ExpertBalance, "grad", lambda self, x, ids, **kw: calls[-1].append(ids.long()) or balance_grad(self, x, ids, **kw))
    monkeypatch.setattr(binding.Pruner, "step", lambda self, grads, master, update: steps.append(grads.clone()) or step(self, grads, master, update))
    features = []
    monkeypatch.setattr(losses.HeadLoss, "distill_grad", record(features, losses.HeadLoss.distill_grad))
    train_head.train(steps=1, workers=2, tokens=T, vocab=V, dim=D, experts=E)
    for w, ((scores, ids), x) in enumerate(zip(calls, features)):
        got = steps[0][w, V * D :].view(E, D).double()
        x, s64 = x.double(), scores.double().requires_grad_()
        f = torch.bincount(ids.flatten(), minlength=E).double() / ids.numel()
        p = torch.softmax(s64, 1)
        (balance,) = torch.autograd.grad(E * (f * p.mean(0)).sum(), s64)
        p = p.detach()
        bound = (64 * U * E / T * p * (f + (f * p).sum(1, keepdim=True))).T @ x.abs() + T * U * (balance.abs().T @ x.abs())
        want = balance.T @ x
        assert ((got - want).abs() <= bound).all() and (want.abs() > bound).double().mean() > 0.9


def record(into, call):
    """call, whose first argument is kept."""

    def wrapped(self, x, *a, **kw):
        into.append(x.clone())
        return call(self, x, *a, **kw)

    return wrapped


def test_losses_are_those_of_choices_by_topk(monkeypatch):
    args = dict(steps=3, workers=2, tokens=128, vocab=503, dim=64)
    own = train_head.train(**args)
    again = train_head.train(**args)

    def topk(self, x, bias=None, mask=None):
        top = torch.topk(x, self.top_k, dim=1)
        return routing.Route(top.indices, torch.softmax(top.values, 1), None)

    monkeypatch.setattr(routing.ExpertRouter, "route", topk)
    assert own == again and train_head.train(**args) == own


@pytest.mark.parametrize("seed", range(4))
def test_chooses_as_topk(seed):
    """ids alone; of logits without ties."""
    x = torch.randn(300, 16, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    assert all(len(torch.unique(row)) == 16 for row in x)
    assert torch.equal(routing.ExpertRouter(16, 2).route(x).ids.long(), torch.topk(x, 2, dim=1).indices)
