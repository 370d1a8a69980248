"""The example that trains a head and a router through the pruned step: with its router, with the mixture of experts, clipped."""
import math

import pytest
import torch

from paper_1901_01544_b200 import routing, train_head

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_gradients_of_the_mixture():
    """bf16 features: the mixture rounds them twice and its gradients once more each, by half a step (2^-8) of values of their
    size; sums over the tokens and features of a few hundred terms with random signs stay within 8 of their root mean square."""
    T, D, E, k = 96, 64, 8, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    x = torch.randn(T, D, generator=g, device=DEV).bfloat16()
    gain, logits, up = (torch.randn(*s, generator=g, device=DEV) for s in ((E, D), (T, E), (T, D)))
    router, exchange = routing.ExpertRouter(E, k), routing.ExpertExchange(E)
    r = router.route(logits)
    y, saved = train_head.mixture(exchange, x, gain, r)
    dgain, dweights = train_head.mixture_grad(exchange, up.bfloat16(), gain, r, saved)
    g64, w64 = gain.double().requires_grad_(), r.weights.double().requires_grad_()
    parts = x.double()[:, None, :] * (1 + g64[r.ids.long()])
    want = (w64[:, :, None] * parts).sum(1)
    want.backward(up.bfloat16().double())
    h = 2.0**-8
    size = (w64[:, :, None] * parts).abs().sum(1).detach()
    assert ((y.double() - want).abs() <= 2 * h * size).all()
    per_pair = (up.abs().double()[:, None, :] * w64[:, :, None] * x.double().abs()[:, None, :]).detach()
    bound = torch.zeros(E, D, dtype=torch.float64, device=DEV).index_add_(0, r.ids.long().flatten(), (2 * h * per_pair).flatten(0, 1))
    assert ((dgain.double() - g64.grad).abs() <= bound).all()
    assert ((dweights.double() - w64.grad).abs() <= 2 * h * (up.abs().double()[:, None, :] * parts.abs()).sum(2).detach()).all()


@pytest.mark.parametrize("kw", [dict(), dict(mix=True), dict(mix=True, clip=0.5), dict(clip=1e-3)])
def test_example_runs(kw):
    history, counts = train_head.train(steps=3, workers=2, tokens=128, vocab=503, dim=64, **kw)
    assert len(history) == 3 and all(math.isfinite(v) for row in history for v in row) and sum(counts) == 2 * 128 * 2


def test_router_chooses_as_before():
    """The example's losses are those that choosing by torch.topk gives."""
    x = torch.randn(300, 16, device=DEV)
    ids = routing.ExpertRouter(16, 2).route(x).ids
    assert torch.equal(ids.long(), torch.topk(x, 2, dim=1).indices)
