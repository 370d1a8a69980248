"""Example: W simulated workers train an output head and a router, their gradients reduced by the pruned step.

    python -m paper_1901_01544_b200.train_head [--steps 20] [--workers 4] [--ratio 16] [--mixture] [--clip 1.0]

Every step each worker takes its own batch of features (fixed random ones here, where a model would compute them), adds
the cross entropy of its targets and the distillation from a teacher's top logits straight into its head segment of
grads[w], routes its tokens and takes the balance loss's gradient for the router's segment; `Pruner.step` then prunes,
reduces and leaves the rest in the workers' residuals, and plain gradient descent applies the update.

With --mixture the router's experts do something: expert e scales the features by 1 + gain[e], each token's features go to its
experts and come back weighted, and the cross entropy's gradient reaches gains and router.  With --clip every worker's
gradients are clipped by their norm before the step.
"""
from __future__ import annotations

import argparse


def mixture(exchange, x, gain, route):
    """Features [T, D] after the experts of `route`; what the gradient needs besides."""
    import torch

    order = exchange.order(route.ids)
    sent = exchange.dispatch(x, order)
    slots = torch.arange(sent.shape[0], device=x.device, dtype=torch.int32)
    owner = torch.searchsorted(order.offsets[1:].contiguous(), slots, right=True).clamp_(max=gain.shape[0] - 1)
    scaled = (sent.float() * (1.0 + gain[owner])).to(x.dtype)
    return exchange.combine(scaled, order, route.weights), (order, sent, owner, scaled)


def mixture_grad(exchange, dy, gain, route, saved):
    """Gradients [E, D] to the gains and [T, k] to the route's weights, for the gradient dy to the mixture's features."""
    import torch

    order, sent, owner, scaled = saved
    dscaled, dweights = exchange.combine_grad(dy, scaled, order, route.weights)
    dgain = torch.zeros_like(gain).index_add_(0, owner, dscaled.float() * sent.float())
    return dgain, dweights


def train(steps: int = 20, workers: int = 4, ratio: float = 16.0, tokens: int = 512, vocab: int = 5003, dim: int = 256, experts: int = 16,
          top_k: int = 2, teacher_k: int = 8, temperature: float = 2.0, lr: float = 4.0, seed: int = 0, mix: bool = False, clip: float = 0.0):
    """Returns the mean losses of each step: a list of (cross entropy, distillation, balance) and the counts per expert."""
    import torch

    from . import clipping, losses, routing
    from .binding import Pruner

    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    # the task: a teacher's head over the same features, whose best column is the target
    teacher = normal(vocab, dim) / dim**0.5
    batches = []
    for _ in range(workers):
        x = normal(tokens, dim).to(torch.bfloat16)
        top = torch.topk(4.0 * x.float() @ teacher.T, teacher_k, dim=1)
        batches.append((x, top.indices[:, 0].contiguous(), top.indices, top.values))

    sizes = [vocab * dim, experts * dim]  # one selection unit per tensor
    master = torch.cat([(normal(n) * 0.02) for n in sizes])
    if mix:
        sizes.append(experts * dim)
        master = torch.cat([master, torch.zeros(experts * dim, device=dev)])
    grads, update = torch.empty(workers, sum(sizes), device=dev), torch.empty(sum(sizes), device=dev)
    segments = [torch.split(grads[w], sizes) for w in range(workers)]
    pruner = Pruner(sizes, workers, ratio, 1e-8, seed)
    head, balance = losses.HeadLoss(tokens, vocab, dim, torch.bfloat16, top_k=teacher_k), losses.ExpertBalance(tokens, experts)
    router, exchange = routing.ExpertRouter(experts, top_k), routing.ExpertExchange(experts)
    clipper = clipping.GradientClip([s for row in segments for s in row], groups=[w for w in range(workers) for _ in sizes]) if clip else None
    history = []
    for _ in range(steps):
        weight, gate, *gain = (p.view(-1, dim) for p in torch.split(master, sizes))
        weight = weight.to(torch.bfloat16)
        grads.zero_()
        sums = torch.zeros(3, device=dev)
        counts = torch.zeros(experts, dtype=torch.int64, device=dev)
        for (x, targets, ids, logits), (into, dgate, *dgain) in zip(batches, segments):
            into = into.view(vocab, dim)
            scores = x.float() @ gate.T
            route = router.route(scores)
            bal = balance.grad(scores, route.ids, coef=1.0)
            if mix:
                y, saved = mixture(exchange, x, gain[0], route)
                ce = head.cross_entropy_grad(y, weight, targets, dhidden=torch.empty_like(y), dweight=into)
                d, dweights = mixture_grad(exchange, ce.dhidden, gain[0], route, saved)
                dgain[0].copy_(d.view(-1))
                router.grad(scores, route.ids, route.weights, dweights, dlogits=bal.dlogits, accumulate=True)
            else:
                ce = head.cross_entropy_grad(x, weight, targets, dweight=into, accumulate=True, want=("weight",))
            kd = head.distill_grad(x, weight, ids, logits, temperature, dweight=into, accumulate=True, want=("weight",))
            dgate.copy_((bal.dlogits.T @ x.float()).view(-1))
            sums += torch.stack([ce.loss, kd.loss, bal.loss])
            counts += bal.counts
        if clipper:
            clipper.clip(clip, drop_nonfinite=True)
        pruner.step(grads, master, update)
        master -= lr / workers * update
        history.append((sums / workers).tolist())
    pruner.check()
    head.check()
    balance.check()
    pruner.close()
    return history, counts.tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--ratio", type=float, default=16.0)
    ap.add_argument("--mixture", action="store_true", help="the experts scale the features that the head sees")
    ap.add_argument("--clip", type=float, default=0.0, help="largest norm of a worker's gradients (0: as they are)")
    a = ap.parse_args()
    history, counts = train(a.steps, a.workers, a.ratio, mix=a.mixture, clip=a.clip)
    for t, (ce, kd, bal) in enumerate(history):
        print(f"step {t:3d}  cross entropy {ce:.4f}  distillation {kd:.4f}  balance {bal:.4f}")
    print("tokens per expert in the last step:", counts)


if __name__ == "__main__":
    main()
