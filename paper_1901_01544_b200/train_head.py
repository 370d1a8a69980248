"""Example: W simulated workers train an output head and a router, their gradients reduced by the pruned step.

    python -m paper_1901_01544_b200.train_head [--steps 20] [--workers 4] [--ratio 16]

Every step each worker takes its own batch of features (fixed random ones here, where a model would compute them), adds
the cross entropy of its targets and the distillation from a teacher's top logits straight into its head segment of
grads[w], routes its tokens and takes the balance loss's gradient for the router's segment; `Pruner.step` then prunes,
reduces and leaves the rest in the workers' residuals, and plain gradient descent applies the update.
"""
from __future__ import annotations

import argparse


def train(steps: int = 20, workers: int = 4, ratio: float = 16.0, tokens: int = 512, vocab: int = 5003, dim: int = 256, experts: int = 16,
          top_k: int = 2, teacher_k: int = 8, temperature: float = 2.0, lr: float = 4.0, seed: int = 0):
    """Returns the mean losses of each step: a list of (cross entropy, distillation, balance) and the counts per expert."""
    import torch

    from . import losses
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
    grads, update = torch.empty(workers, sum(sizes), device=dev), torch.empty(sum(sizes), device=dev)
    pruner = Pruner(sizes, workers, ratio, 1e-8, seed)
    head, router = losses.HeadLoss(tokens, vocab, dim, torch.bfloat16, top_k=teacher_k), losses.ExpertBalance(tokens, experts)
    history = []
    for _ in range(steps):
        weight = master[: sizes[0]].view(vocab, dim).to(torch.bfloat16)
        gate = master[sizes[0] :].view(experts, dim)
        grads.zero_()
        sums = torch.zeros(3, device=dev)
        counts = torch.zeros(experts, dtype=torch.int64, device=dev)
        for w, (x, targets, ids, logits) in enumerate(batches):
            into = grads[w, : sizes[0]].view(vocab, dim)
            ce = head.cross_entropy_grad(x, weight, targets, dweight=into, accumulate=True, want=("weight",))
            kd = head.distill_grad(x, weight, ids, logits, temperature, dweight=into, accumulate=True, want=("weight",))
            scores = x.float() @ gate.T
            chosen = torch.topk(scores, top_k, dim=1).indices
            bal = router.grad(scores, chosen, coef=1.0)
            grads[w, sizes[0] :] = (bal.dlogits.T @ x.float()).reshape(-1)
            sums += torch.stack([ce.loss, kd.loss, bal.loss])
            counts += bal.counts
        pruner.step(grads, master, update)
        master -= lr / workers * update
        history.append((sums / workers).tolist())
    pruner.check()
    head.check()
    router.check()
    pruner.close()
    return history, counts.tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--ratio", type=float, default=16.0)
    a = ap.parse_args()
    history, counts = train(a.steps, a.workers, a.ratio)
    for t, (ce, kd, bal) in enumerate(history):
        print(f"step {t:3d}  cross entropy {ce:.4f}  distillation {kd:.4f}  balance {bal:.4f}")
    print("tokens per expert in the last step:", counts)


if __name__ == "__main__":
    main()
