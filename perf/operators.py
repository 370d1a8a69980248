"""Cases of the training losses: output head with cross entropy, output head with a teacher's top logits, balance loss of a router.

`own` selects between the plain forms below (elementary torch operations in 32 bits) and the library's kernels."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
IGNORE = -100  # target of a token that carries no loss (padding, prompt)


def listed():
    def ce(name, T, V, D, dtype, grad):
        return {"name": name, "op": "cross_entropy", "T": T, "V": V, "D": D, "dtype": dtype, "grad": grad}

    def kd(name, T, V, D, K, tau, dtype, grad):
        return {"name": name, "op": "distill", "T": T, "V": V, "D": D, "K": K, "tau": tau, "dtype": dtype, "grad": grad}

    def bal(name, T, E, k, dtype, masked):
        return {"name": name, "op": "balance", "T": T, "E": E, "k": k, "dtype": dtype, "masked": masked}

    return [
        # the log-probability of one token, as a scorer asks for it: latency, and the head's weights read once
        ce("ce_score_one_token", 1, 32768, 1024, "bf16", False),
        # the classifier head of ResNet-50 (2048 x 1000) on a worker's batch
        ce("ce_train_classifier", 256, 1000, 2048, "bf16", True),
        # a validation batch: losses only
        ce("ce_eval_batch", 4096, 65536, 2048, "bf16", False),
        # a packed batch of odd length, a vocabulary that no tile divides, loss-scaled fp16
        ce("ce_train_ragged", 1021, 50021, 1032, "fp16", True),
        # a worker's batch on a large vocabulary
        ce("ce_train_large", 8192, 131072, 4096, "bf16", True),
        # distillation of a small head on a short batch
        kd("kd_train_short", 40, 8192, 512, 16, 1.0, "bf16", True),
        # odd sizes, odd number of teacher logits, fp16
        kd("kd_train_ragged", 777, 32003, 1536, 50, 1.5, "fp16", True),
        # an ordinary distillation step
        kd("kd_train_batch", 4096, 32768, 2048, 64, 2.0, "bf16", True),
        # one router on a handful of tokens: latency
        bal("balance_few_tokens", 64, 8, 2, "fp32", False),
        # odd counts, padded batch
        bal("balance_padded", 5003, 60, 4, "fp16", True),
        # a worker's batch on many experts
        bal("balance_batch", 16384, 128, 8, "bf16", False),
        # the longest batch, router kept in fp32
        bal("balance_large", 131072, 256, 8, "fp32", True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cross_entropy", "distill", "balance"])
    if op == "balance":
        E = _log_uniform(rng, 8, 256)
        return {"op": op, "T": _log_uniform(rng, 1, 131072), "E": E, "k": rng.randint(1, min(8, E)),
                "dtype": rng.choice(["fp32", "bf16", "fp16"]), "masked": rng.random() < 0.5}
    T, V, D = _log_uniform(rng, 1, 8192), _log_uniform(rng, 1000, 131072), _log_uniform(rng, 64, 4096)
    if rng.random() < 0.8:  # most models have a width that 8 divides
        D = max(64, D // 8 * 8)
    case = {"op": op, "T": T, "V": V, "D": D, "dtype": rng.choice(["bf16", "fp16"]), "grad": rng.random() < 0.7}
    if op == "distill":
        case |= {"K": rng.randint(1, 64), "tau": rng.choice([1.0, 1.5, 2.0, 4.0])}
    return case


def work(case):
    if case["op"] == "balance":
        T, E, k, size = case["T"], case["E"], case["k"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": 2 * T * E * size + 8 * T * k + (T if case["masked"] else 0) + 8 * E + 4, "flops": 8 * T * E}
    T, V, D, K = case["T"], case["V"], case["D"], case.get("K", 0)
    operands = 2 * (T * D + V * D)
    products = 3 if case["grad"] else 1
    return {"bytes": operands * (2 if case["grad"] else 1) + T * K * 12 + (0 if K else 8 * T) + 8 * T, "flops": products * 2 * T * V * D}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    T = case["T"]
    if case["op"] == "balance":
        E, k = case["E"], case["k"]
        # a router in training: some experts are preferred by everybody, the rest is the token's own
        logits = (normal(T, E) + 0.7 * normal(E)).to(dtype)
        experts = torch.sort(logits.float(), dim=1, descending=True, stable=True).indices[:, :k].contiguous()
        mask = uniform(T) < 0.9 if case["masked"] else None
        state = {"logits": logits, "experts": experts, "mask": mask, "coef": 0.01, "case": case}
        state["scale"] = 16384.0 if case["dtype"] == "fp16" else 1.0  # fp16 training scales its loss
        if own:
            from paper_1901_01544_b200 import losses

            state["plan"] = losses.ExpertBalance(T, E)
        return state
    V, D, K = case["V"], case["D"], case.get("K", 0)
    weight = normal(V, D).mul_(2.0 / math.sqrt(D)).to(dtype)
    # frequent tokens are frequent (a power law), and the model already knows some of its targets
    targets = (V * uniform(T) ** 3).long().clamp_(max=V - 1)
    hidden = (normal(T, D) + 2.5 * uniform(T, 1) * weight[targets].float()).to(dtype)
    # fp16 training scales its loss so that small gradients stay above the type's smallest value
    state = {"hidden": hidden, "weight": weight, "scale": 1024.0 if case["dtype"] == "fp16" else 1.0, "case": case}
    if K:
        # the teacher's K largest logits and where they are: distinct tokens in descending order of their logit
        gaps = torch.randint(1, max(2, V // K), (T, K), generator=g, device="cuda")
        ids = torch.cumsum(gaps, 1) - 1
        order = torch.argsort(uniform(T, K), dim=1)
        state["top_ids"] = torch.gather(ids, 1, order)
        state["top_logits"] = (12.0 + normal(T, 1) - torch.cumsum(uniform(T, K), 1) * 0.5).to(dtype)
    else:
        targets[uniform(T) < (0.05 if T > 1 else 0.0)] = IGNORE
        state["targets"] = targets
    if own:
        from paper_1901_01544_b200 import losses

        state["plan"] = losses.HeadLoss(T, V, D, dtype, top_k=max(1, K))
    return state


def run(state):
    case = state["case"]
    if case["op"] == "balance":
        return _balance_own(state) if own else _balance_plain(state)
    return _head_own(state) if own else _head_plain(state)


# ---- the library's kernels ---------------------------------------------------------------------


def _balance_own(state):
    r = state["plan"].grad(state["logits"], state["experts"], state["mask"], coef=state["coef"], scale=state["scale"])
    return {"loss": r.loss, "counts": r.counts, "dlogits": r.dlogits}


def _head_own(state):
    case, plan = state["case"], state["plan"]
    if case["op"] == "cross_entropy":
        what = (state["hidden"], state["weight"], state["targets"])
        r = plan.cross_entropy_grad(*what, ignore_index=IGNORE, scale=state["scale"]) if case["grad"] else plan.cross_entropy(*what, ignore_index=IGNORE)
    else:
        what = (state["hidden"], state["weight"], state["top_ids"], state["top_logits"], case["tau"])
        r = plan.distill_grad(*what, scale=state["scale"]) if case["grad"] else plan.distill(*what)
    out = {"loss": r.loss, "rows": r.rows, "lse": r.lse}
    return out | {"dhidden": r.dhidden, "dweight": r.dweight} if case["grad"] else out


# ---- the plain forms ---------------------------------------------------------------------------


def _balance_plain(state):
    x, experts, mask = state["logits"].float(), state["experts"], state["mask"]
    (T, E), k = x.shape, experts.shape[1]
    m = torch.ones(T, device=x.device) if mask is None else mask.float()
    e = torch.exp(x - x.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    n = m.sum().clamp(min=1.0)
    kept = experts if mask is None else torch.where(mask[:, None], experts, E)
    counts = torch.bincount(kept.reshape(-1), minlength=E + 1)[:E]
    f = counts.float() / (n * k)
    c = state["coef"] * E
    loss = c * (f * ((p * m[:, None]).sum(0) / n)).sum()
    dx = (state["scale"] * c / n) * m[:, None] * p * (f - (p * f).sum(1, keepdim=True))
    return {"loss": loss, "counts": counts.int(), "dlogits": dx.to(state["logits"].dtype)}


def _head_plain(state):
    case, h, w = state["case"], state["hidden"].float(), state["weight"].float()
    dtype = state["hidden"].dtype
    if case["op"] == "cross_entropy":
        tau = 1.0
        valid = (state["targets"] != IGNORE).float()
        ids = state["targets"].clamp(min=0)[:, None]
        q = valid[:, None]
        entropy = torch.zeros_like(valid)
    else:
        tau = case["tau"]
        ids = state["top_ids"]
        t = state["top_logits"].float() / tau
        e = torch.exp(t - t.amax(1, keepdim=True))
        q = e / e.sum(1, keepdim=True)
        valid = torch.ones_like(q[:, 0])
        entropy = (q * torch.where(q > 0, torch.log(q), 0.0)).sum(1)
    z = (h @ w.T) / tau
    top = z.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    rows = tau * tau * (entropy - (q * torch.gather(z, 1, ids)).sum(1) + lse * valid)
    n = valid.sum().clamp(min=1.0)
    out = {"loss": rows.sum() / n, "rows": rows, "lse": lse}
    if not case["grad"]:
        return out
    dz = torch.exp(z - lse[:, None]) * valid[:, None]
    dz = dz.scatter_add(1, ids, -q) * (tau * state["scale"] / n)
    return out | {"dhidden": (dz @ w).to(dtype), "dweight": (dz.T @ h).to(dtype)}


# ---- the definitions in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    return _balance_exact(state) if case["op"] == "balance" else _head_exact(state)


def _balance_exact(state):
    x, experts, mask = state["logits"].double(), state["experts"], state["mask"]
    (T, E), k = x.shape, experts.shape[1]
    if mask is not None:
        rows = mask.nonzero()[:, 0]
        x, experts = x[rows], experts[rows]
    n = x.shape[0]
    counts = torch.stack([(experts == e).sum() for e in range(E)])
    dlogits = torch.zeros(T, E, dtype=torch.float64, device=x.device)
    if n == 0:
        return {"loss": torch.zeros((), dtype=torch.float64), "counts": counts.int(), "dlogits": dlogits}
    p = torch.softmax(x, 1)
    share = counts.double() / (n * k)
    slope = state["coef"] * E * share / n  # of the loss to each token's probability
    loss = (p @ slope).sum()
    dx = state["scale"] * p * (slope - (p @ slope)[:, None])
    if mask is None:
        dlogits = dx
    else:
        dlogits[rows] = dx
    return {"loss": loss, "counts": counts.int(), "dlogits": dlogits}


def _head_exact(state):
    """The vocabulary in slices, 64 bits throughout."""
    case, h, weight = state["case"], state["hidden"].double(), state["weight"]
    (T, D), V = h.shape, weight.shape[0]
    if case["op"] == "cross_entropy":
        tau, ids = 1.0, state["targets"][:, None]
        q = (ids != IGNORE).double()
        logq = torch.zeros_like(q)
    else:
        tau, ids = float(case["tau"]), state["top_ids"]
        logq = torch.log_softmax(state["top_logits"].double() / tau, 1)
        q = torch.exp(logq)
    live = q.sum(1) > 0
    n = max(1, int(live.sum()))
    step = 8192
    spans = [(a, min(V, a + step)) for a in range(0, V, step)]
    lse = torch.full((T,), -math.inf, dtype=torch.float64, device=h.device)
    at = torch.zeros_like(q)  # the logits at the targets
    for a, b in spans:
        z = h @ weight[a:b].double().T / tau
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
        here = (ids >= a) & (ids < b)
        at += torch.where(here, torch.gather(z, 1, (ids - a).clamp(0, b - a - 1)), 0.0)
    rows = tau * tau * (q * (logq - at + lse[:, None])).sum(1)
    out = {"loss": rows.sum() / n, "rows": rows, "lse": lse}
    if not case["grad"]:
        return out
    g = tau * state["scale"] / n
    dhidden = torch.zeros_like(h)
    dweight = torch.empty(V, D, dtype=torch.float64, device=h.device)
    for a, b in spans:
        w = weight[a:b].double()
        p = torch.exp(h @ w.T / tau - lse[:, None]) * live[:, None]
        here = (ids >= a) & (ids < b)
        p.scatter_add_(1, (ids - a).clamp(0, b - a - 1), torch.where(here, -q, 0.0))
        p *= g
        dhidden += p @ w
        dweight[a:b] = p.T @ h
    return out | {"dhidden": dhidden, "dweight": dweight}
