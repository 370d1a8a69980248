"""Cases of the operators around the training losses: routing tokens to experts, exchanging rows with the experts, norms and
clipping of gradients.

`own` selects between the plain forms below (elementary torch operations in 32 bits, 64 where a choice or a long sum needs
them) and the library's kernels."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    def route(name, T, E, k, score, dtype, grad, masked=False, bias=False, groups=1, top_groups=1, renormalize=True, weight_scale=1.0):
        return {"name": name, "op": "route", "T": T, "E": E, "k": k, "score": score, "dtype": dtype, "grad": grad, "masked": masked, "bias": bias,
                "groups": groups, "top_groups": top_groups, "renormalize": renormalize, "weight_scale": weight_scale}

    def exchange(name, T, D, E, k, dtype, grad, masked=False):
        return {"name": name, "op": "exchange", "T": T, "D": D, "E": E, "k": k, "dtype": dtype, "grad": grad, "masked": masked}

    def clip(name, tensors, dtype, **kw):
        case = {"name": name, "op": "clip", "tensors": tensors, "dtype": dtype, "into": "", "groups": 1, "ratio": 0.25, "scale": 1.0, "offset": 0}
        return case | kw

    return [
        # one router on a handful of tokens, scores only: latency
        route("route_few_tokens", 64, 8, 2, "softmax", "fp32", False),
        # odd counts, a padded batch, softmax scores taken as they are: the gradient reaches every logit
        route("route_train_padded", 5003, 60, 4, "softmax", "fp16", True, masked=True, renormalize=False),
        # a worker's batch on many experts in groups, sigmoid scores, a bias that balances
        route("route_train_groups", 16384, 256, 8, "sigmoid", "bf16", True, bias=True, groups=8, top_groups=4, weight_scale=2.5),
        # the longest batch, router kept in fp32
        route("route_train_large", 131072, 256, 8, "softmax", "fp32", True, masked=True),
        # rows of a handful of tokens to their experts and back: latency
        exchange("exchange_few_tokens", 64, 1024, 8, 2, "bf16", False),
        # odd counts, a padded batch, a width that no power of two divides
        exchange("exchange_train_ragged", 1021, 1032, 60, 4, "fp16", True, masked=True),
        # a worker's batch
        exchange("exchange_train_large", 16384, 4096, 128, 8, "bf16", True),
        # a router's gate and two vectors: latency
        clip("clip_few_small", "small", "fp32"),
        # the classic worker of the pruned step: its model's gradients, clipped, into its fp32 segment
        clip("clip_resnet50_to_segment", "resnet50", "bf16", into="fp32"),
        # one norm per tensor, as a monitor of training asks for them
        clip("norm_resnet50_tensors", "resnet50", "fp32", groups=161, ratio=0.0),
        # odd sizes, segments that start anywhere, loss-scaled fp16
        clip("clip_ragged_scaled", "ragged", "fp16", into="fp32", scale=1.0 / 1024, offset=1),
        # eight workers' gradients, each worker clipped by its own norm
        clip("clip_alexnet_workers", "alexnet", "fp32", into="fp32", groups=8),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "exchange", "clip"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if op == "route":
        groups = rng.choice([1, 1, 1, 2, 4, 5, 8])
        E = groups * max(2, _log_uniform(rng, 8, 512) // groups)
        T = min(_log_uniform(rng, 1, 131072), 131072 * 256 // E)
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(8, top_groups * (E // groups)))
        return {"op": op, "T": T, "E": E, "k": k, "score": rng.choice(["softmax", "sigmoid"]), "dtype": dtype, "grad": rng.random() < 0.7,
                "masked": rng.random() < 0.5, "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups,
                "renormalize": rng.random() < 0.7, "weight_scale": rng.choice([1.0, 2.5])}
    if op == "exchange":
        T, D, E = _log_uniform(rng, 1, 16384), _log_uniform(rng, 32, 4096), _log_uniform(rng, 8, 256)
        if rng.random() < 0.8:  # most models have a width that 8 divides
            D = max(32, D // 8 * 8)
        case = {"op": op, "T": T, "D": D, "E": E, "k": rng.randint(1, 8), "dtype": dtype, "grad": rng.random() < 0.7, "masked": rng.random() < 0.5}
        if dtype == "fp32":
            case["D"] = max(16, D // 2)
        return case
    groups = rng.choice([1, 1, 2, 4, 8])
    count, total = _log_uniform(rng, groups, 200), _log_uniform(rng, 1000, 300_000_000)
    return {"op": op, "tensors": f"{count}x{total}", "dtype": dtype, "into": rng.choice(["", dtype, "fp32"]) if count > groups else dtype,
            "groups": groups, "ratio": rng.choice([0.25, 0.5, 4.0]), "scale": rng.choice([1.0, 1.0, 1.0 / 1024]), "offset": rng.choice([0, 0, 1])}


def _resnet50():
    """Sizes of ResNet-50's tensors in module order: convolutions with their two vectors, then the classifier."""
    out = [64 * 3 * 49, 64, 64]
    inside = 64
    for planes, blocks in zip((64, 128, 256, 512), (3, 4, 6, 3)):
        for b in range(blocks):
            convs = [(planes, inside, 1), (planes, planes, 9), (planes * 4, planes, 1)] + ([(planes * 4, inside, 1)] if b == 0 else [])
            for cout, cin, taps in convs:
                out += [cout * cin * taps, cout, cout]
            inside = planes * 4
    return out + [1000 * 2048, 1000]


def _alexnet():
    out = []
    for rows, columns in [(96, 3 * 121), (256, 48 * 25), (384, 256 * 9), (384, 192 * 9), (256, 192 * 9), (4096, 9216), (4096, 4096), (1000, 4096)]:
        out += [rows * columns, rows]
    return out


def _sizes(case):
    """(size, group) of every tensor."""
    kind, G = case["tensors"], case["groups"]
    if kind == "small":
        return [(16 * 256, 0), (1000, 0), (64, 0)]
    if kind == "resnet50":
        return [(n, i if G > 1 else 0) for i, n in enumerate(_resnet50())]
    if kind == "alexnet":
        return [(n, w) for w in range(G) for n in _alexnet()]
    if kind == "ragged":
        return [(1003 * 257, 0), (31, 0), (7, 0), (640 * 1021 + 3, 0), (1, 0), (2048 * 1999, 0), (255, 0)]
    count, total = (int(x) for x in kind.split("x"))
    share = [1 + (i * 2654435761 % 1000) ** 2 for i in range(count)]  # sizes of very different order
    return [(max(1, total * s // sum(share)), i * G // count) for i, s in enumerate(share)]


def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        moved = T * E * size + 8 * T * k + 4 * E + (T if case["masked"] else 0) + (4 * E if case["bias"] else 0)
        if case["grad"]:
            moved += T * E * size + 4 * T * k
        return {"bytes": moved, "flops": (8 if case["grad"] else 5) * T * E}
    if case["op"] == "exchange":
        T, D, k, E = case["T"], case["D"], case["k"], case["E"]
        once, rows = T * D * size, T * k * D * size
        # ids, offsets, slots, rows, weights; x -> dispatched, z -> y; dy -> dz, dispatched gradient -> dx
        moved = 4 * T * k * 4 + 4 * (E + 1) + 2 * (once + rows)
        flops = 2 * T * k * D
        if case["grad"]:
            moved += 2 * (once + rows) + 4 * T * k
            flops *= 3
        return {"bytes": moved, "flops": flops}
    n = sum(s for s, _ in _sizes(case))
    written = 0 if case["ratio"] == 0 or not case["into"] else n * SIZE[case["into"]]
    return {"bytes": n * size + written + 8 * case["groups"], "flops": 3 * n}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    state = {"case": case}
    if case["op"] == "clip":
        sizes = _sizes(case)
        off = case["offset"]
        # every tensor has its own scale, as layers do; tensors that carry an offset are views into a larger buffer
        spread = [10.0 ** (-4 + 2 * u) for u in uniform(len(sizes)).tolist()]
        state["tensors"] = [(normal(n + off) * s / case["scale"]).to(dtype)[off:] for (n, _), s in zip(sizes, spread)]
        squares = [0.0] * case["groups"]
        for (n, w), s in zip(sizes, spread):
            squares[w] += n * s * s
        state["max_norm"] = case["ratio"] * math.sqrt(sum(squares) / len(squares))
        state["group"] = [w for _, w in sizes]
        into = None
        if case["into"]:
            # the worker's segment: the tensors one after another
            flat = torch.zeros(off + sum(n for n, _ in sizes), dtype=TYPES[case["into"]], device="cuda")[off:]
            into = list(torch.split(flat, [n for n, _ in sizes]))
            state["flat"], state["into"] = flat, into
        if own:
            from paper_1901_01544_b200 import clipping

            state["plan"] = clipping.GradientClip(state["tensors"], into=into, groups=state["group"])
        return state
    T, E, k = case["T"], case["E"], case["k"]
    # a router in training: some experts are preferred by everybody, the rest is the token's own
    logits = normal(T, E) + 0.7 * normal(E)
    if case["op"] == "route":
        state["logits"] = logits.to(dtype)
        state["bias"] = 0.05 * normal(E) if case["bias"] else None
        state["mask"] = uniform(T) < 0.9 if case["masked"] else None
        state["dweights"] = normal(T, k) * (16.0 if case["dtype"] == "fp16" else 0.25)  # fp16 training scales its loss
        if own:
            from paper_1901_01544_b200 import routing

            state["plan"] = routing.ExpertRouter(E, k, score=case["score"], groups=case["groups"], top_groups=case["top_groups"],
                                                 renormalize=case["renormalize"], weight_scale=case["weight_scale"])
        return state
    D = case["D"]
    top = torch.sort(logits, dim=1, descending=True).values
    ids = torch.argsort(logits, dim=1, descending=True)[:, :k].int()
    state["ids"] = ids
    state["weights"] = torch.softmax(top[:, :k], 1).contiguous()
    if case["masked"]:
        gone = uniform(T) >= 0.9  # padding: no expert, no weight
        ids[gone], state["weights"][gone] = -1, 0.0
    state["x"], state["z"] = normal(T, D).to(dtype), normal(T * k, D).to(dtype)
    if case["grad"]:
        state["dy"], state["dx_rows"] = normal(T, D).to(dtype), normal(T * k, D).to(dtype)
    if own:
        from paper_1901_01544_b200 import routing

        state["plan"] = routing.ExpertExchange(E)
    return state


def run(state):
    op = state["case"]["op"]
    if op == "route":
        return _route_own(state) if own else _route_plain(state)
    if op == "exchange":
        return _exchange_own(state) if own else _exchange_plain(state)
    return _clip_own(state) if own else _clip_plain(state)


# ---- the library's kernels ---------------------------------------------------------------------


def _route_own(state):
    plan, x = state["plan"], state["logits"]
    r = plan.route(x, state["bias"], state["mask"])
    out = {"ids": r.ids, "weights": r.weights, "counts": r.counts}
    if state["case"]["grad"]:
        out["dlogits"] = plan.grad(x, r.ids, r.weights, state["dweights"])
    return out


def _exchange_own(state):
    plan = state["plan"]
    order = plan.order(state["ids"])
    out = {"offsets": order.offsets, "slots": order.slots, "rows": order.rows}
    out["sent"] = plan.dispatch(state["x"], order)
    out["y"] = plan.combine(state["z"], order, state["weights"])
    if state["case"]["grad"]:
        out["dz"], out["dweights"] = plan.combine_grad(state["dy"], state["z"], order, state["weights"])
        out["dx"] = plan.dispatch_grad(state["dx_rows"], order)
    return out


def _clip_own(state):
    plan, case = state["plan"], state["case"]
    if case["ratio"] == 0 or not case["into"]:
        return {"norms": plan.norm(scale=case["scale"]).norms}
    r = plan.clip(state["max_norm"], scale=case["scale"])
    return {"norms": r.norms, "factors": r.factors, "grads": state["flat"]}


# ---- the plain forms ---------------------------------------------------------------------------


def _route_plain(state):
    case, x, mask = state["case"], state["logits"].float(), state["mask"]
    (T, E), k, G = x.shape, case["k"], case["groups"]
    e64 = torch.exp(x.double() - x.double().amax(1, keepdim=True)) if case["score"] == "softmax" else None
    # the choice is made in 64 bits: neighbours may be closer than 32 bits tell apart
    c = e64 / e64.sum(1, keepdim=True) if case["score"] == "softmax" else 1.0 / (1.0 + torch.exp(-x.double()))
    s = c.float()
    if case["bias"]:
        c = c + state["bias"].double()
    if G > 1:
        by_group = torch.sort(c.view(T, G, E // G), dim=2, descending=True).values
        score = by_group[:, :, 0] + by_group[:, :, 1]
        kept = torch.sort(score, dim=1, descending=True, stable=True).indices[:, : case["top_groups"]]
        open_groups = torch.zeros(T, G, dtype=torch.bool, device=x.device).scatter_(1, kept, True)
        c = torch.where(open_groups[:, :, None].expand(T, G, E // G).reshape(T, E), c, -math.inf)
    ids = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
    chosen = torch.gather(s, 1, ids)
    total = chosen.sum(1, keepdim=True)
    p = chosen / total if case["renormalize"] else chosen
    if mask is not None:
        p = p * mask[:, None].float()
    weights = p * case["weight_scale"]
    kept = ids if mask is None else torch.where(mask[:, None], ids, E)
    counts = torch.bincount(kept.reshape(-1), minlength=E + 1)[:E]
    out = {"ids": torch.where(kept == E, -1, kept).int(), "weights": weights, "counts": counts.int()}
    if case["grad"]:
        dw = state["dweights"]
        dots = (dw * weights).sum(1, keepdim=True)
        if case["score"] == "softmax":
            dx = torch.zeros_like(x) if case["renormalize"] else -s * dots
            at = weights * dw - (p * dots if case["renormalize"] else 0.0)
        else:
            dx = torch.zeros_like(x)
            at = (weights * dw - (p * dots if case["renormalize"] else 0.0)) * (1.0 / (1.0 + torch.exp(torch.gather(x, 1, ids))))
        out["dlogits"] = dx.scatter_add(1, ids, at).to(state["logits"].dtype)
    return out


def _exchange_plain(state):
    case, ids, w = state["case"], state["ids"].long(), state["weights"]
    (T, k), E, D, dtype = ids.shape, case["E"], case["D"], state["x"].dtype
    key = torch.where(ids < 0, E, ids).reshape(-1)
    pairs = torch.sort(key, stable=True).indices  # by expert, then by token
    counts = torch.bincount(key, minlength=E + 1)
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts[:E], 0)])
    live = torch.arange(T * k, device=ids.device) < offsets[E]
    rows = torch.where(live, pairs // k, -1)
    slots = torch.empty_like(pairs)
    slots[pairs] = torch.arange(T * k, device=ids.device)
    slots = torch.where(key < E, slots, -1).view(T, k)
    x, z = state["x"].float(), state["z"].float()
    out = {"offsets": offsets.int(), "slots": slots.int(), "rows": rows.int()}
    out["sent"] = torch.where(live[:, None], x[rows.clamp(min=0)], 0.0).to(dtype)
    on = (slots >= 0).float()
    y = torch.zeros(T, D, device=ids.device)
    for j in range(k):
        y += (w[:, j] * on[:, j])[:, None] * z[slots[:, j].clamp(min=0)]
    out["y"] = y.to(dtype)
    if case["grad"]:
        dy, back = state["dy"].float(), state["dx_rows"].float()
        by_slot = torch.where(live, w.reshape(-1)[pairs], 0.0)
        dz = by_slot[:, None] * dy[rows.clamp(min=0)]
        dw, dx = torch.zeros(T, k, device=ids.device), torch.zeros(T, D, device=ids.device)
        for j in range(k):
            at = slots[:, j].clamp(min=0)
            dw[:, j] = on[:, j] * (dy * z[at]).sum(1)
            dx += on[:, j, None] * back[at]
        out |= {"dz": dz.to(dtype), "dweights": dw, "dx": dx.to(dtype)}
    return out


def _clip_plain(state):
    case, device = state["case"], state["tensors"][0].device
    squares = torch.zeros(case["groups"], dtype=torch.float64, device=device)
    for x, w in zip(state["tensors"], state["group"]):
        y = x.float()
        squares[w] += (y * y).sum(dtype=torch.float64)
    norms = torch.sqrt(squares) * case["scale"]
    if case["ratio"] == 0 or not case["into"]:
        return {"norms": norms.float()}
    limit = state["max_norm"]
    factors = (torch.where(norms > limit, limit / norms, 1.0) * case["scale"]).float()
    for x, to, w in zip(state["tensors"], state["into"], state["group"]):
        to.copy_(x.float() * factors[w])
    return {"norms": norms.float(), "factors": factors, "grads": state["flat"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    return {"route": _route_exact, "exchange": _exchange_exact, "clip": _clip_exact}[case["op"]](state)


def _route_exact(state):
    case, x, k = state["case"], state["logits"].double(), state["case"]["k"]
    T, E = x.shape
    on = torch.ones(T, dtype=torch.bool, device=x.device) if state["mask"] is None else state["mask"]
    s = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
    c = s.clone() if state["bias"] is None else s + state["bias"]
    G, size = case["groups"], E // case["groups"]
    if G > 1:
        best = torch.stack([torch.topk(c[:, q * size : (q + 1) * size], 2, dim=1).values.sum(1) for q in range(G)], 1)
        for q in range(G):
            ahead = (best > best[:, q : q + 1]).sum(1) + (best[:, :q] == best[:, q : q + 1]).sum(1)
            c[ahead >= case["top_groups"], q * size : (q + 1) * size] = -math.inf
    column = torch.arange(E, device=x.device)
    ids = []
    for _ in range(k):
        first = torch.where(c == c.amax(1, keepdim=True), column, E).amin(1)
        ids.append(first)
        c[torch.arange(T, device=x.device), first] = -math.inf
    ids = torch.stack(ids, 1)
    chosen = torch.zeros(T, E, dtype=torch.bool, device=x.device).scatter_(1, ids, True) & on[:, None]
    w = torch.gather(s, 1, ids)
    S = w.sum(1, keepdim=True) if case["renormalize"] else 1.0
    w = case["weight_scale"] * w / S * on[:, None]
    out = {"ids": torch.where(on[:, None], ids, -1).int(), "weights": w, "counts": chosen.sum(0).int()}
    if case["grad"]:
        # through the chosen scores, then through the scores' own function
        up = torch.zeros_like(x).scatter_(1, ids, state["dweights"].double()) * chosen * case["weight_scale"]
        if case["renormalize"]:
            up = (up - (up * s / S).sum(1, keepdim=True)) / S * chosen
        out["dlogits"] = s * (up - (up * s).sum(1, keepdim=True)) if case["score"] == "softmax" else up * s * (1.0 - s)
    return out


def _exchange_exact(state):
    case, ids = state["case"], state["ids"].long()
    (T, k), E, D = ids.shape, case["E"], case["D"]
    # expert by expert: the pairs of an expert in the order of their tokens
    lists = [(ids == e).reshape(-1).nonzero()[:, 0] for e in range(E)]
    pairs = torch.cat(lists)
    n = pairs.numel()
    offsets = torch.tensor([0] + [p.numel() for p in lists], device=ids.device).cumsum(0)
    rows = torch.full((T * k,), -1, device=ids.device)
    rows[:n] = torch.div(pairs, k, rounding_mode="floor")
    slots = torch.full((T * k,), -1, device=ids.device)
    slots[pairs] = torch.arange(n, device=ids.device)
    token = rows[:n]
    w = state["weights"].double().reshape(-1)[pairs]
    out = {"offsets": offsets.int(), "slots": slots.view(T, k).int(), "rows": rows.int()}

    def padded(m):
        return torch.cat([m, m.new_zeros(T * k - n, D)]) if n < T * k else m

    def summed(values, factor):
        total = torch.zeros(T, D, dtype=torch.float64, device=ids.device)
        for a in range(0, n, 16384):  # in pieces, for the memory of 64-bit rows
            part = values[a : min(n, a + 16384)].double()
            total.index_add_(0, token[a : a + 16384], part if factor is None else part * factor[a : a + 16384, None])
        return total

    out["sent"] = padded(state["x"][token])
    out["y"] = summed(state["z"], w)
    if case["grad"]:
        dz, dots = [], []
        for a in range(0, n, 16384):
            d = state["dy"][token[a : a + 16384]].double()
            dz.append(d * w[a : a + 16384, None])
            dots.append((d * state["z"][a : min(n, a + 16384)].double()).sum(1))
        out["dz"] = padded(torch.cat(dz) if dz else torch.zeros(0, D, dtype=torch.float64, device=ids.device))
        dw = torch.zeros(T * k, dtype=torch.float64, device=ids.device)
        if n:
            dw[pairs] = torch.cat(dots)
        out["dweights"] = dw.view(T, k)
        out["dx"] = summed(state["dx_rows"], None)
    return out


def _clip_exact(state):
    case = state["case"]
    norms = []
    for w in range(case["groups"]):
        parts = [torch.linalg.vector_norm(x.double()) for x, v in zip(state["tensors"], state["group"]) if v == w]
        norms.append(torch.linalg.vector_norm(torch.stack(parts)) * case["scale"])
    norms = torch.stack(norms)
    if case["ratio"] == 0 or not case["into"]:
        return {"norms": norms}
    factors = torch.clamp(state["max_norm"] / norms, max=1.0) * case["scale"]
    return {"norms": norms, "factors": factors, "grads": torch.cat([x.double() * factors[w] for x, w in zip(state["tensors"], state["group"])])}
