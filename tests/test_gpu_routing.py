"""The router (choice of experts, weights, gradient to the logits) and the exchange of rows with the experts, against plain
64-bit statements of their formulas.

Roundings: h(t) = finfo(t).eps / 2 is the relative error of one rounding to t.  A weight is a ratio of exponentials: an
argument's rounding (its size times h), two units in the last place of exp (4 h), sums of at most 64 terms in a row (64 h)
and two products, in numerator and denominator."""
import math

import pytest
import torch

from paper_1901_01544_b200 import losses, routing

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF, FP = torch.float32, torch.bfloat16, torch.float16
U = 2.0**-24


def half(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def plain(x, k, score="softmax", bias=None, mask=None, groups=1, top_groups=1, group_top=2, renormalize=True, weight_scale=1.0):
    """(ids, weights, scores) in 64 bits; sorts are stable, so ties go to the lower expert."""
    T, E = x.shape
    x = x.double()
    on = torch.ones(T, dtype=torch.bool, device=x.device) if mask is None else mask.bool()
    bad = torch.isnan(x).any(1) | ((x == math.inf).any(1) if score == "softmax" else False)
    s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
    s = torch.where(x == -math.inf, 0.0, s)
    c = s if bias is None else s + bias.double()
    c = torch.where((x == -math.inf) | torch.isnan(c), -math.inf, c)
    open_groups = torch.ones(T, groups, dtype=torch.bool, device=x.device)
    if top_groups < groups:
        by = x if bias is None and group_top == 1 else c
        top = torch.sort(by.view(T, groups, E // groups), dim=2, descending=True).values[:, :, :group_top].sum(2)
        kept = torch.sort(top, dim=1, descending=True, stable=True).indices[:, :top_groups]
        open_groups = torch.zeros_like(open_groups).scatter_(1, kept, True)
    if bias is None:
        c = torch.where(c > -math.inf, x, c)
    c = torch.where(open_groups[:, :, None].expand(T, groups, E // groups).reshape(T, E), c, -math.inf)
    order = torch.sort(c, dim=1, descending=True, stable=True)
    ids, there = order.indices[:, :k], (order.values[:, :k] > -math.inf) & (on & ~bad)[:, None]
    logs = torch.nn.functional.logsigmoid(x) if score == "sigmoid" else torch.log_softmax(x, 1)
    chosen = torch.where(there, torch.gather(logs, 1, ids), -math.inf)
    if renormalize:
        p = torch.where(there, torch.softmax(chosen, 1), 0.0)
    else:
        p = torch.exp(chosen)
    weights = torch.where((bad & on)[:, None], math.nan, weight_scale * p)
    return torch.where(there, ids, -1), weights, s


def slack(x, ids):
    """Bound of a weight's relative error (see above), by row."""
    y = torch.where(ids >= 0, torch.gather(x.double(), 1, ids.clamp(min=0)), torch.nan)
    top = x.double().masked_fill(x == math.inf, 0).amax(1, keepdim=True).clamp(min=-1e4, max=1e4)
    far = torch.nan_to_num((top - y).abs(), nan=0.0).amax(1, keepdim=True).clamp(max=200.0)
    return (2 * far + 2 * 4 + 2 * 64 + 8) * U


def check_route(plan, x, bias=None, mask=None, **kw):
    r = plan.route(x, bias, mask)
    ids, w, _ = plain(x, plan.top_k, bias=bias, mask=mask, **kw)
    assert torch.equal(r.ids.long(), ids)
    ok = torch.isnan(w)
    assert torch.equal(torch.isnan(r.weights), ok)
    err = (r.weights.double() - w).abs()
    # (a score below fp32's normal range keeps fewer bits)
    assert ((err <= slack(x, ids) * w.abs() + 2.0**-126) | ok).all(), (err / w.abs()).nan_to_num().max()
    assert torch.equal(r.counts.long(), torch.bincount(ids[ids >= 0], minlength=plan.experts))
    return r


FORMS = [
    dict(score="softmax"), dict(score="sigmoid"), dict(score="softmax", renormalize=False, weight_scale=2.5), dict(score="sigmoid", renormalize=False),
]
SIZES = [(1, 1, 1), (1, 256, 8), (7, 3, 2), (64, 8, 2), (1000, 60, 4), (257, 64, 6), (33, 257, 8), (129, 512, 10), (65, 1024, 32), (50, 37, 32), (3, 32, 32), (2500, 128, 8),
         (700, 31, 2), (701, 24, 1), (333, 33, 4), (90, 64, 2), (91, 100, 3), (64, 300, 20), (24600, 31, 2), (24577, 33, 4), (24576, 64, 1), (24576, 20, 7)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [F32, BF, FP])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_route(T, E, k, dtype, form):
    x = (2 * torch.randn(T, E, generator=gen(T + E), device=DEV)).to(dtype)
    plan = routing.ExpertRouter(E, k, **form)
    check_route(plan, x, **form)
    bias = 0.1 * torch.randn(E, generator=gen(1), device=DEV)
    mask = torch.rand(T, generator=gen(2), device=DEV) < 0.7
    check_route(plan, x, bias, mask, **form)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("T,E,k,groups,top_groups,group_top", [
    (500, 256, 8, 8, 4, 2), (500, 256, 8, 8, 3, 1), (100, 60, 4, 5, 2, 2), (100, 60, 6, 20, 3, 2), (64, 32, 3, 32, 3, 1), (40, 1024, 8, 32, 1, 2),
    (200, 96, 5, 3, 2, 2), (200, 8, 2, 4, 1, 2), (30, 640, 9, 2, 1, 2)])
def test_groups(T, E, k, groups, top_groups, group_top, with_bias, score):
    for dtype in (F32, BF):
        x = torch.randn(T, E, generator=gen(E + k), device=DEV).to(dtype)
        bias = 0.05 * torch.randn(E, generator=gen(1), device=DEV) if with_bias else None
        kw = dict(score=score, groups=groups, top_groups=top_groups, group_top=group_top)
        check_route(routing.ExpertRouter(E, k, **kw), x, bias, **kw)


def test_all_groups_is_no_choice_among_them():
    x = torch.randn(50, 64, generator=gen(0), device=DEV)
    a = routing.ExpertRouter(64, 6).route(x)
    b = routing.ExpertRouter(64, 6, groups=8, top_groups=8).route(x)
    assert torch.equal(a.ids, b.ids) and torch.equal(a.weights, b.weights)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups", [(64, 1), (256, 8), (1024, 4)])
def test_choices_that_fp32_cannot_tell_apart(E, groups, score):
    """Biases that bring every expert's s + b to the same value but for the bias's own rounding (2^-26 or so)."""
    T, k = 40, 8
    row = torch.randn(1, E, generator=gen(3), device=DEV)
    s = (torch.softmax(row.double(), 1) if score == "softmax" else torch.sigmoid(row.double()))[0]
    bias = (0.75 - s).float()
    x = row.repeat(T, 1)
    x[1::2] = torch.randn(T // 2, E, generator=gen(4), device=DEV)
    kw = dict(score=score, groups=groups, top_groups=max(1, groups // 2))
    check_route(routing.ExpertRouter(E, k, **kw), x, bias, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [2, 3, 5, 12])
@pytest.mark.parametrize("E,k,groups", [(64, 8, 1), (64, 5, 8), (256, 8, 8), (200, 7, 5), (16, 2, 1), (512, 8, 4)])
def test_clusters_of_choices_as_good(E, k, groups, size, score):
    """Clusters of `size` experts whose s + b differ by the rounding of b alone, clusters 0.01 apart, some of a cluster equal in
    every bit; wherever the k-th falls in its cluster."""
    for seed in range(4):
        g = gen(100 + seed)
        x = torch.randn(1, E, generator=g, device=DEV)
        order = torch.randperm(E, generator=g, device=DEV)
        cluster = torch.empty(E, dtype=torch.long, device=DEV)
        cluster[order] = torch.arange(E, device=DEV) // size
        for c in range(0, E // size, 2):  # two of every other cluster have the same logit, and so the same bias
            pair = (cluster == c).nonzero()[:2, 0]
            x[0, pair[-1]] = x[0, pair[0]]
        s = (torch.softmax(x.double(), 1) if score == "softmax" else torch.sigmoid(x.double()))[0]
        bias = (0.01 * cluster.double() + 0.3 - s).float()
        rows = torch.cat([x.repeat(20, 1), torch.randn(20, E, generator=g, device=DEV)])
        for kw in (dict(score=score, groups=groups, top_groups=max(1, groups // 2)), dict(score=score, groups=groups, top_groups=max(1, groups - 1), group_top=1)):
            if k <= E // groups * kw["top_groups"]:
                check_route(routing.ExpertRouter(E, k, **kw), rows, bias, **kw)


@pytest.mark.parametrize("groups", [1, 4])
def test_clusters_of_logits_as_good(groups):
    """fp32 logits that differ in their last bits, and some that do not."""
    E, k = 128, 8
    for seed in range(4):
        g = gen(200 + seed)
        base = torch.randint(-4, 5, (60, E), generator=g, device=DEV).float() + 0.1
        x = base * (1 + torch.randint(0, 3, (60, E), generator=g, device=DEV) * 2.0**-23)
        for score in ("softmax", "sigmoid"):
            kw = dict(score=score, groups=groups, top_groups=max(1, groups // 2))
            check_route(routing.ExpertRouter(E, k, **kw), x, **kw)
            check_route(routing.ExpertRouter(E, k, group_top=1, **kw), x, group_top=1, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_go_to_the_lower_expert(score):
    T, E, k = 300, 96, 8
    x = torch.randint(-2, 3, (T, E), generator=gen(5), device=DEV).to(BF)
    bias = 0.25 * torch.randint(0, 2, (E,), generator=gen(6), device=DEV).float()
    for b in (None, bias, torch.zeros(E, device=DEV)):
        check_route(routing.ExpertRouter(E, k, score=score), x, b, score=score)
        for group_top in (1, 2):
            kw = dict(score=score, groups=8, top_groups=3, group_top=group_top)
            check_route(routing.ExpertRouter(E, k, **kw), x, b, **kw)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("E", [12, 300])
def test_rows_and_experts_that_are_not_available(E, form):
    k = 5
    x = torch.randn(16, E, generator=gen(7), device=DEV)
    x[0] = -math.inf  # nothing left
    x[1, 3:] = -math.inf  # fewer than k
    x[2, ::2] = -math.inf
    x[3, 4] = math.nan
    x[4] = math.nan
    x[5, 7] = math.inf
    x[6] = torch.finfo(F32).min
    x[7, 1:] = torch.finfo(F32).min
    x[8] = torch.finfo(F32).max
    x[9, 0], x[9, 1] = torch.finfo(F32).max, -math.inf
    x[10] = -100.0 + x[10]  # scores below fp32's normal range
    x[11, 2] = 90.0
    mask = torch.ones(16, dtype=torch.bool, device=DEV)
    mask[[4, 12]] = False
    bias = 0.1 * torch.randn(E, generator=gen(8), device=DEV)
    bias[5], bias[6], bias[8] = -math.inf, math.nan, math.inf
    plan = routing.ExpertRouter(E, k, **form)
    for b in (None, bias):
        for m in (None, mask):
            r = check_route(plan, x, b, m, **form)
            d = plan.grad(x, r.ids, r.weights, torch.ones_like(r.weights))
            none = (r.ids < 0).all(1)
            assert (d[none] == 0).all()
    kw = form | dict(groups=3, top_groups=2)
    check_route(routing.ExpertRouter(E, k, **kw), x, bias, mask, **kw)


def grad_bound(x, ids, p, dw, form, dtype):
    """(dlogits, bound) in 64 bits: through the chosen weights' formula.  Each a_j carries its weight's error, their sum k + 5
    additions, and the result the roundings of a difference, a product and the type."""
    T, E = x.shape
    k = ids.shape[1]
    x, dw = x.double(), dw.double()
    there = (ids >= 0).double()
    scale = form.get("weight_scale", 1.0)
    w = torch.nan_to_num(p) * there
    a = dw * w
    A, size = a.sum(1, keepdim=True), a.abs().sum(1, keepdim=True)
    s = torch.softmax(x, 1) if form["score"] == "softmax" else torch.sigmoid(x)
    s = torch.nan_to_num(s) * there.amax(1, keepdim=True)
    at = ids.clamp(min=0)
    out = torch.zeros_like(x).scatter_add_(1, at, a)
    share = torch.zeros_like(x).scatter_add_(1, at, w / scale)
    bound = torch.zeros_like(x).scatter_add_(1, at, a.abs())
    if form.get("renormalize", True):
        out, bound = out - share * A, bound + share * size
    elif form["score"] == "softmax":
        out, bound = out - s * A, bound + s * size
    if form["score"] == "sigmoid":
        out, bound = out * (1 - s), bound * (1 - s)
    rel = 2 * slack(x, ids) + (k + 5 + 8) * U
    return out, half(dtype) * out.abs() + rel * bound + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [F32, BF, FP])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_grad(T, E, k, dtype, form):
    x = torch.randn(T, E, generator=gen(T), device=DEV).to(dtype)
    mask = torch.rand(T, generator=gen(2), device=DEV) < 0.8
    plan = routing.ExpertRouter(E, k, **form)
    r = plan.route(x, None, mask)
    dw = torch.randn(T, k, generator=gen(9), device=DEV)
    got = plan.grad(x, r.ids, r.weights, dw)
    ids, w, _ = plain(x, k, mask=mask, **form)
    want, bound = grad_bound(x, ids, w, dw, form, dtype)
    assert ((got.double() - want).abs() <= bound).all(), ((got.double() - want).abs() / bound).max()
    # scaled, and added to another gradient: one rounding more, of the sum
    base = torch.randn(T, E, generator=gen(10), device=DEV).to(dtype)
    sums = plan.grad(x, r.ids, r.weights, dw, scale=0.5, dlogits=base.clone(), accumulate=True)
    assert ((sums.double() - base.double() - 0.5 * want).abs() <= bound + half(dtype) * (base.double() + 0.5 * want).abs()).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_grad_of_choices_that_are_sure(score):
    """One expert per token, or one that outweighs the others by e^12: the gradient is a sum of p_j (dw_i - dw_j), each term off by
    the weights' errors and two roundings, and none of a choice of one."""
    T, E = 200, 40
    x = torch.randn(T, E, generator=gen(50), device=DEV)
    for scale in (1.0, 2.5):
        one = routing.ExpertRouter(E, 1, score=score, weight_scale=scale)
        r = one.route(x)
        assert (r.weights == scale).all() and (one.grad(x, r.ids, r.weights, torch.randn(T, 1, device=DEV)) == 0).all()
    x -= 6.0
    x[:, 7] += 12.0
    plan = routing.ExpertRouter(E, 4, score="softmax")
    r = plan.route(x)
    dw = torch.randn(T, 4, generator=gen(51), device=DEV)
    got = torch.gather(plan.grad(x, r.ids, r.weights, dw), 1, r.ids.long()).double()
    ids, p, _ = plain(x, 4)
    d = dw.double()[:, :, None] - dw.double()[:, None, :]
    want, size = p * (p[:, None, :] * d).sum(2), p * (p[:, None, :] * d.abs()).sum(2)
    assert ((got - want).abs() <= (2 * slack(x, ids) + 16 * U) * size).all()


@pytest.mark.parametrize("form", FORMS)
def test_an_expert_named_twice_gets_both(form):
    T, E, k = 50, 20, 3
    x = torch.randn(T, E, generator=gen(52), device=DEV)
    ids = torch.randint(0, E, (T, k), generator=gen(53), device=DEV)
    ids[:, 2] = ids[:, 0]
    dw = torch.randn(T, k, generator=gen(54), device=DEV)
    plan = routing.ExpertRouter(E, k, **form)
    w = torch.rand(T, k, generator=gen(55), device=DEV)
    w = form.get("weight_scale", 1.0) * w / w.sum(1, keepdim=True)
    got = plan.grad(x, ids, w, dw)
    want, bound = grad_bound(x, ids, w.double(), dw, form, F32)
    # the weights' sum is 1 but for its roundings
    assert ((got.double() - want).abs() <= bound + 8 * U * (w * dw).abs().sum(1, keepdim=True).double()).all()


@pytest.mark.parametrize("form", FORMS)
def test_grad_against_differences(form):
    """The plain weights in 64 bits, at x + h v and x - h v with the choice held: the difference is off by h^2 / 6 times a third
    derivative below 30 per unit of sum |dw| |v|^3 (|v| <= 5), the kernel's gradient by its bound."""
    T, E, k, h = 20, 24, 4, 1e-4
    x = torch.randn(T, E, generator=gen(11), device=DEV)
    plan = routing.ExpertRouter(E, k, **form)
    r = plan.route(x)
    dw, v = torch.randn(T, k, generator=gen(12), device=DEV), torch.randn(T, E, generator=gen(13), device=DEV).clamp(-5, 5)
    got = plan.grad(x, r.ids, r.weights, dw)

    def value(y):
        s = torch.softmax(y, 1) if form["score"] == "softmax" else torch.sigmoid(y)
        p = torch.gather(s, 1, r.ids.long())
        if form.get("renormalize", True):
            p = p / p.sum(1, keepdim=True)
        return form.get("weight_scale", 1.0) * (p * dw.double()).sum(1)

    slope = (value(x.double() + h * v.double()) - value(x.double() - h * v.double())) / (2 * h)
    _, bound = grad_bound(x, r.ids.long(), r.weights.double(), dw, form, F32)
    assert ((got.double() * v.double()).sum(1) - slope).abs().max() <= (bound * v.abs()).sum(1).max() + 3 * h * h / 6 * 30 * 125 * dw.abs().sum(1).max() + 1e-11


def test_strides_types_of_ids_and_bits():
    T, E, k = 301, 60, 4
    wide = torch.randn(T, 2 * E + 1, generator=gen(14), device=DEV)
    x = wide[:, 1 : E + 1]  # neither the rows nor the columns start at a multiple of 16 bytes
    a = routing.ExpertRouter(E, k).route(x.contiguous())
    b = routing.ExpertRouter(E, k, int64_ids=True).route(x)
    assert b.ids.dtype == torch.int64 and torch.equal(a.ids.long(), b.ids) and torch.equal(a.weights, b.weights) and torch.equal(a.counts, b.counts)
    plan = routing.ExpertRouter(E, k, renormalize=False)
    r = plan.route(x)
    dw = torch.randn(T, 2 * k, generator=gen(15), device=DEV)[:, ::1][:, :k]
    into = torch.full((T, 2 * E), 7.0, device=DEV)
    got = plan.grad(x, r.ids.long(), r.weights, dw, dlogits=into[:, 3 : E + 3])
    # words of other widths add up a row's exponentials in another order: each result is within its bound
    _, bound = grad_bound(x, r.ids.long(), r.weights.double(), dw, dict(score="softmax", renormalize=False), F32)
    assert ((got.double() - plan.grad(x.contiguous(), r.ids, r.weights, dw.contiguous()).double()).abs() <= 2 * bound).all()
    assert (into[:, :3] == 7).all() and (into[:, E + 3 :] == 7).all()
    again = plan.route(x)
    assert torch.equal(r.ids, again.ids) and torch.equal(r.weights, again.weights) and torch.equal(r.counts, again.counts)


def test_no_tokens():
    plan, exchange = routing.ExpertRouter(16, 2), routing.ExpertExchange(16)
    x = torch.empty(0, 16, device=DEV)
    r = plan.route(x)
    assert r.ids.shape == (0, 2) and (r.counts == 0).all()
    assert plan.grad(x, r.ids, r.weights, r.weights).shape == (0, 16)
    o = exchange.order(r.ids)
    assert (o.offsets == 0).all() and o.rows.numel() == 0
    z = exchange.dispatch(torch.empty(0, 8, device=DEV), o)
    assert z.shape == (0, 8) and exchange.combine(z, o, r.weights).shape == (0, 8)
    assert exchange.combine_grad(torch.empty(0, 8, device=DEV), z, o, r.weights)[0].shape == (0, 8)
    # rows without columns
    o = exchange.order(torch.zeros(5, 2, dtype=torch.int32, device=DEV))
    z = exchange.dispatch(torch.empty(5, 0, device=DEV), o)
    assert z.shape == (10, 0) and (exchange.combine_grad(torch.empty(5, 0, device=DEV), z, o)[1] == 0).all()


def test_offsets_beyond_32_bits():
    T, E, k = (1 << 21) + 3, 1024, 2
    x = torch.zeros(T, E, dtype=BF, device=DEV)
    x[-3:, 1000] = 1.0
    x[-3:, 17] = 2.0
    plan = routing.ExpertRouter(E, k)
    r = plan.route(x)
    assert r.ids[-3:].tolist() == [[17, 1000]] * 3 and r.ids[:-3].amax().item() == 1 and r.counts.tolist()[0] == T - 3
    x.fill_(7.0)
    d = plan.grad(x, r.ids, r.weights, torch.tensor([[1.0, -1.0]], device=DEV).repeat(T, 1), dlogits=x)
    p = torch.softmax(torch.tensor([2.0, 1.0], dtype=torch.float64), 0)
    want = 2 * p[0] * p[1]
    assert abs(d[-1, 17].item() - want) <= 1e-2 * want and d[-1, 17] == -d[-1, 1000] and (d[-1] != 0).sum() == 2 and (d[-4] != 0).sum() == 2


# ---- exchange -----------------------------------------------------------------------------------------


def plain_order(ids, E):
    T, k = ids.shape
    key = torch.where((ids < 0) | (ids >= E), E, ids.long()).reshape(-1)
    pairs = torch.sort(key, stable=True).indices
    n = int((key < E).sum())
    rows = torch.full((T * k,), -1, device=DEV)
    rows[:n] = pairs[:n] // k
    slots = torch.full((T * k,), -1, device=DEV)
    slots[pairs[:n]] = torch.arange(n, device=DEV)
    return torch.cat([torch.zeros(1, device=DEV).long(), torch.bincount(key, minlength=E + 1)[:E].cumsum(0)]), slots.view(T, k), rows, n


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (64, 8, 2), (333, 60, 4), (1024, 8, 8), (1025, 8, 8), (5000, 256, 8), (3000, 1024, 32), (40000, 128, 1), (70001, 5, 3)])
@pytest.mark.parametrize("wide", [False, True])
def test_order(T, E, k, wide):
    ids = torch.randint(-1, E + 1, (T, k), generator=gen(T), device=DEV)  # -1 and E belong to nobody
    if T == 1024:
        ids[:] = 3  # one expert takes them all, the same one several times in a row
    ids = ids if wide else ids.int()
    ex = routing.ExpertExchange(E)
    o = ex.order(ids)
    offsets, slots, rows, _ = plain_order(ids, E)
    assert torch.equal(o.offsets.long(), offsets) and torch.equal(o.slots.long(), slots) and torch.equal(o.rows.long(), rows)
    strided = torch.full((T, k + 3), 1, device=DEV, dtype=ids.dtype)
    strided[:, :k] = ids
    again = ex.order(strided[:, :k])
    assert all(torch.equal(a, b) for a, b in zip(o, again))


def test_order_of_nobody():
    ex = routing.ExpertExchange(4)
    o = ex.order(torch.full((70, 3), -1, device=DEV))
    assert (o.offsets == 0).all() and (o.slots == -1).all() and (o.rows == -1).all()
    x = torch.randn(70, 40, device=DEV)
    w = torch.full((70, 3), math.nan, device=DEV)
    z = torch.full((210, 40), math.nan, device=DEV)
    assert (ex.dispatch(x, o) == 0).all() and (ex.combine(z, o, w) == 0).all()
    dz, dw = ex.combine_grad(x, z, o, w)
    assert (dz == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF, FP])
@pytest.mark.parametrize("T,D,E,k", [(1, 1, 1, 1), (1, 4096, 8, 8), (64, 1024, 8, 2), (100, 33, 7, 3), (259, 1032, 60, 4), (50, 6, 5, 32), (20, 2050, 40, 12), (2100, 516, 16, 8)])
def test_exchange(T, D, E, k, dtype):
    g = gen(T + D)
    ids = torch.randint(-1, E, (T, k), generator=g, device=DEV).int()
    ex = routing.ExpertExchange(E)
    o = ex.order(ids)
    offsets, slots, rows, n = plain_order(ids, E)
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, z, dy, w = normal(T, D).to(dtype), normal(T * k, D).to(dtype), normal(T, D).to(dtype), normal(T, k)
    z[n:] = math.nan  # rows of no pair are not read
    sent = ex.dispatch(x, o)
    assert torch.equal(sent[:n], x[rows[:n]]) and (sent[n:] == 0).all()
    on = (slots >= 0).double()[:, :, None]
    picked = torch.where(on > 0, z.double()[slots.clamp(min=0)], 0.0)
    # k products added up in fp32 and rounded once
    for weights in (w, None):
        f = (torch.ones_like(w) if weights is None else weights).double()[:, :, None] * on
        y = ex.combine(z, o, weights)
        want, size = (f * picked).sum(1), (f * picked).abs().sum(1)
        assert ((y.double() - want).abs() <= half(dtype) * want.abs() + (k + 1) * U * size + 2.0**-25).all()
        dz, dw = ex.combine_grad(dy, z, o, weights)
        rows_f = torch.zeros(T * k, dtype=torch.float64, device=DEV)
        rows_f[slots[slots >= 0]] = f[:, :, 0][slots >= 0]
        want = rows_f[:, None] * dy.double()[rows.clamp(min=0)]
        assert ((dz.double() - want).abs() <= half(dtype) * want.abs() + U * want.abs() + 2.0**-25).all() and (dz[n:] == 0).all()
        products = picked * dy.double()[:, None, :] * on
        assert ((dw.double() - products.sum(2)).abs() <= (D + 1) * U * products.abs().sum(2)).all()
        assert torch.equal(ex.combine_grad(dy, z, o, weights, want=("rows",))[0], dz)
        assert torch.equal(ex.combine_grad(dy, z, o, weights, want=("weights",))[1], dw)
    back = ex.dispatch_grad(z, o)
    assert torch.equal(back, ex.combine(z, o))


def test_exchange_strides():
    T, D, E, k = 130, 72, 9, 3
    g = gen(21)
    ids = torch.randint(0, E, (T, k), generator=g, device=DEV)
    ex = routing.ExpertExchange(E)
    o = ex.order(ids)
    for step, first in ((80, 8), (81, 1)):  # rows at multiples of 16 bytes, and not
        x, z = torch.randn(T, step, generator=g, device=DEV).to(BF)[:, first:][:, :D], torch.randn(T * k, step, generator=g, device=DEV).to(BF)[:, first:][:, :D]
        w = torch.randn(T, 5, generator=g, device=DEV)[:, 1:4]
        a, b = torch.full((T * k, step), 3.0, device=DEV, dtype=BF), torch.full((T, step), 3.0, device=DEV, dtype=BF)
        assert torch.equal(ex.dispatch(x, o, out=a[:, first:][:, :D]), ex.dispatch(x.contiguous(), o))
        assert torch.equal(ex.combine(z, o, w, out=b[:, first:][:, :D]), ex.combine(z.contiguous(), o, w.contiguous()))
        for m in (a, b):
            assert (m[:, :first] == 3).all() and (m[:, first + D :] == 3).all()
        p, q = ex.combine_grad(x, z, o, w, out=a[:, first:][:, :D]), ex.combine_grad(x.contiguous(), z.contiguous(), o, w.contiguous())
        assert torch.equal(p[0], q[0])
        # words of other widths add up the D products in another order: each order is within (D + 1) U of their absolute sum
        size = (z.double()[o.slots.long()] * x.double()[:, None, :]).abs().sum(2)
        assert ((p[1].double() - q[1].double()).abs() <= 2 * (D + 1) * U * size).all()


def test_exchange_beyond_32_bits():
    T, D, E, k = 8200, 8192, 4, 32
    ids = torch.zeros(T, k, dtype=torch.int32, device=DEV)
    ids[-1] = 3
    ex = routing.ExpertExchange(E)
    o = ex.order(ids)
    x = torch.zeros(T, D, dtype=BF, device=DEV)
    x[-1] = 1.0
    z = ex.dispatch(x, o)  # 2.1e9 elements
    assert (z[-k:] == 1).all() and (z[-k - 1] == 0).all()
    y = ex.combine(z, o)
    assert (y[-1] == k).all() and (y[-2] == 0).all()
    _, dw = ex.combine_grad(x, z, o, None, want=("weights",))
    assert (dw[-1] == D).all() and (dw[:-1] == 0).all()


# ---- together -----------------------------------------------------------------------------------------


def test_differentiable_forms_together():
    """Tokens to experts that scale them, and back: gradients to the logits, the tokens and the scales against 64 bits."""
    T, D, E, k = 90, 48, 12, 3
    g = gen(30)
    x, logits, gain = (torch.randn(*s, generator=g, device=DEV) for s in ((T, D), (T, E), (E, D)))
    up = torch.randn(T, D, generator=g, device=DEV)
    router, ex = routing.ExpertRouter(E, k), routing.ExpertExchange(E)
    a = [v.clone().requires_grad_() for v in (x, logits, gain)]
    r = routing.route(router, a[1])
    o = ex.order(r.ids)
    z = routing.dispatch(ex, a[0], o)
    owner = torch.searchsorted(o.offsets[1:].contiguous(), torch.arange(T * k, device=DEV, dtype=torch.int32), right=True)
    y = routing.combine(ex, z * a[2][owner], o, r.weights)
    y.backward(up)
    b = [v.double().requires_grad_() for v in (x, logits, gain)]
    ids = r.ids.long()
    w = torch.softmax(torch.gather(b[1], 1, ids), 1)
    want = (w[:, :, None] * b[0][:, None, :] * b[2][ids]).sum(1)
    want.backward(up.double())
    assert (y.double() - want).abs().max() <= 1e-5
    # sums of at most T products of values below 100, each with a handful of roundings
    for p, q in zip(a, b):
        assert (p.grad.double() - q.grad).abs().max() <= 200 * 100 * U * 8
    with pytest.raises(RuntimeError):
        (d,) = torch.autograd.grad(routing.route(router, a[1]).weights.square().sum(), a[1], create_graph=True)
        d.sum().backward()


def test_captured_and_replayed_with_the_balance_loss():
    """Routing, its gradient added to the balance loss's, and the exchange, in one graph over new inputs."""
    T, E, k, D = 2000, 64, 4, 96
    router, ex, balance = routing.ExpertRouter(E, k, score="sigmoid"), routing.ExpertExchange(E), losses.ExpertBalance(T, E)
    x, v, dw, bias = torch.empty(T, E, device=DEV), torch.empty(T, D, device=DEV), torch.empty(T, k, device=DEV), torch.zeros(E, device=DEV)

    def step():
        r = router.route(x, bias)
        b = balance.grad(x, r.ids, coef=0.5)
        router.grad(x, r.ids, r.weights, dw, dlogits=b.dlogits, accumulate=True)
        o = ex.order(r.ids)
        return r.ids, r.weights, r.counts, b.counts, b.dlogits, ex.combine(ex.dispatch(v, o), o, r.weights)

    def fill(seed):
        g = gen(seed)
        for m in (x, v, dw):
            m.copy_(torch.randn(m.shape, generator=g, device=DEV))
        bias.copy_(0.1 * torch.randn(E, generator=g, device=DEV))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2):
        fill(seed)
        want = [m.clone() for m in step()]
        for m in out:
            m.zero_()
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(out, want))
        assert torch.equal(want[2], want[3])


def test_other_streams():
    T, E, k = 4000, 128, 8
    router, ex = routing.ExpertRouter(E, k), routing.ExpertExchange(E)
    x = torch.randn(T, E, generator=gen(40), device=DEV)
    want = router.route(x)
    order = ex.order(want.ids)
    torch.cuda.synchronize()
    for _ in range(3):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            r = router.route(x)
            o = ex.order(r.ids)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(r, want)) and all(torch.equal(a, b) for a, b in zip(o, order))


def test_refusals():
    for bad in (dict(experts=0, top_k=1), dict(experts=1025, top_k=1), dict(experts=8, top_k=9), dict(experts=64, top_k=33), dict(experts=8, top_k=0),
                dict(experts=60, top_k=2, groups=7), dict(experts=64, top_k=9, groups=8, top_groups=1), dict(experts=64, top_k=1, groups=8, top_groups=9),
                dict(experts=64, top_k=1, groups=64, top_groups=2), dict(experts=8, top_k=1, groups=8, top_groups=2, group_top=2),
                dict(experts=8, top_k=1, weight_scale=0.0), dict(experts=8, top_k=1, weight_scale=math.nan)):
        with pytest.raises(losses.IwpError):
            routing.ExpertRouter(**bad)
    with pytest.raises(ValueError):
        routing.ExpertRouter(8, 2, score="tanh")
    with pytest.raises(losses.IwpError):
        routing.ExpertExchange(2000)
    plan, ex = routing.ExpertRouter(8, 2), routing.ExpertExchange(8)
    x = torch.randn(5, 8, device=DEV)
    r = plan.route(x)
    o = ex.order(r.ids)
    for call in (lambda: plan.route(x.double()), lambda: plan.route(x, torch.zeros(8, device=DEV, dtype=BF)), lambda: plan.route(x, None, torch.ones(5, device=DEV)),
                 lambda: plan.grad(x, r.ids.float(), r.weights, r.weights), lambda: plan.grad(x, r.ids, r.weights, r.weights.to(BF)),
                 lambda: plan.grad(x, r.ids, r.weights, r.weights, dlogits=x.to(BF)), lambda: ex.order(r.ids.short()),
                 lambda: ex.combine(torch.zeros(10, 4, device=DEV), o, r.weights.double()), lambda: ex.dispatch(x.double(), o)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: plan.route(x[:, :7]), lambda: plan.route(x[0]), lambda: plan.route(x.t().contiguous().t()), lambda: plan.route(x.cpu()),
                 lambda: plan.route(x, torch.zeros(7, device=DEV)), lambda: plan.route(x, None, torch.ones(4, device=DEV, dtype=torch.bool)),
                 lambda: plan.route(x[:1].expand(5, 8)), lambda: plan.grad(x, r.ids[:, :1], r.weights, r.weights),
                 lambda: plan.grad(x, r.ids, r.weights, r.weights, accumulate=True), lambda: ex.order(r.ids.flatten()),
                 lambda: ex.dispatch(torch.zeros(4, 3, device=DEV), o), lambda: ex.combine(torch.zeros(9, 3, device=DEV), o),
                 lambda: ex.combine(torch.zeros(10, 3, device=DEV), o, r.weights[:4]), lambda: routing.ExpertExchange(9).dispatch(x, o)):
        with pytest.raises(ValueError):
            call()
    # what is in range but not a slot is nobody's
    y = ex.combine(torch.ones(10, 3, device=DEV), routing.Order(o.offsets, torch.full_like(o.slots, 1000), o.rows))
    assert (y == 0).all()


def test_order_of_another_plan():
    """An order is taken as made by the plan that made it alone; by another it is looked at like any other tensors."""
    one, two = routing.ExpertExchange(8), routing.ExpertExchange(8)
    x = torch.randn(5, 4, device=DEV)
    o = one.order(torch.randint(0, 8, (5, 2), device=DEV))
    assert torch.equal(one.dispatch(x, o), two.dispatch(x, o))
    other = routing._Made(*(y.cpu() for y in o))
    other.made = o.made
    with pytest.raises(ValueError):
        two.dispatch(x, other)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,k", [(300, 24, 5), (301, 31, 2), (200, 257, 8)])
def test_values_at_the_ends_of_the_types(T, E, k, dtype, score):
    """Zeros of both signs (which are equal), subnormal numbers, the lowest and the largest ones, -inf; also in rows of nothing else."""
    f = torch.finfo(dtype)
    least = f.smallest_normal * f.eps
    values = torch.tensor([0.0, -0.0, least, -least, 3 * least, f.smallest_normal, -f.smallest_normal, f.min, f.max if score == "sigmoid" else 1.0,
                           f.min * (1 - f.eps), -math.inf], dtype=torch.float64, device=DEV).to(dtype)
    g = torch.Generator(device=DEV).manual_seed(T)
    x = values[torch.randint(0, len(values), (T, E), device=DEV, generator=g)]
    x[:100] = values[torch.randint(0, 7, (100, E), device=DEV, generator=g)]
    x[100:110] = values[torch.tensor([7, 10], device=DEV)[torch.randint(0, 2, (10, E), device=DEV, generator=g)]]
    plan = routing.ExpertRouter(E, k, score=score, renormalize=False)
    check_route(plan, x, score=score, renormalize=False)
