"""The losses where their numbers are delicate: factors that cancel, confident rows, upstream gradients of very different
sizes, the lowest values, sums over long rows.

Most cases take a head whose weights are the identity: the logits are then the hidden states (products with one and zero,
sums of one term: exact), and the gradient to the hidden states is the factor exp(..) - q itself, times the upstream
gradient.  With logits below 32 in magnitude a probability formed in fp32 is off by at most P = 2^-16 of itself: five
roundings of exponents below 64 (2^-19 each, in log2), the sum's 64 additions per lane (2^-18), exp2 and log (2^-20)."""
import math

import pytest
import torch
from test_gpu_losses import BF, DEV, F32, HF, TINY, U, gen, soft_targets

from paper_1901_01544_b200 import losses

pytestmark = pytest.mark.gpu
P = 2.0**-16


def identity_head(T, V, D, dtype, seed, spread=3.0):
    """Hidden states that are the logits of the first D columns (the others' logits are zero)."""
    g = gen(seed)
    h = (torch.randn(T, D, generator=g, device=DEV) * spread).to(dtype)
    return h, torch.eye(V, D, device=DEV).to(dtype), g


def within(got, want, tol, name):
    got = got.double()
    assert torch.isfinite(got).all(), name + " is not finite"
    worst = ((got - want).abs() / tol).max().item()
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound"


def factor_error(p, q, dtype, at_target):
    """Bound on one factor p - q: one rounding to the type (fp16 factors are kept 2^13 higher, so its smallest steps are
    2^-38), the errors of p and of the teacher's q; where nothing is subtracted a code of p may have been rounded once more,
    and be cut off below 2^-24 of its row's largest."""
    f = (p - q).abs()
    return U[dtype] * f + P * (p + q) + 2.0**-37 + torch.where(at_target, 0.0, U[dtype] * p + 2.0**-24 * p.amax(1, keepdim=True))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("eps", [1e-1, 1e-3, 0.0])
@pytest.mark.parametrize("T,n,tau,piece", [(70, 64, 1.0, 0), (70, 64, 2.0, 0), (33, 1024, 1.0, 1), (33, 1024, 1.0, 0), (300, 200, 1.0, 0)])
def test_student_close_to_its_teacher(T, n, tau, piece, eps, dtype):
    """Teacher's logits = the student's plus a little noise, for every column: p - q is `eps` of p, and keeps the relative
    error of one rounding as far as fp32 can tell p from q."""
    h, w, g = identity_head(T, n, n, dtype, 700 + T + n)
    ids = torch.rand(T, n, generator=g, device=DEV).argsort(1)
    logits = h.float().gather(1, ids) + eps * torch.randn(T, n, generator=g, device=DEV)
    q = torch.zeros(T, n, dtype=torch.float64, device=DEV).scatter_(1, ids, soft_targets(ids, logits, tau))
    p = torch.softmax(h.double() / tau, 1)
    f = tau * (p - q)
    f_err = tau * factor_error(p, q, dtype, torch.ones_like(p, dtype=torch.bool))
    w_err = f_err.T @ h.double().abs() + (T / 16 + 8) * 2.0**-22 * (f.abs().T @ h.double().abs())
    plan = losses.HeadLoss(T, n, n, dtype, top_k=n, piece_bytes=piece)
    lse = plan.distill(h, w, ids, logits, tau).lse
    for saved in (None, lse):
        dh, dw = torch.empty(T, n, device=DEV), torch.empty(n, n, device=DEV)
        plan.distill_grad(h, w, ids, logits, tau, reduction="sum", lse=saved, dhidden=dh, dweight=dw)
        within(dh, f, f_err + 2.0**-23 * f.abs() + 1e-37, "dhidden")
        within(dw, f.T @ h.double(), w_err + 2.0**-23 * (f.T @ h.double()).abs() + 1e-37, "dweight")
    assert plan.status() == 0


@pytest.mark.parametrize("piece", [0, 1])
@pytest.mark.parametrize("T,V,n,K,tau", [(50, 300, 64, 9, 1.0), (150, 700, 128, 50, 2.0), (5, 1100, 72, 64, 0.5)])
def test_distillation_in_fp16(T, V, n, K, tau, piece):
    h, w, g = identity_head(T, V, n, HF, 720 + T)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :K].contiguous()
    logits = torch.randn(T, K, generator=g, device=DEV) * 3
    q = torch.zeros(T, V, dtype=torch.float64, device=DEV).scatter_(1, ids, soft_targets(ids, logits, tau))
    hit = torch.zeros(T, V, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
    z = torch.cat([h.double(), torch.zeros(T, V - n, dtype=torch.float64, device=DEV)], 1)
    p = torch.softmax(z / tau, 1)
    f, f_err = tau * (p - q), tau * factor_error(p, q, HF, hit)
    plan = losses.HeadLoss(T, V, n, HF, top_k=K, piece_bytes=piece)
    dh, dw = torch.empty(T, n, device=DEV), torch.empty(V, n, device=DEV)
    plan.distill_grad(h, w, ids, logits, tau, reduction="sum", dhidden=dh, dweight=dw)
    within(dh, f[:, :n], f_err[:, :n] + 2.0**-23 * f[:, :n].abs(), "dhidden")
    want = f.T @ h.double()
    within(dw, want, f_err.T @ h.double().abs() + (T / 16 + 8) * 2.0**-22 * (f.abs().T @ h.double().abs()) + 2.0**-23 * want.abs(), "dweight")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D", [(1, 64, 64), (2, 300, 64), (40, 64, 64), (300, 900, 128), (5000, 300, 64)])
def test_confident_rows(T, V, D, dtype):
    """Rows whose target has all the mass lose nothing at all, whatever the size of their logits; with a little mass
    elsewhere the loss is log(1 + s), s of few terms: right to the last bits of fp32."""
    w = torch.eye(V, D, device=DEV).to(dtype)
    y = torch.arange(T, device=DEV) % D
    top = torch.tensor([20.0, 37.5, 60.0, 300.0, 500.0], device=DEV)[torch.arange(T, device=DEV) % 5][:, None]
    on = torch.nn.functional.one_hot(y, D).bool()
    plan = losses.HeadLoss(T, V, D, dtype)
    for gap in (400.0, 12.0, 4.0):
        h = torch.where(on, top, top - gap).to(dtype)
        if gap == 400.0:
            h = torch.where(on, h, -200.0).to(dtype)
        z = torch.cat([h.double(), torch.zeros(T, V - D, dtype=torch.float64, device=DEV)], 1)
        lse = torch.logsumexp(z, 1)
        want = torch.log1p(torch.where(torch.nn.functional.one_hot(y, V).bool(), 0.0, torch.exp(z - top.double())).sum(1)) if gap < 400 or V > D else 0 * lse
        r = plan.cross_entropy(h, w, y)
        # a lane adds at most 64 terms to a sum that starts at 1 or more, 20 more additions join lanes and parts; a term is
        # off by 2^-19 of itself (its exponent is rounded below 64)
        tol = 84 * 2.0**-24 * (1 + want) + 2.0**-19 * want
        if gap == 400.0 and V == D:
            assert not r.rows.any() and torch.equal(r.lse, top[:, 0]) and r.loss == 0
        assert (r.rows >= 0).all()
        within(r.rows, want, tol, "rows")
        within(r.lse, lse, tol + 2.0**-23 * lse.abs(), "lse")


def test_confident_rows_of_a_distillation():
    T, n, tau = 60, 64, 2.0
    w = torch.eye(n, device=DEV).to(BF)
    y = torch.arange(T, device=DEV) % n
    h = torch.where(torch.nn.functional.one_hot(y, n).bool(), 300.0, -100.0).to(BF)
    plan = losses.HeadLoss(T, n, n, BF, top_k=1)
    r = plan.distill(h, w, y[:, None], torch.zeros(T, 1, device=DEV), tau)
    assert not r.rows.any() and r.loss == 0 and (r.lse == 150.0).all()


def spread_rows(T, dtype, seed, hard=True, V=64, D=64):
    h, w, g = identity_head(T, V, D, dtype, seed)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    sign = torch.randint(0, 2, (T,), generator=g, device=DEV) * 2 - 1
    up = sign * 10.0 ** (-9.0 * torch.arange(T, device=DEV) / max(1, T - 1))
    return h, w, y, up.float()[torch.randperm(T, generator=g, device=DEV)].contiguous(), g


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,piece", [(48, 64, 0), (300, 900, 0), (300, 900, 1), (7, 64, 0)])
def test_upstream_gradients_of_very_different_sizes(T, V, piece, dtype):
    """A row's gradient to the hidden states depends on its own upstream gradient alone, and is as precise whatever the
    others' are; the head's gradient is as precise as its largest rows allow."""
    D = 64
    h, w, y, up, g = spread_rows(T, dtype, 740 + T, V=V, D=D)
    z = torch.cat([h.double(), torch.zeros(T, V - D, dtype=torch.float64, device=DEV)], 1)
    p = torch.softmax(z, 1)
    hot = torch.nn.functional.one_hot(y, V).bool()
    f_err = factor_error(p, hot.double(), dtype, hot)
    f, up64 = p - hot.double(), up.double()[:, None]
    plan = losses.HeadLoss(T, V, D, dtype, piece_bytes=piece)
    lse = plan.cross_entropy(h, w, y).lse
    for saved in (None, lse):
        dh, dw = torch.empty(T, D, device=DEV), torch.empty(V, D, device=DEV)
        plan.cross_entropy_grad(h, w, y, reduction="sum", lse=saved, dloss=up, dhidden=dh, dweight=dw)
        want = up64 * f
        within(dh, want[:, :D], (up64.abs() * f_err)[:, :D] + 2.0**-22 * want[:, :D].abs() + 1e-37, "dhidden")
        H = h.double()
        # the rows' scales may be carried by a copy of the hidden states in their type, relative to the largest scale
        # (a power of two up to twice it): steps of 2^-24 in fp16
        copy = 2.0 * up64.abs().max() * 2.0**-24 * f.abs().T @ torch.ones_like(H) if dtype == HF else 0.0
        tol = (up64.abs() * f_err).T @ H.abs() + copy + (T / 16 + 8) * 2.0**-22 * (want.abs().T @ H.abs())
        within(dw, want.T @ H, tol + 1e-37, "dweight")
    assert plan.status() == 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D,piece", [(40, 8192, 512, 0), (200, 3001, 72, 0), (200, 3001, 33, 1), (1021, 5000, 136, 0)])
def test_upstream_gradients_that_are_powers_of_two_scale_rows_exactly(T, V, D, piece, dtype):
    g = gen(760 + T)
    h = torch.randn(T, D, generator=g, device=DEV).to(dtype)
    w = (torch.randn(V, D, generator=g, device=DEV) / math.sqrt(D)).to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    up = 2.0 ** torch.randint(-12, 13, (T,), generator=g, device=DEV).float() * (torch.randint(0, 2, (T,), generator=g, device=DEV) * 2 - 1)
    up[3] = 0
    plan = losses.HeadLoss(T, V, D, dtype, piece_bytes=piece)
    for out in (F32, dtype):
        base, got = (torch.zeros(T, D, dtype=out, device=DEV) for _ in range(2))
        plan.cross_entropy_grad(h, w, y, reduction="sum", dloss=torch.ones(T, device=DEV), dhidden=base, accumulate=True, want=("hidden",))
        plan.cross_entropy_grad(h, w, y, reduction="sum", dloss=up, dhidden=got, accumulate=True, want=("hidden",))
        if out == F32:
            # (fp16 factors that are below the normal numbers may round differently: half a step of 2^-24 / 2^13 per column)
            slack = 2.0**-37 * w.double().abs().sum(0) if dtype == HF else 0.0
            assert ((got.double() - base.double() * up.double()[:, None]).abs() <= slack * up.double().abs()[:, None]).all()
        assert not got[3].any()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_upstream_gradients_that_are_not_finite_stay_in_their_rows(dtype):
    T = 48
    h, w, y, up, _ = spread_rows(T, dtype, 780)
    plan = losses.HeadLoss(T, 64, 64, dtype)
    fine = plan.cross_entropy_grad(h, w, y, reduction="sum", dloss=up, want=("hidden",)).dhidden
    for bad in (math.inf, -math.inf, math.nan):
        off = up.clone()
        off[5] = bad
        got = plan.cross_entropy_grad(h, w, y, reduction="sum", dloss=off, want=("hidden",)).dhidden
        rest = torch.arange(T, device=DEV) != 5
        assert torch.equal(got[rest], fine[rest]) and not torch.isfinite(got[5]).any()
    y[5] = -100  # a row without a target gives nothing, whatever its upstream gradient is
    got = plan.cross_entropy_grad(h, w, y, reduction="sum", dloss=off)
    assert not got.dhidden[5].any() and torch.equal(got.dhidden[rest], fine[rest]) and torch.isfinite(got.dweight).all()


def test_an_invalid_target_is_reported_by_a_backward_pass_of_its_own():
    T, V, D = 40, 64, 64
    h, w, g = identity_head(T, V, D, BF, 810)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    lse = losses.HeadLoss(T, V, D, BF).cross_entropy(h, w, y).lse
    y[3] = V
    plan = losses.HeadLoss(T, V, D, BF)
    r = plan.cross_entropy_grad(h, w, y, lse=lse)
    assert plan.status() == -1 and not r.dhidden[3].any() and torch.isfinite(r.dhidden.float()).all()
    plan = losses.HeadLoss(T, V, D, BF, top_k=2)
    ids = torch.stack([y.clamp(max=V - 1), y], 1)
    r = plan.distill_grad(h, w, ids, torch.zeros(T, 2, device=DEV), lse=lse)
    assert plan.status() == -1 and not r.dhidden[3].any()


def test_teachers_lowest_logits_at_low_temperature():
    """The type's lowest value is a logit like any other; divided by a temperature below one it leaves the type."""
    T, n = 40, 64
    h, w, g = identity_head(T, n, n, BF, 800)
    for top_type in (F32, BF, HF):
        for tau in (0.5, 0.75, 1.0):
            ids = torch.rand(T, n, generator=g, device=DEV).argsort(1)[:, :7].contiguous()
            logits = torch.randn(T, 7, generator=g, device=DEV).to(top_type)
            logits[3] = torch.finfo(top_type).min  # equal ones: a uniform teacher
            logits[4, 1:] = torch.finfo(top_type).min
            logits[5] = torch.finfo(top_type).max
            logits[6, 2] = torch.finfo(top_type).max
            q = torch.zeros(T, n, dtype=torch.float64, device=DEV).scatter_(1, ids, soft_targets(ids, logits, tau))
            hit = torch.zeros(T, n, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
            p = torch.softmax(h.double() / tau, 1)
            f, f_err = tau * (p - q), tau * factor_error(p, q, BF, hit)
            plan = losses.HeadLoss(T, n, n, BF, top_k=7)
            dh = torch.empty(T, n, device=DEV)
            r = plan.distill_grad(h, w, ids, logits, tau, reduction="sum", dhidden=dh, want=("hidden",))
            within(dh, f, f_err + 2.0**-23 * f.abs() + 1e-37, "dhidden")
            z = h.double() / tau
            entropy = torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(1)
            rows = tau * tau * (entropy - (q * z).sum(1) + torch.logsumexp(z, 1))
            within(r.rows, rows, tau * tau * 2.0**-16 * (40 + z.abs().amax(1)), "rows")


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_probabilities_see_the_logits_that_lse_saw(dtype, saved):
    """All columns of the head are one vector, with which every row's product is a sum of 4096 terms of one sign, about 1000:
    p = 1 / V exactly.  lse is near 1031, so p is off by less than 2^-12 of itself (three exponents below 2048 rounded by
    half a step of 2^-13, times log 2, and lse by as much), which is less than half a step of either type (2^-9, 2^-12
    below a power of two): columns that are nobody's target get the sum of the hidden states, times 2^-10 exactly."""
    T, V, D = 130, 1024, 4096
    g = gen(790)
    row = (0.5 + torch.rand(D, generator=g, device=DEV)).to(dtype)
    h = (0.2 + 0.1 * torch.rand(T, D, generator=g, device=DEV)).to(dtype)
    w = row.expand(V, D).contiguous()
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    plan = losses.HeadLoss(T, V, D, dtype, piece_bytes=1)  # pieces of 256 columns: all but one from a second product
    lse = plan.cross_entropy(h, w, y).lse if saved else None
    dw = torch.empty(V, D, device=DEV)
    plan.cross_entropy_grad(h, w, y, reduction="sum", lse=lse, dweight=dw, want=("weight",))
    cols = torch.bincount(y, minlength=V) == 0
    want = (2.0**-10 * h.double().sum(0)).expand(int(cols.sum()), D)
    within(dw[cols], want, (T / 16 + 8) * 2.0**-22 * want, "dweight")


def test_long_sums_of_one_sign():
    """Rows whose logits are all equal have p = 2^-k exactly, and a factor of -1 (rounded) at the target.  The gradients are then
    sums of exactly known terms, here of one sign.  Sums of at most 1024 terms in the tensor cores lose (1024 / 16 + 2) 2^-22 of
    themselves at most, adding those up in fp32 2^-24 each: below 2^-15 in all.  (Left to the tensor cores alone, 65536
    terms came out 4e-4 low, 32768 7e-5.)"""
    for T, V, D in ((8192, 65536, 1024), (32768, 1024, 128)):
        g = gen(820)
        w = (torch.rand(V, D, generator=g, device=DEV) ** 4).to(BF)
        w[:, :64] = 1.0
        h = torch.zeros(T, D, device=DEV, dtype=BF)
        h[:, :64] = (torch.rand(T, 64, generator=g, device=DEV) ** 4).to(BF)
        y = torch.randint(0, V // 2, (T,), generator=g, device=DEV)
        plan = losses.HeadLoss(T, V, D, BF)
        dh, dw = torch.empty(T, D, device=DEV), torch.empty(V, D, device=DEV)
        plan.cross_entropy_grad(h, w, y, reduction="sum", dhidden=dh, dweight=dw)
        rows = slice(T - 256, T)
        total = sum(w[i : i + 4096, 64:].double().sum(0) for i in range(0, V, 4096)) / V
        own = w[y[rows], 64:].double()
        at = torch.tensor(1 / V - 1, device=DEV).to(BF).double()
        want = total - own / V + at * own
        within(dh[rows, 64:], want, 2.0**-15 * (total + own), "dhidden")
        want = (h[:, :64].double().sum(0) / V).expand(V - V // 2, 64)
        within(dw[V // 2 :, :64], want, 2.0**-15 * want, "dweight")


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D,piece", [(130, 700, 72, 0), (300, 2000, 264, 1), (40, 300, 33, 0), (1100, 500, 64, 0)])
def test_rows_that_give_nothing_may_hold_anything(T, V, D, piece, dtype, saved):
    """NaN and infinities in the hidden states of rows without a target, or without an upstream gradient, reach nothing:
    all results are those of the same rows filled with zeros."""
    g = gen(840 + T)
    h = torch.randn(T, D, generator=g, device=DEV).to(dtype)
    w = (torch.randn(V, D, generator=g, device=DEV) / math.sqrt(D)).to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    off = torch.rand(T, generator=g, device=DEV) < 0.2
    off[1], off[2] = True, False
    clean, dirty = h.clone(), h.clone()
    clean[off] = 0
    junk = torch.tensor([math.nan, math.inf, -math.inf, 0.0], device=DEV)[torch.randint(0, 4, (T, D), generator=g, device=DEV)].to(dtype)
    junk[:, D // 2] = math.nan
    junk[::2] = math.inf  # a row of nothing but infinities
    dirty[off] = junk[off]
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :5].contiguous()
    teacher = torch.randn(T, 5, generator=g, device=DEV)
    up = torch.where(off, 0.0, torch.randn(T, generator=g, device=DEV))
    y_off, ids_off = torch.where(off, -100, y), torch.where(off[:, None], -1, ids)
    plan = losses.HeadLoss(T, V, D, dtype, top_k=5, piece_bytes=piece)
    calls = [
        (plan.cross_entropy, plan.cross_entropy_grad, (y_off,), {}),
        (plan.distill, plan.distill_grad, (ids_off, teacher, 2.0), {}),
        (plan.cross_entropy, plan.cross_entropy_grad, (y,), dict(dloss=up)),
    ]
    for forward, grad, args, kw in calls:
        out = []
        for hidden in (dirty, clean):
            lse = forward(hidden, w, *args).lse.clone() if saved else None
            r = grad(hidden, w, *args, lse=lse, reduction="sum", dweight=torch.empty(V, D, device=DEV), **kw)
            out.append((r.dhidden, r.dweight))
        for a, b in zip(*out):
            assert torch.isfinite(a.float()).all() and torch.equal(a, b)
        again = grad(clean, w, *args, reduction="sum", dweight=torch.empty(V, D, device=DEV), **kw)  # and leave nothing behind
        if not saved:
            assert torch.equal(again.dweight, out[1][1])
    assert plan.status() == 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D,piece,pad", [(130, 700, 72, 0, 0), (130, 700, 72, 0, 3), (40, 8192, 512, 0, 8), (300, 2000, 33, 1, 0), (1500, 900, 200, 0, 5)])
def test_gradients_of_16_bits_accumulate(T, V, D, piece, pad, dtype):
    """Added to what is there in fp32 and rounded once; in rows of any alignment, and nothing beside them."""
    g = gen(860 + T + pad)
    h = torch.randn(T, D, generator=g, device=DEV).to(dtype)
    w = (torch.randn(V, D, generator=g, device=DEV) / math.sqrt(D)).to(dtype)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :6].contiguous()
    teacher = torch.randn(T, 6, generator=g, device=DEV) * 2
    plan = losses.HeadLoss(T, V, D, dtype, top_k=6, piece_bytes=piece)
    plain = [torch.zeros(n, D, device=DEV) for n in (T, V)]
    plan.distill_grad(h, w, ids, teacher, 1.5, reduction="sum", dhidden=plain[0], dweight=plain[1])
    wide = [torch.randn(n, D + pad, generator=g, device=DEV).to(dtype) for n in (T, V)]
    old = [x.clone() for x in wide]
    views = [x[:, pad // 2 : pad // 2 + D] for x in wide]
    plan.distill_grad(h, w, ids, teacher, 1.5, reduction="sum", dhidden=views[0], dweight=views[1], accumulate=True)
    for x, before, got, grad in zip(wide, old, views, plain):
        want = before[:, pad // 2 : pad // 2 + D].double() + grad.double()
        # the fp32 gradients are the same products: only the sum's two roundings differ
        within(got, want, 1.01 * U[dtype] * want.abs() + 2.0**-22 * (grad.double().abs() + want.abs()) + TINY[dtype], "sum")
        x[:, pad // 2 : pad // 2 + D] = before[:, pad // 2 : pad // 2 + D]
        assert torch.equal(x, before)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,n,K", [(50, 300, 64, 9), (150, 700, 128, 50), (33, 1100, 72, 64), (300, 2049, 64, 7)])
def test_distillation_does_not_depend_on_the_pieces(T, V, n, K, dtype):
    """The rows' losses are the same bits whatever the pieces; gradients differ by what a code may (see factor_error)."""
    h, w, g = identity_head(T, V, n, dtype, 880 + T)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :K].contiguous()
    teacher = torch.randn(T, K, generator=g, device=DEV) * 3
    q = torch.zeros(T, V, dtype=torch.float64, device=DEV).scatter_(1, ids, soft_targets(ids, teacher, 1.0))
    hit = torch.zeros(T, V, dtype=torch.bool, device=DEV).scatter_(1, ids, True)
    p = torch.softmax(torch.cat([h.double(), torch.zeros(T, V - n, dtype=torch.float64, device=DEV)], 1), 1)
    f_err = factor_error(p, q, dtype, hit)[:, :n]
    first = None
    for piece in (0, 1, 2 * T * 512, 2 * T * 768):
        plan = losses.HeadLoss(T, V, n, dtype, top_k=K, piece_bytes=piece)
        dh = torch.empty(T, n, device=DEV)
        r = plan.distill_grad(h, w, ids, teacher, reduction="sum", dhidden=dh)
        within(dh, (p - q)[:, :n], f_err + 2.0**-23 * (p - q)[:, :n].abs(), "dhidden")
        if first is None:
            first = r
        assert torch.equal(r.rows, first.rows) and torch.equal(r.lse, first.lse)
