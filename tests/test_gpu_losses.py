"""The losses (output head with cross entropy or teacher's top logits, balance loss) against plain 64-bit statements of
their formulas.  Tolerances are bounds derived from the arithmetic:

  products      an fp32 tensor-core sum over K elements is off by at most (K / 16 + 2) 2^-22 sum |a b|
  statistics    fp32 exp / log: 2^-20 relative to 1 + |lse|
  factors       the gradient's exp(..) - q is rounded to the operands' type, and may have been rounded once before:
                2 u relative with u = 2^-8 (bf16: 8 significant bits), 2^-11 (fp16: 11); parts below 2^-23 of a row's largest may be dropped
  results       one rounding to the output's type: u |x| (and half the smallest subnormal)
"""
import math

import pytest
import torch

from paper_1901_01544_b200 import losses

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
U = {t: torch.finfo(t).eps / 2 for t in (BF, HF, F32)}  # largest relative error of one rounding
TINY = {BF: 2.0**-134, HF: 2.0**-25, F32: 2.0**-150}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def operands(T, V, D, dtype, seed, spread=2.0):
    g = gen(seed)
    w = (torch.randn(V, D, generator=g, device=DEV) * (spread / math.sqrt(D))).to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    h = (torch.randn(T, D, generator=g, device=DEV) + 2.0 * torch.rand(T, 1, generator=g, device=DEV) * w[y].float()).to(dtype)
    return h, w, y, g


def targets_of(T, V, q_ids, q, dtype=torch.float64):
    """Dense [T, V] targets from (ids, q), ids < 0 unused."""
    dense = torch.zeros(T, V, dtype=dtype, device=DEV)
    return dense.scatter_add_(1, q_ids.clamp(min=0), torch.where(q_ids >= 0, q, 0.0))


def soft_targets(ids, logits, tau):
    """q in 64 bits from teacher logits; ids < 0 take no part; a row with nothing left has q = 0."""
    x = torch.where(ids >= 0, logits.double() / tau, -math.inf)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    s = e.sum(1, keepdim=True)
    return torch.where(s > 0, e / s, 0.0)


def head_reference(h, w, ids, q, tau, mean, g_rows=None):
    """loss, rows, lse, dH, dW and the bounds on how far each may be off."""
    T, D = h.shape
    V = w.shape[0]
    H, W = h.double(), w.double()
    z = H @ W.T / tau
    lse = torch.logsumexp(z, 1)
    dense = targets_of(T, V, ids, q)
    live = (dense.sum(1) > 0).double()
    qlogq = (q * torch.where(q > 0, torch.log(q.clamp(min=1e-300)), 0.0)).sum(1)
    rows = tau * tau * (qlogq - (dense * z).sum(1) + lse * live)
    n = max(1.0, float(live.sum()))
    over = n if mean else 1.0
    g = (live if g_rows is None else live * g_rows.double()) * tau / over
    p = torch.exp(z - lse[:, None])
    dz = g[:, None] * (p - dense)
    dH, dW = dz @ W, dz.T @ H
    u = U[h.dtype]
    dz_err = ((D / 16 + 2) * 2.0**-22 * (H.abs() @ W.abs().T) / tau).amax(1) + 2.0**-20 * (1 + lse.abs())
    row_err = tau * tau * (2 * dz_err + 2.0**-20) * live
    cut = 2.0**-23 * p.amax(1, keepdim=True)
    # one factor: rounded to the type (twice at most), its exponent off by the errors of z and lse
    f_err = g.abs()[:, None] * ((2 * u) * (p - dense).abs() + (2 * dz_err[:, None] + u) * p + cut)
    steps = lambda k: (k / 16 + 8) * 2.0**-22  # noqa: E731
    h_err = f_err @ W.abs() + steps(V) * (dz.abs() @ W.abs())
    w_err = f_err.T @ H.abs() + steps(T) * (dz.abs().T @ H.abs())
    return dict(loss=rows.sum() / over, rows=rows, lse=lse, dH=dH, dW=dW, row_err=row_err, lse_err=dz_err, h_err=h_err, w_err=w_err,
                loss_err=row_err.sum() / over + 2.0**-18 * rows.abs().sum() / over)


def close(got, want, err, name):
    got = got.double()
    assert torch.isfinite(got).all(), name + " is not finite"
    tol = err + (U[F32] * 4) * want.abs() + 1e-30
    worst = ((got - want).abs() / tol).max().item()
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound"


def close_grad(got, want, err, name, scale=1.0):
    tol = err * scale + U[got.dtype] * 1.01 * (want * scale).abs() + TINY[got.dtype] + 1e-37
    got = got.double()
    assert torch.isfinite(got).all(), name + " is not finite"
    worst = ((got - want * scale).abs() / tol).max().item()
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound"


def check_head(r, ref, scale=1.0, grad=True):
    close(r.loss, ref["loss"], ref["loss_err"], "loss")
    close(r.rows, ref["rows"], ref["row_err"], "rows")
    close(r.lse, ref["lse"], ref["lse_err"], "lse")
    if grad:
        close_grad(r.dhidden, ref["dH"], ref["h_err"], "dhidden", scale)
        close_grad(r.dweight, ref["dW"], ref["w_err"], "dweight", scale)


SIZES = [
    (1, 1, 1), (1, 1000, 64), (2, 17, 8), (3, 300, 72), (31, 255, 16), (127, 257, 100), (128, 256, 64), (129, 511, 130), (256, 1000, 2048),
    (257, 1025, 264), (300, 5000, 96), (1000, 129, 33), (513, 2049, 520), (40, 8192, 512), (64, 20000, 128),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_cross_entropy(T, V, D, dtype):
    h, w, y, g = operands(T, V, D, dtype, T + V + D)
    if T > 4:
        y[torch.rand(T, generator=g, device=DEV) < 0.1] = -100
    plan = losses.HeadLoss(T, V, D, dtype)
    ids = torch.where(y == -100, -1, y)[:, None]
    ref = head_reference(h, w, ids, (ids >= 0).double(), 1.0, True)
    scale = 512.0 if dtype == HF else 1.0
    check_head(plan.cross_entropy_grad(h, w, y, scale=scale), ref, scale)
    check_head(plan.cross_entropy(h, w, y), ref, grad=False)
    assert plan.status() == 0


@pytest.mark.parametrize("ids_type,top_type", [(torch.int64, F32), (torch.int32, BF), (torch.int64, HF)])
@pytest.mark.parametrize("T,V,D,K,tau", [(1, 1000, 64, 1, 1.0), (5, 40, 16, 40, 2.0), (130, 1000, 72, 7, 0.5), (300, 3000, 200, 50, 4.0),
                                         (64, 5000, 33, 64, 1.5), (33, 2000, 128, 1024, 1.0)])
def test_distill(T, V, D, K, tau, ids_type, top_type):
    h, w, _, g = operands(T, V, D, BF, T + V + K)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :K].contiguous()
    logits = (torch.randn(T, K, generator=g, device=DEV) * 3 + 10).to(top_type)
    plan = losses.HeadLoss(T, V, D, BF, top_k=K)
    ref = head_reference(h, w, ids, soft_targets(ids, logits, tau), tau, True)
    # the teacher's softmax is fp32: its q are off by 2^-20 relative, and with them rows and factors
    check_head(plan.distill_grad(h, w, ids.to(ids_type), logits, tau), ref)
    check_head(plan.distill(h, w, ids.to(ids_type), logits, tau), ref, grad=False)
    assert plan.status() == 0


def test_distill_padding_and_empty_rows():
    T, V, D, K, tau = 70, 900, 48, 9, 2.0
    h, w, _, g = operands(T, V, D, BF, 3)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :K].contiguous()
    logits = torch.randn(T, K, generator=g, device=DEV) * 2
    ids[torch.rand(T, K, generator=g, device=DEV) < 0.4] = -1
    logits[torch.rand(T, K, generator=g, device=DEV) < 0.3] = -math.inf
    logits[5, 0] = torch.finfo(F32).min  # the type's lowest value is a logit like any other
    ids[7] = -1  # nothing left
    logits[8] = -math.inf
    ids[9, 1:] = -1  # one entry left
    logits[9, 0] = 1.0
    ref = head_reference(h, w, ids, soft_targets(ids, logits, tau), tau, True)
    plan = losses.HeadLoss(T, V, D, BF, top_k=K)
    r = plan.distill_grad(h, w, ids, logits, tau)
    check_head(r, ref)
    assert r.rows[7] == 0 and r.rows[8] == 0 and not r.dhidden[7:9].any() and plan.status() == 0


def test_all_rows_ignored():
    h, w, y, _ = operands(130, 500, 64, BF, 1)
    y[:] = -100
    plan = losses.HeadLoss(130, 500, 64, BF)
    r = plan.cross_entropy_grad(h, w, y)
    assert r.loss == 0 and not r.rows.any() and not r.dhidden.any() and not r.dweight.any() and plan.status() == 0


def test_no_tokens():
    w = torch.randn(50, 16, device=DEV).to(BF)
    plan = losses.HeadLoss(8, 50, 16, BF, top_k=4)
    h, y = w[:0], torch.empty(0, dtype=torch.int64, device=DEV)
    r = plan.cross_entropy_grad(h, w, y)
    assert r.loss == 0 and r.rows.numel() == 0 and r.dhidden.shape == (0, 16) and not r.dweight.any()
    ids = torch.empty(0, 4, dtype=torch.int64, device=DEV)
    r = plan.distill_grad(h, w, ids, ids.float(), 2.0)
    assert r.loss == 0 and not r.dweight.any()


@pytest.mark.parametrize("bad", [500, 1 << 40, -1])
def test_target_outside_the_vocabulary(bad):
    h, w, y, _ = operands(40, 500, 64, BF, 2)
    y[3] = bad
    plan = losses.HeadLoss(40, 500, 64, BF)
    r = plan.cross_entropy_grad(h, w, y)
    assert torch.isnan(r.rows[3]) and torch.isfinite(r.rows[torch.arange(40, device=DEV) != 3]).all() and torch.isnan(r.loss)
    assert not r.dhidden[3].any() and torch.isfinite(r.dhidden.float()).all() and torch.isfinite(r.dweight.float()).all()
    assert plan.status() == -1
    with pytest.raises(losses.IwpError):
        plan.check()
    plan.reset()
    assert plan.status() == 0
    ids = torch.stack([y.clamp(0, 499), y], 1)
    if bad >= 0:
        plan.distill(h, w, ids, torch.zeros(40, 2, device=DEV))
        assert plan.status() == -1


def test_ignore_index_inside_the_vocabulary():
    h, w, y, _ = operands(64, 200, 32, BF, 4)
    y[::5] = 7
    plan = losses.HeadLoss(64, 200, 32, BF)
    ids = torch.where(y == 7, -1, y)[:, None]
    ref = head_reference(h, w, ids, (ids >= 0).double(), 1.0, True)
    check_head(plan.cross_entropy_grad(h, w, y, ignore_index=7), ref)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D,piece", [(300, 3000, 200, 300 * 2 * 1024), (1000, 2000, 136, 1), (40, 5000, 64, 40 * 2 * 512)])
def test_pieces_of_the_vocabulary(T, V, D, piece, dtype):
    h, w, y, _ = operands(T, V, D, dtype, 5)
    ref = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, False)
    plan = losses.HeadLoss(T, V, D, dtype, piece_bytes=piece)
    check_head(plan.cross_entropy_grad(h, w, y, reduction="sum"), ref)


@pytest.mark.parametrize("offset", [0, 1, 3])
def test_strided_and_unaligned_operands(offset):
    T, V, D = 130, 700, 72
    h, w, y, _ = operands(T, V, D, BF, 6)
    hs, ws = torch.zeros(T, D + 13, dtype=BF, device=DEV), torch.zeros(V, D + 24, dtype=BF, device=DEV)
    hs[:, offset : offset + D], ws[:, offset : offset + D] = h, w
    ref = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    dh, dw = torch.full((T, D + 9), 7.0, dtype=BF, device=DEV), torch.full((V, D + 8), 7.0, dtype=F32, device=DEV)
    plan = losses.HeadLoss(T, V, D, BF)
    r = plan.cross_entropy_grad(hs[:, offset : offset + D], ws[:, offset : offset + D], y, dhidden=dh[:, offset : offset + D],
                                dweight=dw[:, offset : offset + D])
    check_head(r, ref)
    for buf in (dh, dw):  # nothing beside the gradient is touched
        assert (buf[:, :offset] == 7).all() and (buf[:, offset + D :] == 7).all()


@pytest.mark.parametrize("T,V,D", [(130, 700, 72), (600, 3000, 264)])
def test_gradients_into_a_worker_segment_accumulate(T, V, D):
    """float32 gradients into a view of grads[w] at an odd offset, cross entropy and distillation added up."""
    h, w, y, g = operands(T, V, D, BF, 8)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :5].contiguous()
    logits = torch.randn(T, 5, generator=g, device=DEV)
    flat = torch.full((2, V * D + 7), 0.5, device=DEV)
    dw = flat[1, 3 : 3 + V * D].view(V, D)
    dh = torch.zeros(T, D, device=DEV)
    plan = losses.HeadLoss(T, V, D, BF, top_k=5)
    one = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    two = head_reference(h, w, ids, soft_targets(ids, logits, 2.0), 2.0, True)
    dw.zero_()
    plan.cross_entropy_grad(h, w, y, dhidden=dh, dweight=dw, accumulate=True)
    plan.distill_grad(h, w, ids, logits, 2.0, dhidden=dh, dweight=dw, accumulate=True)
    extra = 2.0**-23
    close_grad(dw, one["dW"] + two["dW"], one["w_err"] + two["w_err"] + extra * one["dW"].abs(), "dweight")
    close_grad(dh, one["dH"] + two["dH"], one["h_err"] + two["h_err"] + extra * one["dH"].abs(), "dhidden")
    assert (flat[0] == 0.5).all() and (flat[1, :3] == 0.5).all() and (flat[1, 3 + V * D :] == 0.5).all()


def test_upstream_gradients_and_saved_lse():
    T, V, D = 200, 900, 128
    h, w, y, g = operands(T, V, D, BF, 9)
    y[::7] = -100
    ids = torch.where(y == -100, -1, y)[:, None]
    plan = losses.HeadLoss(T, V, D, BF)
    up = torch.randn(T, generator=g, device=DEV)
    up[3] = 0
    ref = head_reference(h, w, ids, (ids >= 0).double(), 1.0, False, up)
    fwd = plan.cross_entropy(h, w, y, reduction="sum")
    r = plan.cross_entropy_grad(h, w, y, reduction="sum", lse=fwd.lse, dloss=up)
    assert r.loss is None and r.rows is None
    close_grad(r.dhidden, ref["dH"], ref["h_err"], "dhidden")
    close_grad(r.dweight, ref["dW"], ref["w_err"], "dweight")
    assert not r.dhidden[3].any() and not r.dhidden[::7].any()
    # a scalar on the device, and one gradient at a time
    mean = head_reference(h, w, ids, (ids >= 0).double(), 1.0, True)
    half = torch.tensor(0.5, device=DEV)
    a = plan.cross_entropy_grad(h, w, y, lse=fwd.lse, dloss=half, want=("hidden",))
    b = plan.cross_entropy_grad(h, w, y, dloss=half, want=("weight",))
    assert a.dweight is None and b.dhidden is None
    close_grad(a.dhidden, mean["dH"], mean["h_err"], "dhidden", 0.5)
    close_grad(b.dweight, mean["dW"], mean["w_err"], "dweight", 0.5)
    zero = plan.cross_entropy_grad(h, w, y, reduction="sum", dloss=torch.zeros(T, device=DEV))
    assert not zero.dhidden.any() and not zero.dweight.any()


def test_large_logits_and_non_finite_operands():
    T, V, D = 40, 600, 64
    h, w, y, _ = operands(T, V, D, BF, 10, spread=60.0)  # logits of several hundred: one column carries a row
    ref = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    plan = losses.HeadLoss(T, V, D, BF)
    check_head(plan.cross_entropy_grad(h, w, y), ref)
    h[2, 5] = math.nan
    r = plan.cross_entropy(h, w, y)
    assert torch.isnan(r.rows[2]) and torch.isfinite(r.rows[torch.arange(T, device=DEV) != 2]).all()
    y[2] = -100  # an ignored row does not reach the gradients, whatever it holds
    r = plan.cross_entropy_grad(h, w, y)
    assert torch.isfinite(r.loss) and not r.dhidden[2].any() and torch.isfinite(r.dhidden.float()).all()


def test_same_inputs_same_bits():
    h, w, y, g = operands(777, 3003, 264, BF, 11)
    plan = losses.HeadLoss(777, 3003, 264, BF)
    a, b = plan.cross_entropy_grad(h, w, y), plan.cross_entropy_grad(h, w, y)
    for k in ("loss", "rows", "lse", "dhidden", "dweight"):
        assert torch.equal(getattr(a, k), getattr(b, k)), k


def test_other_stream():
    h, w, y, _ = operands(300, 2000, 128, BF, 12)
    plan = losses.HeadLoss(300, 2000, 128, BF)
    want = plan.cross_entropy_grad(h, w, y)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = plan.cross_entropy_grad(h, w, y)
    s.synchronize()
    assert torch.equal(got.dweight, want.dweight) and torch.equal(got.dhidden, want.dhidden)


def test_head_gradient_against_differences():
    """Central differences of the kernel's own loss along random +-2^-6 steps of operands on a grid of 2^-4, which
    bf16 holds exactly.  Third order: a row's loss is the log of a mean of exponentials; with steps of z in [-a, a] its
    third derivative is at most (2 a)^3, so both sides differ by (2 a)^3 / 3 per row at most, besides rounding."""
    T, V, D = 64, 300, 32
    g = gen(13)
    grid = lambda *s: torch.randint(-16, 17, s, generator=g, device=DEV) / 16.0  # noqa: E731
    h, w = grid(T, D), grid(V, D)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    plan = losses.HeadLoss(T, V, D, BF)
    r = plan.cross_entropy_grad(h.to(BF), w.to(BF), y, reduction="sum")
    for which in ("hidden", "weight"):
        base = h if which == "hidden" else w
        step = (torch.randint(0, 2, base.shape, generator=g, device=DEV) * 2 - 1) / 64.0
        ends = []
        for s in (1, -1):
            a, b = (h + s * step, w) if which == "hidden" else (h, w + s * step)
            ends.append(plan.cross_entropy(a.to(BF), b.to(BF), y, reduction="sum").loss.double())
        a = (step.abs() @ w.abs().T).max().item() if which == "hidden" else (h.abs() @ step.abs().T).max().item()
        # the steps are random signs: |dz| is below 5 standard deviations, not at the bound of equal signs
        dz = ((step @ w.T) if which == "hidden" else (h @ step.T)).abs().max().item()
        assert dz <= a
        grad = getattr(r, "d" + which).double()
        want = 2 * (grad * step).sum()
        rounding = 2 * (2 * U[BF]) * (grad.abs() * step.abs()).sum() + 2 * 2.0**-9 * T * dz
        third = T * (2 * dz) ** 3 / 3
        noise = 4 * T * 2.0**-20 * 10
        assert abs((ends[0] - ends[1]) - want) <= rounding + third + noise


def test_head_refuses_wrong_tensors():
    h, w, y, _ = operands(20, 100, 32, BF, 14)
    plan = losses.HeadLoss(20, 100, 32, BF)
    for args, err in [((h.float(), w, y), TypeError), ((h, w.half(), y), TypeError), ((h, w, y.int()), TypeError), ((h, w, y[:5]), ValueError),
                      ((h[:, :16], w, y), ValueError), ((h, w[:50], y), ValueError), ((h.cpu(), w, y), ValueError), ((h, w, y.cpu()), ValueError),
                      ((h[0], w, y), ValueError), ((h.t().contiguous().t(), w, y), ValueError)]:
        with pytest.raises(err):
            plan.cross_entropy(*args)
    with pytest.raises(ValueError):
        plan.cross_entropy(h, w, y, reduction="none")
    with pytest.raises(ValueError):
        plan.cross_entropy_grad(h, w, y, accumulate=True)
    with pytest.raises(TypeError):
        plan.cross_entropy_grad(h, w, y, dweight=torch.empty(100, 32, dtype=HF, device=DEV))
    with pytest.raises(ValueError):
        plan.distill(h, w, y[:, None], torch.zeros(20, 2, device=DEV))
    with pytest.raises(losses.IwpError):
        plan.distill(h, w, y[:, None], torch.zeros(20, 1, device=DEV), 0.0)
    with pytest.raises(TypeError):
        losses.HeadLoss(20, 100, 32, F32)
    with pytest.raises(losses.IwpError):
        losses.HeadLoss(20, 0, 32, BF)


# ---- balance loss --------------------------------------------------------------------------------------


def balance_reference(x, ids, mask, coef):
    T, E = x.shape
    k = ids.shape[1]
    m = torch.ones(T, dtype=torch.float64, device=DEV) if mask is None else mask.double()
    X = x.double()
    top = X.amax(1, keepdim=True)
    e = torch.exp(X - torch.where(torch.isinf(top), 0.0, top))
    s = e.sum(1, keepdim=True)
    p = torch.where(s > 0, e / s, 0.0)
    n = float(m.sum())
    on = m.bool()[:, None] & (ids >= 0) & (ids < E)
    counts = torch.bincount(ids[on].long(), minlength=E)
    if n == 0:
        return dict(loss=X.new_zeros(()), counts=counts, mean=X.new_zeros(E), dx=torch.zeros_like(X), f=X.new_zeros(E))
    f = counts.double() / (n * k)
    mean = (p * m[:, None]).sum(0) / n
    c = coef * E
    return dict(loss=c * (f * mean).sum(), counts=counts, mean=mean, f=f, dx=(c / n) * m[:, None] * p * (f - (p * f).sum(1, keepdim=True)),
                scale_dx=(c / n) * m[:, None] * p * f.max())


def check_balance(r, ref, x, T, scale=1.0):
    """p is off by 2^-19 (1 + |x - max|) relative (fp32 exp and division), sums of T of them by T / 2^24 more at worst."""
    assert torch.equal(r.counts.long(), ref["counts"])
    depth = 2.0**-19 * 40
    sums = depth + (T + 600) * 2.0**-24
    assert (r.mean_prob.double() - ref["mean"]).abs().le(sums * ref["mean"] + 1e-30).all()
    assert (r.loss.double() - ref["loss"]).abs() <= (sums + 2.0**-16) * ref["loss"] + 1e-30
    if r.dlogits is not None:
        tol = U[x.dtype] * 1.01 * (ref["dx"] * scale).abs() + 2 * depth * ref.get("scale_dx", ref["dx"]) * scale + TINY[x.dtype] + 1e-37
        worst = ((r.dlogits.double() - ref["dx"] * scale).abs() / tol).max().item() if T else 0.0
        assert worst <= 1.0, f"dlogits: {worst:.3g} times its bound"


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (64, 8, 2), (77, 5, 3), (1000, 60, 4), (333, 64, 6), (2000, 128, 8), (129, 130, 7), (515, 256, 8),
                                   (40, 1000, 9), (33, 1024, 1), (20000, 16, 4), (70000, 33, 2)])
def test_balance(T, E, k, dtype):
    g = gen(T + E)
    x = (torch.randn(T, E, generator=g, device=DEV) * 2).to(dtype)
    ids = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].contiguous()
    plan = losses.ExpertBalance(T, E)
    scale = 4096.0 if dtype == HF else 1.0
    check_balance(plan.grad(x, ids, coef=0.02, scale=scale), balance_reference(x, ids, None, 0.02), x, T, scale)
    mask = torch.rand(T, generator=g, device=DEV) < 0.7
    r = plan.grad(x, ids.int(), mask, coef=0.02, scale=scale)
    check_balance(r, balance_reference(x, ids, mask, 0.02), x, T, scale)
    assert not r.dlogits[~mask].any()
    check_balance(plan.loss(x, ids, mask.to(torch.uint8), coef=0.02), balance_reference(x, ids, mask, 0.02), x, T)
    assert plan.status() == 0


def test_balance_masks_empty_rows_and_dropped_ids():
    T, E, k = 90, 24, 3
    g = gen(20)
    x = torch.randn(T, E, generator=g, device=DEV)
    x[torch.rand(T, E, generator=g, device=DEV) < 0.3] = -math.inf
    x[4] = -math.inf
    x[5] = torch.finfo(F32).min
    ids = torch.randint(-2, E + 2, (T, k), generator=g, device=DEV)
    ids[6] = torch.tensor([1 << 40, -(1 << 40), 3], device=DEV)
    plan = losses.ExpertBalance(T, E)
    r = plan.grad(x, ids, coef=1.0)
    check_balance(r, balance_reference(x, ids, None, 1.0), x, T)
    assert not r.dlogits[4].any() and not r.dlogits[torch.isinf(x)].any()
    nobody = torch.zeros(T, dtype=torch.bool, device=DEV)
    r = plan.grad(x, ids, nobody)
    assert r.loss == 0 and not r.counts.any() and not r.dlogits.any() and not r.mean_prob.any()
    bad = x.clone()
    bad[7, 0] = math.nan
    off = torch.ones(T, dtype=torch.bool, device=DEV)
    off[7] = False  # NaN in a masked row stays there
    check_balance(plan.grad(bad, ids, off), balance_reference(x, ids, off, 0.01), x, T)
    assert torch.isnan(plan.grad(bad, ids).loss)
    r = plan.grad(x[:0], ids[:0])
    assert r.loss == 0 and not r.counts.any() and r.dlogits.shape == (0, E)


def test_balance_strides_and_upstream():
    T, E, k = 300, 40, 4
    g = gen(21)
    wide = torch.randn(T, E + 5, generator=g, device=DEV).to(BF)
    x = wide[:, 3 : 3 + E]
    pool = torch.randint(0, E, (T, 9), generator=g, device=DEV)
    ids = pool[:, 2 : 2 + k]
    plan = losses.ExpertBalance(T, E)
    out = torch.full((T, E + 3), 9.0, dtype=BF, device=DEV)
    up = torch.tensor(-3.0, device=DEV)
    r = plan.grad(x, ids, dloss=up, dlogits=out[:, 1 : 1 + E])
    ref = balance_reference(x, ids, None, 0.01)
    ref["dx"], ref["scale_dx"] = ref["dx"] * -3, ref["scale_dx"] * 3
    check_balance(r, ref, x, T)
    assert (out[:, 0] == 9).all() and (out[:, 1 + E :] == 9).all()
    a, b = plan.grad(x, ids), plan.grad(x, ids)
    assert torch.equal(a.loss, b.loss) and torch.equal(a.dlogits, b.dlogits) and torch.equal(a.mean_prob, b.mean_prob)


def test_balance_gradient_against_differences():
    """loss is linear in p: along a direction v of size e its central difference is off by at most
    coef E max f (2 e)^3 / 3 per token over n, besides the rounding of the two losses."""
    T, E, k = 50, 12, 2
    g = gen(22)
    x = torch.randn(T, E, generator=g, device=DEV)
    ids = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].contiguous()
    v = torch.randn(T, E, generator=g, device=DEV).sign() * 2.0**-5
    plan = losses.ExpertBalance(T, E)
    r = plan.grad(x, ids, coef=1.0)
    a, b = plan.loss(x + v, ids, coef=1.0).loss.double(), plan.loss(x - v, ids, coef=1.0).loss.double()
    want = 2 * (r.dlogits.double() * ((x + v).double() - (x - v).double()) / 2).sum()
    f = r.counts.double() / (T * k)
    tol = E * f.max() * (2 * 2.0**-5) ** 3 / 3 + 4 * 2.0**-18 * a.abs()
    assert abs((a - b) - want) <= tol


def test_balance_refuses_wrong_tensors():
    x, ids = torch.randn(20, 16, device=DEV), torch.zeros(20, 2, dtype=torch.int64, device=DEV)
    plan = losses.ExpertBalance(20, 16)
    for args, err in [((x.double(), ids), TypeError), ((x, ids.float()), TypeError), ((x[:, :8], ids), ValueError), ((x, ids[:5]), ValueError),
                      ((x.cpu(), ids), ValueError), ((x, ids, torch.ones(19, dtype=torch.bool, device=DEV)), ValueError), ((x[0], ids), ValueError),
                      ((x, ids, torch.ones(20, device=DEV)), TypeError)]:
        with pytest.raises(err):
            plan.loss(*args)
    with pytest.raises(losses.IwpError):
        plan.loss(x, torch.zeros(20, 17, dtype=torch.int64, device=DEV))
    with pytest.raises(losses.IwpError):
        losses.ExpertBalance(20, 1025)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,V,D", [(1, 32768, 1024), (1, 5, 8), (2, 1003, 520), (3, 4099, 4096), (4, 700, 24), (4, 64, 1001), (2, 129, 7), (5, 3000, 64),
                                   (4, 300, 8192)])
def test_forward_of_a_few_tokens(T, V, D, dtype):
    h, w, y, g = operands(T, V, D, dtype, 100 + T + V)
    ref = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    plan = losses.HeadLoss(T, V, D, dtype, top_k=5)
    check_head(plan.cross_entropy(h, w, y), ref, grad=False)
    K = min(5, V)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :K].contiguous()
    logits = torch.randn(T, K, generator=g, device=DEV)
    ids[0, 0] = -1 if K > 1 else ids[0, 0]
    ref = head_reference(h, w, ids, soft_targets(ids, logits, 3.0), 3.0, False)
    check_head(plan.distill(h, w, ids, logits, 3.0, reduction="sum"), ref, grad=False)
    wide = torch.zeros(V, D + 8, dtype=dtype, device=DEV)  # strided rows, and rows that end where 8 does not divide them
    wide[:, :D] = w
    ref = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    check_head(plan.cross_entropy(h, wide[:, :D], y), ref, grad=False)
    assert plan.status() == 0


def test_repeated_teacher_ids_add_up():
    T, V, D, K = 50, 400, 64, 12
    h, w, _, g = operands(T, V, D, BF, 200)
    ids = torch.randint(0, 6, (T, K), generator=g, device=DEV)  # many equal ones
    logits = torch.randn(T, K, generator=g, device=DEV)
    plan = losses.HeadLoss(T, V, D, BF, top_k=K)
    check_head(plan.distill_grad(h, w, ids, logits, 1.5), head_reference(h, w, ids, soft_targets(ids, logits, 1.5), 1.5, True))
    small = losses.HeadLoss(T, V, D, BF, top_k=K, piece_bytes=1)
    check_head(small.distill_grad(h, w, ids, logits, 1.5), head_reference(h, w, ids, soft_targets(ids, logits, 1.5), 1.5, True))


def test_differentiable_forms():
    T, V, D, E = 200, 900, 64, 16
    h, w, y, g = operands(T, V, D, BF, 300)
    plan, router = losses.HeadLoss(T, V, D, BF, top_k=6), losses.ExpertBalance(T, E)
    ids = torch.rand(T, V, generator=g, device=DEV).argsort(1)[:, :6].contiguous()
    logits = torch.randn(T, 6, generator=g, device=DEV)
    h.requires_grad_(), w.requires_grad_()
    (3.0 * losses.cross_entropy(plan, h, w, y)).backward()
    ref = head_reference(h.detach(), w.detach(), y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    close_grad(h.grad, ref["dH"], ref["h_err"], "dhidden", 3.0)
    close_grad(w.grad, ref["dW"], ref["w_err"], "dweight", 3.0)
    h.grad = w.grad = None
    w.requires_grad_(False)
    loss = losses.distill(plan, h, w, ids, logits, 2.0, reduction="sum")
    loss.backward()
    ref = head_reference(h.detach(), w, ids, soft_targets(ids, logits, 2.0), 2.0, False)
    close_grad(h.grad, ref["dH"], ref["h_err"], "dhidden")
    assert w.grad is None
    x = torch.randn(T, E, generator=g, device=DEV, requires_grad=True)
    chosen = torch.topk(x.detach(), 2, dim=1).indices
    loss, counts = losses.balance(router, x, chosen, None, 0.5)
    (2.0 * loss).backward()
    ref = balance_reference(x.detach(), chosen, None, 0.5)
    assert torch.equal(counts.long(), ref["counts"])
    assert (x.grad.double() - 2 * ref["dx"]).abs().max() <= 2.0**-16 * ref["scale_dx"].max() * 2


def test_workspace_grows_and_keeps_the_status_word():
    h, w, y, _ = operands(40, 500, 64, BF, 301)
    plan = losses.HeadLoss(8, 500, 64, BF)
    bad = y.clone()
    bad[0] = 500
    plan.cross_entropy(h[:8], w, bad[:8])
    r = plan.cross_entropy_grad(h, w, y)  # more tokens, and gradients
    ref = head_reference(h, w, y[:, None], torch.ones(40, 1, dtype=torch.float64, device=DEV), 1.0, True)
    check_head(r, ref)
    assert plan.status() == -1


def test_example_trains():
    from paper_1901_01544_b200 import train_head

    history, counts = train_head.train(steps=12, workers=3, tokens=256, vocab=1003, dim=128)
    first, last = history[0], history[-1]
    assert last[0] < 0.8 * first[0] and last[1] < 0.8 * first[1]
    assert sum(counts) == 3 * 256 * 2


def test_offsets_beyond_32_bits():
    """One piece of 20000 x 131072 codes: element offsets beyond 2^31.  Rows and columns at the far end are compared."""
    T, V, D = 20000, 131072, 64
    h, w, y, _ = operands(T, V, D, BF, 400)
    plan = losses.HeadLoss(T, V, D, BF, piece_bytes=6 << 30)
    r = plan.cross_entropy_grad(h, w, y, reduction="sum")
    assert plan.status() == 0
    far = slice(T - 40, T)
    one = torch.ones(40, 1, dtype=torch.float64, device=DEV)
    ref = head_reference(h[far], w, y[far, None], one, 1.0, False)
    close(r.rows[far], ref["rows"], ref["row_err"], "rows")
    close_grad(r.dhidden[far], ref["dH"], ref["h_err"], "dhidden")
    lse = torch.full((T,), -math.inf, dtype=torch.float64, device=DEV)
    for a in range(0, V, 16384):
        lse = torch.logaddexp(lse, torch.logsumexp(h.double() @ w[a : a + 16384].double().T, 1))
    cols = slice(V - 33, V)
    H, W = h.double(), w[cols].double()
    p = torch.exp(H @ W.T - lse[:, None])
    dz = p - (y[:, None] == torch.arange(V - 33, V, device=DEV)).double()
    dz_err = (D / 16 + 2) * 2.0**-22 * (H.abs().sum(1) * w.abs().max().double()) + 2.0**-20 * (1 + lse.abs())
    f_err = 2 * U[BF] * dz.abs() + (2 * dz_err[:, None] + U[BF]) * p + 2.0**-23
    w_err = f_err.T @ H.abs() + (T / 16 + 8) * 2.0**-22 * (dz.abs().T @ H.abs())
    close_grad(r.dweight[cols], dz.T @ H, w_err, "dweight")


def test_balance_offsets_beyond_32_bits():
    T, E, k = 1 << 23, 260, 2
    g = gen(401)
    x = torch.randn(4096, E, generator=g, device=DEV).to(BF).repeat(T // 4096, 1)
    ids = torch.randint(0, E, (T, k), generator=g, device=DEV, dtype=torch.int32)
    plan = losses.ExpertBalance(T, E)
    r = plan.grad(x, ids, coef=1.0, scale=float(T))
    counts = torch.bincount(ids.flatten().long(), minlength=E)
    assert torch.equal(r.counts.long(), counts)
    far = x[-4096:].double()
    p = torch.softmax(far, 1)
    f = counts.double() / (T * k)
    want = E * p * (f - (p * f).sum(1, keepdim=True))
    # p is off by 2^-19 * 40 relative at most (see check_balance), on both sides of the difference
    tol = U[BF] * 1.01 * want.abs() + 2 * 2.0**-19 * 40 * E * p * f.max() + TINY[BF]
    assert ((r.dlogits[-4096:].double() - want).abs() <= tol).all()
    # the same 4096 rows over and over: the mean of p is theirs, and 2^23 / (148 * 32) rows are added up per lane
    mean = p.mean(0)
    assert ((r.mean_prob.double() - mean).abs() <= (2.0**-19 * 40 + T * 2.0**-24 / 64) * mean).all()


def test_captured_in_a_graph():
    T, V, D, E = 200, 1500, 64, 16
    h, w, y, g = operands(T, V, D, BF, 500)
    x = torch.randn(T, E, generator=g, device=DEV)
    ids = torch.topk(x, 2, dim=1).indices
    plan, router = losses.HeadLoss(T, V, D, BF), losses.ExpertBalance(T, E)
    plan.cross_entropy_grad(h, w, y), router.grad(x, ids)  # workspaces and look-ups
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, b = plan.cross_entropy_grad(h, w, y), router.grad(x, ids)
    for seed in (501, 502):
        h2, w2, y2, g = operands(T, V, D, BF, seed)
        h.copy_(h2), w.copy_(w2), y.copy_(y2)
        x.copy_(torch.randn(T, E, generator=g, device=DEV))
        graph.replay()
        want, wb = plan.cross_entropy_grad(h, w, y), router.grad(x, ids)
        assert torch.equal(r.loss, want.loss) and torch.equal(r.dhidden, want.dhidden) and torch.equal(r.dweight, want.dweight)
        assert torch.equal(b.dlogits, wb.dlogits) and torch.equal(b.loss, wb.loss)


@pytest.mark.parametrize("T,V,D", [(130, 700, 72), (300, 6001, 200), (700, 70000, 136)])
def test_strided_gradients_touch_nothing_beside_them(T, V, D):
    """16-bit gradients in aligned strided rows leave by tile copies, which have to stop at the matrix's edges."""
    h, w, y, _ = operands(T, V, D, BF, 600)
    ref = head_reference(h, w, y[:, None], torch.ones(T, 1, dtype=torch.float64, device=DEV), 1.0, True)
    dh, dw = torch.full((T + 40, D + 24), 7.0, dtype=BF, device=DEV), torch.full((V + 40, D + 24), 7.0, dtype=BF, device=DEV)
    plan = losses.HeadLoss(T, V, D, BF)
    r = plan.cross_entropy_grad(h, w, y, dhidden=dh[:T, 8 : 8 + D], dweight=dw[:V, 8 : 8 + D])
    check_head(r, ref)
    for buf, n in ((dh, T), (dw, V)):
        assert (buf[n:] == 7).all() and (buf[:, :8] == 7).all() and (buf[:, 8 + D :] == 7).all()
