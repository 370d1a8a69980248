"""Norms and clipping of gradient tensors against their formulas in 64 bits.

h(t) = finfo(t).eps / 2 is the relative error of one rounding to t, U = h(float32).  Squares are added up eight at a time in
fp32: at most 8 U of a sum of positive terms, so 4 U of its root, and one rounding of the norm.  A factor has that and its own
rounding, a result one product and the rounding to its type besides."""
import math

import pytest
import torch

from paper_1901_01544_b200 import clipping, losses
from paper_1901_01544_b200.binding import Pruner

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


def normal(g, *shape, dtype=F32, size=1.0):
    return (size * torch.randn(shape, generator=g, device=DEV)).to(dtype)


def plain(tensors, groups, max_norm=math.inf, scale=1.0):
    squares = [0.0] * (1 + max(groups))
    for x, g in zip(tensors, groups):
        squares[g] += x.double().square().sum().item()
    norms = torch.tensor(squares, dtype=torch.float64, device=DEV).sqrt() * abs(scale)
    return norms, scale * torch.clamp(max_norm / norms, max=1.0)


def check(r, outs, before, groups, max_norm, scale):
    norms, factors = plain(before, groups, max_norm, scale)
    assert ((r.norms.double() - norms).abs() <= 5 * U * norms).all()
    assert ((r.factors.double() - factors).abs() <= 6 * U * factors.abs()).all()
    for x, y, g in zip(before, outs, groups):
        want = x.double() * factors[g]
        tiny = torch.finfo(y.dtype).smallest_normal * torch.finfo(y.dtype).eps
        assert ((y.double() - want).abs() <= (7 * U + half(y.dtype)) * want.abs() + tiny).all()


SETS = [[1], [7], [64, 1000, 16 * 256], [5, 0, 3, 100_003], [70_001, 31, 1, 2048 * 99 + 1, 255], [3_000_017], [1 << 18], [(1 << 18) + 1], [513] * 300]


@pytest.mark.parametrize("sizes", SETS)
@pytest.mark.parametrize("source", [F32, BF, FP])
def test_clip(sizes, source):
    g = gen(len(sizes))
    for target in (F32, BF, FP):
        for first in (0, 1, 3):  # elements before a multiple of 16 bytes
            xs = [normal(g, n + first, dtype=source)[first:] for n in sizes]
            before = [x.clone() for x in xs]
            groups = [i % 3 for i in range(len(sizes))] if len(sizes) > 3 else [0] * len(sizes)
            flat = torch.full((sum(sizes) + 9,), 5.0, dtype=target, device=DEV)
            into = list(torch.split(flat[2 : sum(sizes) + 2], sizes))
            plan = clipping.GradientClip(xs, into=into, groups=groups)
            check(plan.norm(scale=-3.0), [], before, groups, math.inf, -3.0)
            for limit, scale in ((0.5, 1.0), (1e30, 0.25), (0.5, 1.0 / 1024)):
                check(plan.clip(limit, scale=scale), into, before, groups, limit, scale)
            assert (flat[:2] == 5).all() and (flat[sum(sizes) + 2 :] == 5).all()
            assert all(torch.equal(a, b) for a, b in zip(xs, before))
    plan = clipping.GradientClip(xs, groups=groups)
    check(plan.clip(0.75), xs, before, groups, 0.75, 1.0)
    after = [x.clone() for x in xs]
    plan.clip(math.inf)
    assert all(torch.equal(a, b) for a, b in zip(xs, after))


def test_types_in_one_list():
    g = gen(1)
    xs = [normal(g, 1001, dtype=F32), normal(g, 77, 33, dtype=BF), normal(g, 4, 5, 6, dtype=FP), normal(g, dtype=F32), normal(g, 300_000, dtype=BF)]
    before = [x.clone() for x in xs]
    check(clipping.GradientClip(xs).clip(1.0), xs, before, [0] * 5, 1.0, 1.0)


def test_one_norm_per_tensor():
    g = gen(2)
    for n in (40, 5000):
        xs = [normal(g, 1 + 97 * i % 513, size=10.0 ** (i % 9 - 4)) for i in range(n)]
        r = clipping.GradientClip(xs, groups=range(n)).norm()
        want, _ = plain(xs, list(range(n)))
        assert ((r.norms.double() - want).abs() <= 5 * U * want).all()
        assert ((r.squares - want.square()).abs() <= 8 * U * want.square()).all()


@pytest.mark.parametrize("size", [1e-44, 1e-30, 1e-19, 1e18, 1e25, 3e38])
@pytest.mark.parametrize("n", [5, 1000, 400_000])
def test_squares_outside_fp32(n, size):
    x = (size * (1 - 2 * torch.rand(n, generator=gen(3), device=DEV, dtype=torch.float64))).float()
    y = torch.empty_like(x)
    plan = clipping.GradientClip([x], into=[y])
    norm = x.double().square().sum().sqrt()
    limit = 0.5 * norm.item()
    r = plan.clip(limit)
    assert ((r.squares - norm.square()).abs() <= 8 * U * norm.square()).all()
    assert (r.factors.double() - 0.5).abs().max() <= 6 * U
    assert ((y.double() - 0.5 * x.double()).abs() <= 8 * U * x.double().abs() + 2.0**-149).all()
    if norm > torch.finfo(F32).max:
        assert torch.isinf(r.norms).all()


@pytest.mark.parametrize("n", [100, 700_000])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_gradients_that_are_not_finite(n, what):
    for dtype in (F32, BF, FP):
        a, b = normal(gen(4), n, dtype=dtype), normal(gen(5), n, dtype=dtype)
        a[n // 2] = what
        keep = [a.clone(), b.clone()]
        out = [torch.empty(n, device=DEV) for _ in range(2)]
        plan = clipping.GradientClip([a, b], into=out, groups=[0, 1])
        r = plan.clip(1.0, scale=0.5)
        assert not torch.isfinite(r.norms[0]) and r.factors[0] == 0.5
        assert torch.equal(out[0].nan_to_num(nan=1.0), (0.5 * keep[0].float()).nan_to_num(nan=1.0))
        check_b = plain([keep[1]], [0], 1.0, 0.5)[1]
        assert (r.factors[1].double() - check_b[0]).abs() <= 6 * U * check_b[0]
        r = plan.clip(1.0, drop_nonfinite=True)
        assert r.factors[0] == 0 and (out[0] == 0).all() and (out[1] != 0).any()
        inplace = clipping.GradientClip([a, b], groups=[0, 1])
        inplace.clip(1e30, drop_nonfinite=True)
        assert (a == 0).all() and torch.equal(b, keep[1])


def test_limit_of_zero_and_gradients_of_zero():
    for n in (10, 500_000):
        x, z = normal(gen(6), n), torch.zeros(n, device=DEV)
        plan = clipping.GradientClip([x, z], groups=[0, 1])
        r = plan.clip(0.0)
        assert (x == 0).all() and r.factors.tolist() == [0.0, 1.0] and r.norms[1] == 0
    e = clipping.GradientClip([torch.empty(0, device=DEV), torch.ones(3, device=DEV)], groups=[0, 2])
    assert e.clip(1.0).norms.tolist()[:2] == [0.0, 0.0] and e.groups == 3
    assert clipping.GradientClip([]).clip(1.0).norms.tolist() == [0.0]


def test_strided_gradients():
    g = gen(7)
    wide = normal(g, 300, 1000)
    cube = normal(g, 6, 40, 50, dtype=BF)
    xs = [wide[:, 3:500], wide[:, 500:503], normal(g, 200, 90).t(), cube[1:5, 2:30, 4:44], normal(g, 30, 1, 20).expand(30, 1, 20), wide[::2, 900:]]
    before = [x.clone() for x in xs]
    rest = wide.clone()
    plan = clipping.GradientClip(xs)
    check(plan.clip(1.0), xs, before, [0] * len(xs), 1.0, 1.0)
    for a, b in ((0, 3), (503, 900)):
        assert torch.equal(wide[:, a:b], rest[:, a:b])
    assert torch.equal(wide[1::2, 900:], rest[1::2, 900:])
    # from one layout into another
    x = normal(g, 50, 60)
    into = torch.zeros(50, 100, device=DEV)
    check(clipping.GradientClip([x], into=[into[:, 7:67]]).clip(1.0), [into[:, 7:67]], [x.clone()], [0], 1.0, 1.0)
    assert (into[:, :7] == 0).all() and (into[:, 67:] == 0).all()
    # a broadcast gradient has a norm, but nowhere to be written
    y = torch.ones(1, 8, device=DEV).expand(100, 8)
    plan = clipping.GradientClip([y])
    assert plan.norm().norms.item() == pytest.approx(math.sqrt(800), rel=1e-6)
    with pytest.raises(ValueError):
        plan.clip(1.0)


def test_sums_given_from_elsewhere():
    g = gen(8)
    for n in (1000, 600_000):
        parts = [[normal(g, n), normal(g, 7)] for _ in range(3)]
        plans = [clipping.GradientClip(p) for p in parts]
        total = sum(p.norm().squares for p in plans)
        before = [x.clone() for p in parts for x in p]
        limit = 0.3 * math.sqrt(total.item())
        _, factor = plain(before, [0] * 6, limit)
        for p, q in zip(plans, parts):
            old = [x.clone() for x in q]
            r = p.clip(limit, squares=total)
            assert (r.factors.double() - factor).abs() <= 6 * U * factor
            assert all(((a.double() - b.double() * factor).abs() <= 8 * U * b.double().abs()).all() for a, b in zip(q, old))


def test_beyond_32_bits():
    n = (1 << 31) + 77
    x = torch.zeros(n, dtype=BF, device=DEV)
    x[-1], x[0], x[1 << 31] = 3.0, 4.0, 12.0
    r = clipping.GradientClip([x]).clip(6.5)
    assert r.norms.item() == 13.0 and x[-1] == 1.5 and x[0] == 2.0 and x[1 << 31] == 6.0


def test_equal_bits_again_and_on_other_streams():
    xs = [normal(gen(9), n) for n in (100_000, 7, 2_000_001)]
    out = [torch.empty_like(x) for x in xs]
    plan = clipping.GradientClip(xs, into=out)
    first = plan.clip(1.0)
    keep = [o.clone() for o in out]
    for _ in range(3):
        for o in out:
            o.zero_()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            r = plan.clip(1.0)
        s.synchronize()
        assert torch.equal(r.squares, first.squares) and all(torch.equal(a, b) for a, b in zip(out, keep))


@pytest.mark.parametrize("n", [1000, 900_000])
def test_captured_and_replayed(n):
    x, y = normal(gen(10), n, dtype=FP), torch.empty(n, device=DEV)
    plan = clipping.GradientClip([x], into=[y])
    plan.clip(2.0, scale=0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = plan.clip(2.0, scale=0.5)
    for seed in (11, 12):
        x.copy_(normal(gen(seed), n, dtype=FP))
        y.zero_()
        graph.replay()
        check(r, [y], [x.clone()], [0], 2.0, 0.5)
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            clipping.GradientClip([x])


def test_clipped_into_the_pruned_step():
    """Each worker's gradients, bf16 tensors of its model, clipped by its own norm into its row; the step then reduces what a
    step over rows scaled by the same factors reduces, bit for bit."""
    W, sizes = 3, [40_000, 513, 64]
    g = gen(13)
    xs = [normal(g, n, dtype=BF, size=w + 1.0) for w in range(W) for n in sizes]
    grads = torch.empty(W, sum(sizes), device=DEV)
    into = [v for w in range(W) for v in torch.split(grads[w], sizes)]
    groups = [w for w in range(W) for _ in sizes]
    r = clipping.GradientClip(xs, into=into, groups=groups).clip(50.0)
    check(r, into, xs, groups, 50.0, 1.0)
    rows = torch.stack([torch.cat([x.float() * r.factors[w] for x in xs[w * 3 : w * 3 + 3]]) for w in range(W)])
    assert torch.equal(rows, grads)
    weights = normal(g, sum(sizes))
    a, b = Pruner(sizes, W, 16.0, 1e-8, 0), Pruner(sizes, W, 16.0, 1e-8, 0)
    assert torch.equal(a.step(grads, weights), b.step(rows, weights))
    a.check(), b.check()
    a.close(), b.close()


def test_refusals():
    x = torch.ones(10, device=DEV)
    for call in (lambda: clipping.GradientClip([x.double()]), lambda: clipping.GradientClip([x], into=[x.long()])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: clipping.GradientClip([x.cpu()]), lambda: clipping.GradientClip([x], into=[x[:9]]), lambda: clipping.GradientClip([x], into=[]),
                 lambda: clipping.GradientClip([x], groups=[-1]), lambda: clipping.GradientClip([x], groups=[0, 1]),
                 lambda: clipping.GradientClip([x[::2]]), lambda: clipping.GradientClip([x[:5]], into=[x[2:7]]),
                 lambda: clipping.GradientClip([x, x], into=[torch.empty(10, device=DEV), x]), lambda: clipping.GradientClip([x[:4], x[4:8]], into=[x[4:8], x[:4]]),
                 lambda: clipping.GradientClip([x.view(2, 5)], into=[torch.empty(5, device=DEV).expand(2, 5)]), lambda: clipping.GradientClip([x, x]).clip(1.0)):
        with pytest.raises(ValueError):
            call()
    plan = clipping.GradientClip([x])
    for call in (lambda: plan.clip(-1.0), lambda: plan.clip(math.nan), lambda: plan.clip(1.0, scale=0.0), lambda: plan.norm(scale=math.inf),
                 lambda: clipping.GradientClip([x], groups=[1 << 20])):
        with pytest.raises(losses.IwpError):
            call()
    with pytest.raises(TypeError):
        plan.clip(1.0, squares=torch.ones(1, device=DEV))
    with pytest.raises(ValueError):
        plan.clip(1.0, squares=torch.ones(2, device=DEV, dtype=torch.float64))
    assert (x == 1).all()
    assert clipping.GradientClip([x, x]).norm().norms.item() == pytest.approx(math.sqrt(20), rel=1e-6)


@pytest.mark.parametrize("into", [F32, BF, FP])
@pytest.mark.parametrize("dtype", [F32, BF, FP])
def test_every_alignment_of_short_and_long_runs(dtype, into):
    """Sources and outputs that start anywhere in a word, of all lengths around one; what lies around the outputs stays."""
    g = torch.Generator(device=DEV).manual_seed(5)
    sizes = [*range(1, 40), 255, 1000, 4099]
    pairs = [(a, b) for a in range(8) for b in range(8)]
    xs, ys, outs = [], [], []
    for i, (a, b) in enumerate(pairs):
        n = sizes[i % len(sizes)] + (i // len(sizes))
        xs.append(torch.randn(a + n + 8, generator=g, device=DEV).to(dtype)[a:a + n])
        outs.append(torch.full((b + n + 8,), 7.0, device=DEV, dtype=into))
        ys.append(outs[-1][b:b + n])
    for a in range(8):  # long ones, by warps that start anywhere
        n = 300007 + a
        xs.append(torch.randn(n + 8, generator=g, device=DEV).to(dtype)[a:a + n])
        outs.append(torch.full((n + 16,), 7.0, device=DEV, dtype=into))
        ys.append(outs[-1][3:3 + n])
        pairs.append((a, 3))
    clipping.GradientClip(xs, ys).clip(math.inf, scale=0.5)
    for x, y, out, (_, b) in zip(xs, ys, outs, pairs):
        assert torch.equal(y, (x.float() * 0.5).to(into))
        assert (out[:b] == 7).all() and (out[b + x.numel():] == 7).all()
