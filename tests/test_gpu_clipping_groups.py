"""Norms and clipping of groups about where their sums are added up by a launch of its own."""
import pytest
import torch

from paper_1901_01544_b200 import clipping

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("n", [600_000, 3_900_000, 3_960_000, 8_000_001])
@pytest.mark.parametrize("groups", [1, 2, 3, 8, 9])
def test_groups(groups, n):
    """Squares are added up by eights in fp32 (8 roundings of 2^-24 of a sum of squares, half of that in its root), the norm is
    rounded once; elements times the factor as fp32 has it, rounded once."""
    g = torch.Generator(device=DEV).manual_seed(n + groups)
    xs = [torch.randn(n // groups + 3 * i, generator=g, device=DEV) * (1 + i) for i in range(groups)]
    was = [x.clone() for x in xs]
    clip = clipping.GradientClip(xs, groups=list(range(groups)))
    want = torch.stack([x.double().norm() for x in xs])
    for r in (clip.norm(), clip.norm()):
        assert ((r.norms.double() - want).abs() <= 6 * 2.0**-24 * want).all()
        assert (r.factors == 1).all()
    r = clip.clip(0.5 * float(want.min()))
    assert ((r.norms.double() - want).abs() <= 6 * 2.0**-24 * want).all() and (r.factors < 1).all()
    assert all(torch.equal(x, w * f) for x, w, f in zip(xs, was, r.factors))
    for x, w in zip(xs, was):
        x.copy_(w)
    again = clip.clip(0.5 * float(want.min()))
    assert torch.equal(again.squares, r.squares) and torch.equal(again.factors, r.factors)
    # the same sums, given
    for x, w in zip(xs, was):
        x.copy_(w)
    given = clip.clip(0.5 * float(want.min()), squares=r.squares.clone())
    assert torch.equal(given.factors, r.factors) and all(torch.equal(x, w * f) for x, w, f in zip(xs, was, r.factors))


@pytest.mark.parametrize("groups,n", [(2, 9_000_000), (128, 5_000_000), (129, 5_000_000), (3, 5_000_000)])
def test_groups_of_very_different_sizes(groups, n):
    """One group has nearly all elements, one has none."""
    g = torch.Generator(device=DEV).manual_seed(groups)
    sizes = [n] + [(17 * i) % 300 for i in range(1, groups)]
    sizes[-1] = 0
    xs = [torch.randn(m, generator=g, device=DEV, dtype=torch.float32) for m in sizes]
    clip = clipping.GradientClip(xs, groups=list(range(groups)))
    assert clip.groups == groups
    want = torch.stack([x.double().norm() for x in xs])
    r = clip.norm()
    assert ((r.norms.double() - want).abs() <= 6 * 2.0**-24 * want).all() and r.norms[-1] == 0
    given = clip.clip(float("inf"), squares=r.squares.clone())
    assert torch.equal(given.norms, r.norms)
    xs[0][n // 2] = float("nan")
    r = clip.clip(1.0, drop_nonfinite=True)
    assert r.factors[0] == 0 and torch.isnan(r.norms[0]) and (xs[0] == 0).all() and ((r.norms[1:].double() - want[1:]).abs() <= 6 * 2.0**-24 * want[1:]).all()
