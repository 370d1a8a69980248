"""Choices by softmax scores with a bias whose order hangs on the last places of a row's sum of exponentials."""
import math

import pytest
import torch

from paper_1901_01544_b200 import routing
from test_gpu_routing import check_route, plain

pytestmark = pytest.mark.gpu
DEV = "cuda"

# 31 exponentials at -24 below TOP's are 2^-30 (1 + 4.7e-7) of it, but 2^-30 (1 - 4.7e-7) where the difference is rounded to fp32 first
# (which no error of two units in the last place of fp32's exponential makes up for: 2.4e-7).  TOP's score is then 1 - 2^-30 less or more
# of the same, and with 2^23 added, where 64 bits step by 2^-29, it is below 2^23 + 1 or equal to it.
TOP, REST, MANY = float.fromhex("0x1.d3c482p-3"), -24.0, 31


@pytest.mark.parametrize("first,second", [(0, 1), (1, 0), (3, 30), (32, 4)])
def test_scores_equal_but_for_the_rounding_of_the_sum(first, second):
    x = torch.full((5, MANY + 2), REST, device=DEV)
    bias = torch.full((MANY + 2,), -1.0, device=DEV)
    x[:, first], bias[first] = TOP, 2.0**23
    x[:, second], bias[second] = -200.0, 2.0**23 + 1
    assert (plain(x, 1, bias=bias)[0] == second).all()
    check_route(routing.ExpertRouter(MANY + 2, 1), x, bias)
    check_route(routing.ExpertRouter(MANY + 2, 3), x, bias)


@pytest.mark.parametrize("first,second", [(0, 1), (1, 0), (2, 3), (3, 1)])
def test_groups_equal_but_for_the_rounding_of_the_sum(first, second):
    size = 9
    x = torch.full((5, 4, size), REST, device=DEV)
    bias = -1.0 - torch.arange(4.0 * size, device=DEV).view(4, size)  # (no two of a group are near each other)
    x[:, 0, 6:] = -math.inf
    x[:, first, 1], bias[first, 1] = TOP, 2.0**23
    x[:, second, 2], bias[second, 2] = -200.0, 2.0**23 + 1
    assert int((x == REST).sum()) == 5 * MANY
    kw = dict(groups=4, top_groups=1, group_top=1)
    x, bias = x.flatten(1), bias.flatten()
    assert (plain(x, 1, bias=bias, **kw)[0] == second * size + 2).all()
    check_route(routing.ExpertRouter(4 * size, 1, **kw), x, bias, **kw)


@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("far", [4.0, 4.3, 5.4, 6.1, 7.9, 8.1])
def test_many_equal_logits_below_the_top(far, groups):
    """1023 equal terms, whose rounding adds up to the most that the sum of a row can be off by, and biases that all but make up for
    the scores of a few."""
    E, k = 1024, 4
    g = torch.Generator(device=DEV).manual_seed(int(10 * far))
    for _ in range(8):
        x = torch.full((3, E), 0.1 + float(torch.rand((), generator=g, device=DEV)), device=DEV)
        at = int(torch.randint(0, E, (), generator=g, device=DEV))
        x[:, at] += far + float(torch.rand((), generator=g, device=DEV)) / 16
        s = torch.softmax(x[0].double(), 0)
        few = torch.randperm(E, generator=g, device=DEV)[:6]
        bias = torch.full((E,), -0.5, device=DEV)
        bias[few] = (s[at] - s[few]).float()
        bias[at] = 0.0
        kw = dict(groups=groups, top_groups=max(1, groups // 2))
        check_route(routing.ExpertRouter(E, k, **kw), x, bias, **kw)
