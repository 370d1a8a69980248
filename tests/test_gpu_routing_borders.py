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


def spread(E, word, lanes, columns):
    """`columns` columns of one lane, where words of `word` neighbours go to the lanes in turn."""
    e = torch.arange(E, device=DEV)
    mine = e[e // word % lanes == lanes // 3]
    assert len(mine) >= columns
    return mine[:columns]


@pytest.mark.parametrize("word", [1, 2, 4, 8])
@pytest.mark.parametrize("lanes", [8, 16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("k", [7, 8, 9, 10, 13])
def test_the_best_of_a_row_side_by_side(k, dtype, lanes, word):
    """Up to 16 largest logits in what one lane may hold, which sorts only eight; equal ones among them, and rows with nothing else
    to choose.  (The words are the widest that the number of experts allows.)"""
    E = {1: 249, 2: 250, 4: 252, 8: 256}[word]
    for best in (7, 8, 9, 12):
        at = spread(E, word, lanes, min(best, E // (word * lanes) * word))
        g = torch.Generator(device=DEV).manual_seed(best)
        x = torch.randn(6, E, generator=g, device=DEV).to(dtype)
        x[:4, at] += 20
        x[1, at] = 16.0
        x[2, at[::2]] = 24.0
        x[3] = torch.where(torch.isin(torch.arange(E, device=DEV), at), x[3].double(), -math.inf).to(dtype)
        x[4] = 0.0
        for kw in (dict(), dict(score="sigmoid", renormalize=False)):
            plan = routing.ExpertRouter(E, k, **kw)
            check_route(plan, x, **kw)
            check_route(plan, x, 0.01 * torch.randn(E, generator=g, device=DEV), **kw)
            check_route(plan, x, torch.zeros(E, device=DEV), **kw)


def times(calls, reps=20):
    """Of replays of captured calls, in turn, the shortest of each in ms."""
    graphs = []
    for f in calls:
        f()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(8):
                f()
        graphs.append(g)
    best = [math.inf] * len(graphs)
    for _ in range(reps):
        for i, g in enumerate(graphs):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            g.replay()
            b.record()
            b.synchronize()
            best[i] = min(best[i], a.elapsed_time(b))
    return best


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_equal_logits_take_no_longer(dtype):
    """Rows of equal 16-bit logits (a router before its first step, padding) need no second look: their first eight experts are what one
    lane has.  (With one, each row by a whole warp, it was five to six times as long.)"""
    T, E, k = 65536, 256, 8
    plan = routing.ExpertRouter(E, k)
    equal, random = torch.zeros(T, E, device=DEV, dtype=dtype), torch.randn(T, E, device=DEV).to(dtype)
    ids = plan.route(equal).ids
    assert torch.equal(ids, torch.arange(k, device=DEV, dtype=torch.int32).expand(T, k))
    slow, usual = times([lambda: plan.route(equal), lambda: plan.route(random)])
    assert slow < 2 * usual, (slow, usual)
