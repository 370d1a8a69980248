"""Plans of the losses in CUDA graphs and on several streams: their workspaces live as long as something may use them, and
their state (status word, counters) is prepared once."""
import pytest
import torch
from test_gpu_losses import BF, DEV, operands

from paper_1901_01544_b200 import losses

pytestmark = pytest.mark.gpu


def same(a, b, *names):
    for k in names:
        assert torch.equal(getattr(a, k), getattr(b, k)), k


def test_a_captured_forward_pass_outlives_a_larger_workspace():
    T, V, D = 300, 3000, 64
    h, w, y, _ = operands(T, V, D, BF, 900)
    plan = losses.HeadLoss(T, V, D, BF)
    want = plan.cross_entropy(h, w, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = plan.cross_entropy(h, w, y)
    small = plan._ws_bytes
    grad = plan.cross_entropy_grad(h, w, y)  # needs a larger workspace
    assert plan._ws_bytes > small
    others = [torch.full((small,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]  # whatever was freed is theirs now
    for _ in range(2):
        r.loss.zero_(), r.lse.zero_(), r.rows.zero_()
        graph.replay()
        same(r, want, "loss", "rows", "lse")
    assert all((x == 255).all() for x in others)
    same(plan.cross_entropy_grad(h, w, y), grad, "loss", "dhidden", "dweight")
    assert plan.status() == 0


def test_first_calls_inside_a_capture():
    T, V, D, E = 300, 3000, 64, 16
    h, w, y, g = operands(T, V, D, BF, 901)
    x = torch.randn(T, E, generator=g, device=DEV)
    ids = torch.topk(x, 2, dim=1).indices
    want, wb = losses.HeadLoss(T, V, D, BF).cross_entropy_grad(h, w, y), losses.ExpertBalance(T, E).grad(x, ids)
    torch.cuda.synchronize()
    plan, router = losses.HeadLoss(T, V, D, BF), losses.ExpertBalance(T, E)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, b = plan.cross_entropy_grad(h, w, y), router.grad(x, ids)
    same(plan.cross_entropy_grad(h, w, y), want, "loss", "rows", "dhidden", "dweight")  # before any replay
    same(router.grad(x, ids), wb, "loss", "counts", "dlogits")
    graph.replay()
    same(r, want, "loss", "rows", "dhidden", "dweight")
    same(b, wb, "loss", "counts", "dlogits")
    bad = y.clone()
    bad[0] = V
    plan.cross_entropy(h, w, bad)
    graph.replay()  # does not take the report back
    assert plan.status() == -1


def test_growing_inside_a_capture():
    T, V, D = 300, 3000, 64
    h, w, y, _ = operands(T, V, D, BF, 902)
    want = losses.HeadLoss(T, V, D, BF).cross_entropy_grad(h, w, y)
    plan = losses.HeadLoss(T, V, D, BF)
    forward = plan.cross_entropy(h, w, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = plan.cross_entropy_grad(h, w, y)
    same(plan.cross_entropy(h, w, y), forward, "loss", "rows", "lse")
    graph.replay()
    same(r, want, "loss", "rows", "dhidden", "dweight")


def test_plans_are_not_made_inside_a_capture():
    graph = torch.cuda.CUDAGraph()
    x = torch.zeros(4, device=DEV)
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(RuntimeError):
            losses.HeadLoss(8, 100, 16, BF)
        with pytest.raises(RuntimeError):
            losses.ExpertBalance(8, 4)
    graph.replay()
    assert (x == 1).all()


def test_a_workspace_is_not_handed_on_while_another_stream_uses_it():
    T, V, D = 300, 3000, 64
    h, w, y, _ = operands(T, V, D, BF, 903)
    plan = losses.HeadLoss(T, V, D, BF)
    want = losses.HeadLoss(T, V, D, BF).cross_entropy(h, w, y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan.cross_entropy(h, w, y)  # the workspace is made here,
    torch.cuda.synchronize()
    small = plan._ws_bytes
    torch.cuda._sleep(200_000_000)
    r = plan.cross_entropy(h, w, y)  # used here,
    plan.cross_entropy_grad(h, w, y)  # and outgrown, while the stream it came from goes on
    with torch.cuda.stream(side):
        others = [torch.full((small,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    same(r, want, "loss", "rows", "lse")
    assert all((x == 255).all() for x in others)


def test_a_new_plan_on_another_stream():
    """Its state is zeroed on the stream it was made on; a call elsewhere comes after that."""
    T, V, D = 300, 3000, 64
    h, w, y, _ = operands(T, V, D, BF, 904)
    want = losses.HeadLoss(T, V, D, BF).cross_entropy(h, w, y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(100_000_000)
    plan = losses.HeadLoss(T, V, D, BF)
    with torch.cuda.stream(side):
        r = plan.cross_entropy(h, w, y)
    torch.cuda.synchronize()
    same(r, want, "loss", "rows", "lse")
    assert plan.status() == 0
