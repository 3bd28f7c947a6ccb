"""The optimiser's step number of a HashGridModel whose max_grad_norm is set, taken off and set again: bias corrections go by the steps
that were taken, whoever counted them (the device with a bound, the host without), and neither by steps that were left out nor by
the recording of a captured one.

Each model is compared bit for bit with one that takes the same steps without ever changing the bound.  Batches are one point: then no
scalar of the tables has more than two summands but with three corners of one cell in the same entry, and sums of two are the
same in either order (the network's weights are summed in a fixed one).
"""
import pytest
import torch

from paper_2201_05989_amd import HashGridModel

pytestmark = pytest.mark.gpu
INF = float("inf")


def model(bound=None):
    # a bound of infinity leaves the gradients as they are: the same steps as without one
    return HashGridModel(3, 1, L=4, F=2, T=1 << 14, N_min=16, N_max=128, seed=2, max_grad_norm=bound)


def batch(i):
    gen = torch.Generator(device="cuda").manual_seed(100 + i)
    x = torch.rand((1, 3), device="cuda", generator=gen) * 0.9
    return x, torch.randn((1, 1), device="cuda", generator=gen)


def same(a, b):
    for name in ("tables", "tables_half", "_tab_m", "_tab_v", "weights", "weights_half", "_net_m", "_net_v"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert not a._tab_zeros.any()


def test_a_step_that_was_left_out_does_not_count_when_the_bound_is_taken_off_and_set_again():
    a, b = model(INF), model()
    x, t = batch(0)
    a.step(x, t), b.step(x, t)
    same(a, b)
    for _ in range(3):
        a.step(x, torch.full_like(t, float("nan")))
    same(a, b)
    assert int(a.grad_stats.steps) == 1 and a.steps == 4
    a.max_grad_norm = None
    for i in (1, 2):
        a.step(*batch(i)), b.step(*batch(i))
        same(a, b)
    a.max_grad_norm = INF
    assert int(a.grad_stats.steps) == 3
    a.step(*batch(3)), b.step(*batch(3))
    same(a, b)
    assert int(a.grad_stats.steps) == 4 and a.steps == 7 and b.steps == 4


def test_replays_count_when_the_bound_is_taken_off_and_set_again():
    a, b = model(INF), model()
    x, t = batch(0)
    a.step(x, t), b.step(x, t)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.step(x, t)
    for i in range(1, 7):
        nx, nt = batch(i)
        x.copy_(nx), t.copy_(nt)
        graph.replay()
        b.step(nx, nt)
        same(a, b)
    assert int(a.grad_stats.steps) == 7
    for bound, i in ((None, 7), (INF, 8), (None, 9), (INF, 10)):
        a.max_grad_norm = bound
        a.step(*batch(i)), b.step(*batch(i))
        same(a, b)
    assert int(a.grad_stats.steps) == 11


def test_a_count_that_the_caller_sets_is_kept():
    a, b = model(INF), model()
    a.grad_stats.steps.fill_(500)
    b.steps = 500
    for bound, i in ((INF, 0), (None, 1), (INF, 2)):
        a.max_grad_norm = bound
        a.step(*batch(i)), b.step(*batch(i))
        same(a, b)
    assert int(a.grad_stats.steps) == 503
    a.steps = b.steps = 40
    for bound, i in ((INF, 3), (None, 4)):
        a.max_grad_norm = bound
        a.step(*batch(i)), b.step(*batch(i))
        same(a, b)
    assert a.steps == b.steps == 42
    c = model()  # a bound set for the first time on a model that was resumed
    c.steps = 7
    c.max_grad_norm = INF
    assert int(c.grad_stats.steps) == 7
    c.max_grad_norm = 1.0  # one bound for another: nothing to count
    assert int(c.grad_stats.steps) == 7
