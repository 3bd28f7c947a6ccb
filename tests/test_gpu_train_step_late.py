"""Training steps late in a run, where bias corrections are near 1 and differ from step to step, recorded and clipped ones: all arrays bit for
bit.

Before every step both models get the same tables and weights, small integers, under which nothing rounds on the way to the gradients (points
at vertices, dyadic slopes): sums are the same in any order, and what the optimiser gets is the same bits.  Moments and step counts go
on from step to step.
"""
import pytest
import torch

from paper_2201_05989_amd import HashGridModel

pytestmark = pytest.mark.gpu

STATE = ("tables", "tables_half", "_tab_m", "_tab_v", "weights", "weights_half", "_net_m", "_net_v")


def model(bound, n_out):
    return HashGridModel(3, n_out, L=8, F=2, T=1 << 14, N_min=4, N_max=512, seed=1, max_grad_norm=bound)


def renew(models, gen):
    first = models[0]
    tables = torch.randint(-1, 2, first.tables.shape, device="cuda", generator=gen).float()
    weights = torch.randint(-1, 2, first.weights.shape, device="cuda", generator=gen).float()
    weights *= torch.rand(weights.shape, device="cuda", generator=gen) < 0.2
    for m in models:
        m.tables.copy_(tables)
        m.tables_half.copy_(tables)
        m.weights.copy_(weights)
        m.weights_half.copy_(weights)


def batch(m, B, gen):
    x = (torch.randint(0, 4, (B, 3), device="cuda", generator=gen).float() / 4).contiguous()
    p = m.infer(x)
    return x, (p - torch.randint(-4, 5, p.shape, device="cuda", generator=gen) / 8.0).contiguous()


def same(a, b):
    for name in STATE:
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert not a._tab_zeros.any() and not b._tab_zeros.any()


@pytest.mark.parametrize("B", [300, 40000])
def test_replays_of_a_clipped_step_are_steps_made_one_by_one(B):
    gen = torch.Generator(device="cuda").manual_seed(B)
    a, b = model(1e-4, 2), model(1e-4, 2)
    renew((a, b), gen)
    x, target = batch(b, B, gen)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):  # the stream's own workspace
        a.step(x, target)
    torch.cuda.synchronize()
    b.step(x, target)
    same(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.step(x, target)
    for i, start in enumerate((1, 2, 3, 100, 5000)):
        a.grad_stats.steps.fill_(start)
        b.steps = start
        renew((a, b), gen)
        nx, nt = batch(b, B, gen)
        x.copy_(nx)
        target.copy_(nt)
        before = a.weights.clone()
        graph.replay()
        torch.cuda.synchronize()
        b.step(x, target)
        torch.randn(1000, device="cuda").sum().item()
        assert torch.equal(a.grad_stats.memory[:16], b.grad_stats.memory[:16]) and int(a.grad_stats.steps) == start + 1
        assert 0 < float(a.grad_stats.factor) < 1 and not torch.equal(a.weights, before)
        same(a, b)


@pytest.mark.parametrize("B", [300, 40000])
def test_a_bound_that_nothing_reaches_changes_nothing_at_later_steps(B):
    gen = torch.Generator(device="cuda").manual_seed(B + 1)
    a, b = model(None, 1), model(float("inf"), 1)
    for start in (0, 1, 1000, 1001, 123456):
        a.steps = b.steps = start
        renew((a, b), gen)
        x, target = batch(a, B, gen)
        a.step(x, target)
        b.step(x, target)
        same(a, b)
        assert int(b.grad_stats.steps) == start + 1
