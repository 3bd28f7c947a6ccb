"""What a recorded training step reads and writes stays its own: steps on batches of other sizes in between neither free nor share it."""
import pytest
import torch

from paper_2201_05989_amd import HashGridModel

pytestmark = pytest.mark.gpu

STATE = ("tables", "tables_half", "_tab_m", "_tab_v", "weights", "weights_half", "_net_m", "_net_v")
BOUNDS = [None, 1e-4]


def model(bound):
    return HashGridModel(3, 1, L=8, F=2, T=1 << 14, N_min=4, N_max=512, seed=1, max_grad_norm=bound)


def renew(models, gen):
    tables = torch.randint(-1, 2, models[0].tables.shape, device="cuda", generator=gen).float()
    weights = torch.randint(-1, 2, models[0].weights.shape, device="cuda", generator=gen).float()
    weights *= torch.rand(weights.shape, device="cuda", generator=gen) < 0.2
    for m in models:
        for array, values in ((m.tables, tables), (m.tables_half, tables), (m.weights, weights), (m.weights_half, weights)):
            array.copy_(values)


def batch(m, B, gen):  # nothing rounds on the way to the gradients (small integers, points at vertices): sums are the same in any order
    x = (torch.randint(0, 4, (B, 3), device="cuda", generator=gen).float() / 4).contiguous()
    return x, (m.infer(x) - torch.randint(-4, 5, (B, 1), device="cuda", generator=gen) / 8.0).contiguous()


def record(m, x, target):
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        m.step(x, target)  # (so that buffers and workspace are made outside the recording)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        m.step(x, target)
    return graph, stream


def spans(m):
    return [(t.data_ptr(), t.data_ptr() + t.nbytes) for t in [m._y, m._dy, *m.grid._ws.values()]]


@pytest.mark.parametrize("bound", BOUNDS)
@pytest.mark.parametrize("B,other", [(300, 777), (40000, 60000), (40000, 300)])
def test_nothing_else_gets_the_memory_of_a_recorded_step(B, other, bound):
    m, gen = model(bound), torch.Generator(device="cuda").manual_seed(1)
    graph, stream = record(m, *batch(m, B, gen))
    used = spans(m)
    with torch.cuda.stream(stream):
        m.step(*batch(m, other, gen))
    torch.cuda.synchronize()
    taken = []
    for s in (stream, torch.cuda.current_stream()):
        with torch.cuda.stream(s):
            taken += [torch.empty(end - begin, dtype=torch.uint8, device="cuda") for begin, end in used for _ in range(8)]
    mine = [(t.data_ptr(), t.data_ptr() + t.nbytes) for t in taken]
    assert not any(a < d and c < b for a, b in used for c, d in mine)


@pytest.mark.parametrize("bound", BOUNDS)
@pytest.mark.parametrize("B,other", [(300, 777), (40000, 60000), (40000, 300)])
def test_replays_after_steps_on_other_batches(B, other, bound):
    gen = torch.Generator(device="cuda").manual_seed(2)
    a, b = model(bound), model(bound)
    renew((a, b), gen)
    x, target = batch(b, B, gen)
    graph, stream = record(a, x, target)
    b.step(x, target)
    held = []
    for i in range(3):
        with torch.cuda.stream(stream):
            a.step(*batch(a, other, gen))
            held.append([torch.full((k,), 7.0, device="cuda") for k in (B * 8, B * 8, 1 << 22)])
        torch.cuda.synchronize()
        for name in STATE:
            getattr(b, name).copy_(getattr(a, name))
        renew((a, b), gen)
        nx, nt = batch(b, B, gen)
        x.copy_(nx), target.copy_(nt)
        if bound is not None:
            b.steps = int(a.grad_stats.steps)
        else:
            b.steps = 1  # the number that the recording holds is 2
        graph.replay()
        torch.cuda.synchronize()
        b.step(x, target)
        for name in STATE:
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        assert not a._tab_zeros.any()
        assert all(bool((t == 7.0).all()) for ts in held for t in ts)
