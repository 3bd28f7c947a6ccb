"""Lists of tensors that change between two calls: what the calls read and write afterwards, on the device.  (What a list tells the library:
test_host_lists.py.)"""
import pytest
import torch

from oracle import grad_norm_oracle as gno
from paper_2201_05989_amd import AdamList, AdamTensor, GradStats, adam_step, adam_steps, clip_grads, grad_norm

pytestmark = pytest.mark.gpu


def item(n, value):
    return AdamTensor(torch.zeros(n, device="cuda"), torch.full((n,), value, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"))


def test_norm_and_step_are_those_of_a_tensor_put_into_the_list():
    old, new = item(64, 3.0), item(64, 1.0)
    model, stats = AdamList([old]), GradStats()
    grad_norm(model.grads, stats)
    assert float(stats.norm) == 24.0
    model.tensors[0] = new
    grad_norm(model.grads, stats)
    assert float(stats.norm) == 8.0
    adam_steps(model, stats)
    assert not old.params_master.any() and not old.m.any() and bool((old.grad == 3.0).all())
    assert bool((new.params_master < 0).all()) and bool((new.m > 0).all()) and not new.grad.any()


# A launch holds 240 gradients, 160 pairs of them or 48 tensors of the optimiser: lists that end there, one later, and with nothing but empty
# tensors behind; more workgroups in an earlier launch than in the last one; the longest list.
ENDS = [[100] * n + [0] * z for n in (47, 48, 49, 159, 160, 161, 239, 240, 241, 480, 481) for z in (0, 300)]
ENDS += [[40_000] * 240 + [1], [1] * 240 + [40_000] * 3, [0] * 500 + [70_001, 3] + [0] * 520, [0] * 1024, [2049] * 1024, list(range(1024))]


@pytest.mark.parametrize("sizes", ENDS, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_lists_that_end_where_a_launch_does(sizes):
    n = sum(sizes)
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    flat = torch.randn(n, device="cuda", generator=gen)
    cut = lambda t: list(torch.split(t, sizes))
    p, m, v = torch.randn(n, device="cuda", generator=gen), torch.rand(n, device="cuda", generator=gen), torch.rand(n, device="cuda", generator=gen)
    state = [flat.clone(), p.clone(), m.clone(), v.clone()]
    stats, out = GradStats(), torch.full((n,), 5.0, device="cuda")
    want = gno.norm([flat.cpu().numpy()])
    clip_grads(cut(flat), 0.25, stats, out=cut(out))
    assert abs(float(stats.norm) - want) <= 2.0 ** -24 * (1 + 2.0 ** -10) * want
    assert torch.equal(out, flat * stats.factor)
    bits = stats.memory[:16].clone()
    grad_norm(cut(flat), stats, 0.25)
    assert torch.equal(bits, stats.memory[:16])
    # the clipped gradients through the step on one tensor, which takes them as they are: the same bits
    adam_steps([AdamTensor(*a) for a in zip(cut(p), cut(flat), cut(m), cut(v))], stats)
    assert int(stats.steps) == 1 and not flat.any()
    if n:
        pad = lambda t: t.clone()  # (16-byte aligned)
        q, r, s = (pad(t) for t in state[1:])
        adam_step(q, state[0] * stats.factor, r, s, 1)
        for got, one in zip((p, m, v), (q, r, s)):
            assert torch.equal(got, one)
