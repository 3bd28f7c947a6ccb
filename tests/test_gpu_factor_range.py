"""How far clipping holds the bound where the norm is far beyond it: the clipped gradients' own norm, in extended precision, against the bound.

The factor is an fp32, off by 2^-24 relative from max_norm / norm where that is at least 2^-126 (a norm of up to 2^126 times the
bound), and by half a subnormal step, 2^-150, below.  Each product is rounded once more, 2^-24 relative (the clipped scalars here are far above the
smallest numbers).  So the clipped norm is off by (2^-23 + 2^-48) bound + 2^-150 norm at the most, the last term only below 2^-126.
"""
import numpy as np
import pytest
import torch

from oracle import grad_norm_oracle as gno
from paper_2201_05989_amd import AdamTensor, GradStats, adam_steps, clip_grads, grad_norm

pytestmark = pytest.mark.gpu
N = 10_000


def gradients(size):
    gen = torch.Generator(device="cuda").manual_seed(1)
    return (torch.rand(N, device="cuda", generator=gen) + 0.5) * size


def ldnorm(t):
    return gno.norm([t.cpu().numpy()])


@pytest.mark.parametrize("size", [1e-30, 1.0, 1e20, 7e35])  # the last one: a factor just above 2^-126
@pytest.mark.parametrize("bound", [1.0, 0.3])
def test_the_clipped_norm_is_the_bound(size, bound):
    if size < 1:
        bound *= 1e-30
    g, stats, out = gradients(size), GradStats(), torch.empty(N, device="cuda")
    limit, norm = np.longdouble(np.float32(bound)), ldnorm(g)
    clip_grads([g], bound, stats, out=[out])
    exact = limit / norm
    assert exact < 1
    if exact >= 2.0 ** -126:
        assert abs(np.longdouble(float(stats.factor)) / exact - 1) <= 2.0 ** -24
        assert abs(ldnorm(out) / limit - 1) <= 2.0 ** -23 + 2.0 ** -48
    else:
        assert abs(ldnorm(out) - limit) <= limit * (2.0 ** -23 + 2.0 ** -48) + 2.0 ** -150 * norm


@pytest.mark.parametrize("size,bound", [(3e38 / 1.5, 1.0), (3e38 / 1.5, 0.01), (1e38, 1e-4), (7e35, 1e-3)])
def test_below_the_normal_numbers_the_factor_is_the_nearest_there_is(size, bound):
    g, stats, out = gradients(size), GradStats(), torch.empty(N, device="cuda")
    limit, norm = np.longdouble(np.float32(bound)), ldnorm(g)
    clip_grads([g], bound, stats, out=[out])
    assert limit / norm < 2.0 ** -126 and abs(np.longdouble(float(stats.factor)) - limit / norm) <= 2.0 ** -150
    assert abs(ldnorm(out) - limit) <= limit * (2.0 ** -23 + 2.0 ** -48) + 2.0 ** -150 * norm


def test_a_factor_below_the_smallest_number_is_a_step_of_zeros_that_counts():
    g, stats = gradients(1e38), GradStats()
    p, m, v = torch.ones(N, device="cuda"), torch.rand(N, device="cuda"), torch.rand(N, device="cuda")
    before = [a.clone() for a in (p, m, v)]
    grad_norm([g], stats, 1e-6)  # 1e-6 / 1e40
    assert float(stats.factor) == 0.0 and int(stats.step) == 1
    adam_steps([AdamTensor(p, g, m, v)], stats)
    assert int(stats.steps) == 1 and all(torch.equal(a, b) for a, b in zip((p, m, v), before)) and not g.any()
