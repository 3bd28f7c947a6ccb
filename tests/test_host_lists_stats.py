"""Refusal of arrays that lie in the statistics' own memory, which the calls on lists write: through the C ABI with made-up addresses; every
call here is turned down, so no device is needed."""
import ctypes

import pytest

from paper_2201_05989_amd import binding

A = 1 << 20  # an address that nothing reads
S = 1 << 24  # the statistics
INSIDE = [S - 4 * 63, S, S + 64, S + 128 + 40, S + binding.HG_GRAD_STATS_BYTES - 4]  # of 64 fp32 scalars: one of them shared at the least


def grads(*addresses):
    return (binding.hashgrid_grad * len(addresses))(*[(a, 64, 0, 0) for a in addresses])


@pytest.mark.parametrize("at", INSIDE)
def test_norm_and_clipping(at):
    lib = binding.load_library()
    assert lib.hashgrid_grad_norm(2, grads(A, at), 1.0, 1.0, S, None) == 1
    assert lib.hashgrid_clip_grads(2, grads(at, A), None, 1.0, 1.0, S, None) == 1
    out = (ctypes.c_void_p * 2)(A + 4096, at)
    assert lib.hashgrid_clip_grads(2, grads(A, A + 1024), out, 1.0, 1.0, S, None) == 1


@pytest.mark.parametrize("at", INSIDE)
@pytest.mark.parametrize("name", ["params_master", "params_half", "grad", "m", "v"])
def test_the_optimiser_step(name, at):
    row = dict(params_master=A, params_half=A + 0x1000, grad=A + 0x2000, m=A + 0x3000, v=A + 0x4000)
    if name == "params_half" and at < S:
        at = S - 2
    row[name] = at
    tensor = binding.hashgrid_adam_tensor(**row, n_scalars=64, grad_dtype=0, half_dtype=1, cfg=binding.hashgrid_adam_config(1e-2, 0.9, 0.99, 1e-15, 0.0))
    for zero_grad in (0, 1):
        assert binding.load_library().hashgrid_adam_steps(1, ctypes.byref(tensor), 1.0, zero_grad, 0, S, None) == 1
