"""Refusals of the calls on lists of tensors, through the C ABI with made-up addresses: every call here is turned down before anything
would be launched, so no device is needed."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import grad_norm_oracle as gno
from paper_2201_05989_amd import AdamList, AdamTensor, GradList, HashGridError, binding

A = 1 << 20  # an address that nothing reads


def grads(*rows):
    return (binding.hashgrid_grad * len(rows))(*[(p, n, dtype, 0) for p, n, dtype in rows])


def adam(*rows, **kw):
    def one(i, row):
        d = dict(params_master=A + 0x100000 * i, params_half=None, grad=A + 0x100000 * i + 0x10000, m=A + 0x100000 * i + 0x20000,
                 v=A + 0x100000 * i + 0x30000, n_scalars=64, grad_dtype=0, half_dtype=1, cfg=binding.hashgrid_adam_config(1e-2, 0.9, 0.99, 1e-15, 0.0))
        d.update(row)
        return binding.hashgrid_adam_tensor(**d)
    return (binding.hashgrid_adam_tensor * len(rows))(*[one(i, r) for i, r in enumerate(rows)])


def test_the_oracle_s_norm_and_factor():
    three, four = np.array([[3.0]], dtype=np.float32), np.array([0.0, 4.0], dtype=np.float16)
    assert gno.norm([three, four]) == 5 and gno.norm([three, four], 0.5) == 2.5 and gno.norm([]) == 0
    assert gno.factor(gno.norm([three, four]), 1.0) == np.longdouble(1) / 5 and gno.factor(5.0, 5.0) == 1 and gno.factor(5.0, 0.0) == 0
    # squares beyond the range of 64 bits' neighbours, none lost: 1e-44 is a subnormal fp32
    huge, tiny = np.full(4, 3e38, dtype=np.float32), np.full(9, 1e-44, dtype=np.float32)
    assert abs(gno.norm([huge]) / (2 * np.longdouble(huge[0])) - 1) < 1e-18
    assert abs(gno.norm([tiny]) / (3 * np.longdouble(tiny[0])) - 1) < 1e-18
    for bad in (np.inf, -np.inf, np.nan):
        n = gno.norm([three, np.array([bad], dtype=np.float32)])
        assert not np.isfinite(n) and gno.factor(n, 1.0) == 0


def test_the_structures_are_the_header_s():
    assert ctypes.sizeof(binding.hashgrid_grad) == 24 and ctypes.sizeof(binding.hashgrid_adam_tensor) == 80
    assert binding.HG_GRAD_STATS_BYTES == 128 + 33 * 128 + 8 * 1024


def test_grad_norm_status_codes():
    norm = binding.load_library().hashgrid_grad_norm
    ok = grads((A, 64, 0))
    assert norm(1, ok, 1.0, 1.0, None, None) == 1            # no stats
    assert norm(1, ok, 1.0, 1.0, A + 8, None) == 1           # stats misaligned
    assert norm(1, None, 1.0, 1.0, A, None) == 1             # no list
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert norm(1, ok, scale, 1.0, A, None) == 1
    for bound in (-1.0, math.nan):
        assert norm(1, ok, 1.0, bound, A, None) == 1
    assert norm(1, grads((None, 64, 0)), 1.0, 1.0, A, None) == 1
    assert norm(1, grads((A + 2, 64, 0)), 1.0, 1.0, A, None) == 1   # fp32 on a 2-byte boundary
    assert norm(1, grads((A + 1, 64, 2)), 1.0, 1.0, A, None) == 1
    assert norm(1, grads((A, 64, 3)), 1.0, 1.0, A, None) == 1       # no such type
    assert norm(1025, grads(*[(A, 64, 0)] * 1025), 1.0, 1.0, A, None) == 2
    assert norm(1, grads((A, (1 << 42) + 1, 0)), 1.0, 1.0, A, None) == 2
    assert norm(4, grads(*[(A, 1 << 42, 0)] * 4), 1.0, 1.0, A, None) == 2


def test_clip_grads_status_codes():
    call = binding.load_library().hashgrid_clip_grads
    clip = lambda n, g, out, stats, scale=1.0, bound=1.0: call(n, g, out, scale, bound, stats, None)
    pointers = lambda *p: (ctypes.c_void_p * len(p))(*p)
    two = grads((A, 64, 0), (A + 256, 64, 0))
    assert clip(2, two, None, None) == 1
    assert clip(2, two, None, A + 4) == 1
    assert clip(2, two, pointers(None, A + 4096), A) == 1
    assert clip(2, two, pointers(A + 4096, A + 8190), A) == 1
    assert clip(2, grads((A, 64, 0), (A + 252, 64, 0)), None, A) == 1        # one scalar shared
    assert clip(2, grads((A, 64, 0), (A, 64, 0)), None, A) == 1
    assert clip(2, two, pointers(A + 4096, A + 4096 + 252), A) == 1
    assert clip(2, two, pointers(A + 256, A), A) == 1                        # each into the other
    assert clip(1, grads((A, 64, 1)), pointers(A + 2), A) == 1               # into itself, moved by one
    many = [(A + 0x1000 * i, 64, 2) for i in range(1023, -1, -1)]                  # in falling order, the last one twice
    assert clip(1024, grads(*many[:-1], many[0]), None, A) == 1
    assert clip(2, two, None, A, scale=0.0) == 1 and clip(2, two, None, A, bound=-1.0) == 1 and clip(2, two, None, A, bound=math.nan) == 1
    assert clip(1025, grads(*[(A, 64, 0)] * 1025), None, A) == 2


def test_adam_steps_status_codes():
    steps = binding.load_library().hashgrid_adam_steps
    assert steps(0, None, 1.0, 1, 1, None, None) == 0 and steps(1, adam(dict(n_scalars=0, m=None)), 1.0, 1, 1, None, None) == 0
    ok = adam({}, {})
    assert steps(2, None, 1.0, 1, 1, None, None) == 1
    assert steps(2, ok, 1.0, 1, 0, None, None) == 1     # no step number from anywhere
    assert steps(2, ok, 1.0, 1, 5, A, None) == 1        # two
    assert steps(2, ok, 1.0, 1, 0, A + 4, None) == 1
    assert steps(1025, ok, 1.0, 1, 1, None, None) == 2
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert steps(2, ok, scale, 1, 1, None, None) == 1
    for bad in (dict(params_master=None), dict(grad=None), dict(m=None), dict(v=None), dict(m=A + 0x500002), dict(grad=A + 0x500001, grad_dtype=2),
                dict(params_half=A + 0x500001), dict(grad_dtype=3), dict(params_half=A + 0x500000, half_dtype=0),
                dict(cfg=binding.hashgrid_adam_config(1e-2, 1.0, 0.99, 1e-15, 0.0)), dict(cfg=binding.hashgrid_adam_config(1e-2, 0.9, 0.99, 1e-15, -1.0)),
                dict(m=A + 0x100000), dict(v=A + 252), dict(grad=A + 0x100000 + 252), dict(params_half=A + 0x130000)):
        assert steps(2, adam({}, bad), 1.0, 1, 1, None, None) == 1, bad
    assert steps(1, adam(dict(n_scalars=(1 << 42) + 1)), 1.0, 1, 1, None, None) == 2


def test_the_binding_refuses_host_tensors():
    t = torch.zeros(4)
    with pytest.raises(HashGridError):
        GradList([t])
    with pytest.raises(HashGridError):
        AdamList([AdamTensor(t, t, t, t)])
    assert len(GradList([])) == 0 and len(AdamList([])) == 0
