"""CPU oracle of the gradient norm over many tensors and of clipping by it.  TEST INFRASTRUCTURE ONLY: the test-suite uses
it; the GPU library never does.

Arithmetic: the definitions written out in numpy, each tensor's squares in extended precision (64-bit significands, exponents far
beyond fp64's), so that neither the largest nor the smallest fp32 gradients lose anything.
"""
from __future__ import annotations

import numpy as np


def norm(grads, grad_scale: float = 1.0):
    """grad_scale * sqrt(sum of squares) over a list of float arrays; NaN or infinity where a scalar is."""
    total = np.longdouble(0)
    with np.errstate(invalid="ignore"):
        for g in grads:
            total += np.sum(np.asarray(g, dtype=np.longdouble) ** 2)
    return np.longdouble(grad_scale) * np.sqrt(total)


def factor(norm_value, max_norm: float):
    if not np.isfinite(norm_value):
        return np.longdouble(0)
    return np.longdouble(max_norm) / norm_value if norm_value > max_norm else np.longdouble(1)
