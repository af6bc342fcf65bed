"""fp64 oracle for the global gradient norm and clipping.

norm = scale * sqrt(sum of all squares);  out = scale * min(1, max_norm / norm) * g,
out = scale * g where the norm is not finite.
"""
from __future__ import annotations

import math

import numpy as np


def norm(grads, scale: float = 1.0) -> float:
    flat = [np.asarray(g, np.float64).ravel() for g in grads]
    if any(not np.all(np.isfinite(g)) for g in flat):
        return math.nan
    return scale * math.sqrt(math.fsum(float(x) * float(x) for g in flat for x in g))


def clip(grads, scale: float, max_norm: float):
    """(norm, clipped gradients)."""
    n = norm(grads, scale)
    c = scale * (max_norm / n if math.isfinite(n) and n > max_norm else 1.0)
    return n, [c * np.asarray(g, np.float64) for g in grads]
