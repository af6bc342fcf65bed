"""fp64 oracle for the uncompressed embedding table with a scale.

forward   Y[t, :] = scale * T[ids[t], :], zeros for an id outside [0, V)
backward  dT[v, :] = scale * sum of dY[t, :] over the tokens with ids[t] = v,
          v != pad, token by token
"""
from __future__ import annotations

import numpy as np


def forward(ids, T, scale: float) -> np.ndarray:
    ids, T = np.asarray(ids, np.int64), np.asarray(T, np.float64)
    Y = np.zeros((ids.size, T.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < T.shape[0]:
            Y[t] = scale * T[v]
    return Y


def backward(ids, dY, V: int, scale: float, pad: int = -1) -> np.ndarray:
    dT = np.zeros((V, np.shape(dY)[1]))
    for v, row in zip(np.asarray(ids, np.int64), np.asarray(dY, np.float64)):
        if 0 <= v < V and v != pad:
            dT[v] += scale * row
    return dT
