"""fp64 oracle of the element embedding: a scaled row of a table per atom, and the gradient of the table.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import numpy as np


def forward(z, T, scale: float) -> np.ndarray:
    T = np.asarray(T, np.float64)
    Y = np.zeros((len(z), T.shape[1]))
    for i, e in enumerate(z):
        if 0 <= e < T.shape[0]:
            Y[i] = scale * T[e]
    return Y


def backward(z, dY, num_elements: int, scale: float) -> np.ndarray:
    dY = np.asarray(dY, np.float64)
    dT = np.zeros((num_elements, dY.shape[1]))
    for i, e in enumerate(z):
        if 0 <= e < num_elements:
            dT[e] += dY[i]
    return scale * dT
