"""fp64 oracle of the products by element: loops over the atoms, from the definition.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import numpy as np


def forward(z, X, W, residual=None):
    """Y[i,c] = X[i,c] W[z_i] + residual[i,c]; X [n][components][k_in], W [elements][k_in][k_out]."""
    Y = np.zeros(X.shape[:2] + (W.shape[2],)) if residual is None else np.array(residual, np.float64)
    for i, e in enumerate(z):
        if 0 <= e < W.shape[0]:
            Y[i] += X[i] @ W[e]
    return Y


def backward(z, X, W, dY):
    """dX, dW."""
    dX, dW = np.zeros(X.shape), np.zeros(W.shape)
    for i, e in enumerate(z):
        if 0 <= e < W.shape[0]:
            dX[i] = dY[i] @ W[e].T
            dW[e] += X[i].T @ dY[i]
    return dX, dW
