"""fp64 oracle of the dense layer: Z = X W + b, Y = act(Z) + residual, its gradients and second-order pass.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

The derivatives of the activations are written out here from their closed forms and pinned by finite differences in
tests/test_oracle_dense_layer.py.  GELU is the form with the hyperbolic tangent.
"""
from __future__ import annotations

import numpy as np

ACTIVATIONS = ("none", "relu", "silu", "gelu")
_A, _C = np.sqrt(2.0 / np.pi), 0.044715


def activation(name: str, z: np.ndarray):
    """act(z), act'(z), act''(z)."""
    z = np.asarray(z, dtype=np.float64)
    if name == "none":
        return z, np.ones_like(z), np.zeros_like(z)
    if name == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64), np.zeros_like(z)
    if name == "silu":
        t = np.tanh(z / 2)                       # logistic = (1 + t) / 2
        s, d = (1 + t) / 2, (1 - t * t) / 4      # and its first derivative
        return z * s, s + z * d, 2 * d - z * d * t
    t = np.tanh(_A * (z + _C * z ** 3))
    u1, u2 = _A * (1 + 3 * _C * z ** 2), 6 * _A * _C * z
    d = 1 - t * t
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * d * u1, d * u1 + 0.5 * z * (d * u2 - 2 * t * d * u1 * u1)


def forward(act: str, X, W, b=None, residual=None):
    """Y, Z."""
    Z = np.asarray(X, np.float64) @ np.asarray(W, np.float64)
    if b is not None:
        Z = Z + np.asarray(b, np.float64)
    Y = activation(act, Z)[0]
    return (Y if residual is None else Y + np.asarray(residual, np.float64)), Z


def backward(act: str, X, W, Z, dY):
    """dX, dW, db of sum(dY * Y)."""
    G = np.asarray(dY, np.float64) * activation(act, Z)[1]
    return G @ np.asarray(W, np.float64).T, np.asarray(X, np.float64).T @ G, G.sum(0)


def double_backward(act: str, X, W, Z, dY, HX):
    """ddY, X2, W2, b2: gradients of sum(HX * dX), dX = (dY act'(X W + b)) W^T, with respect to dY, X, W, b."""
    X, W, dY, HX = (np.asarray(x, np.float64) for x in (X, W, dY, HX))
    _, first, second = activation(act, Z)
    V = HX @ W
    S = V * dY * second
    return V * first, S @ W.T, X.T @ S + HX.T @ (dY * first), S.sum(0)
