"""fp64 oracle of the orthogonalised update.  The iteration acts on the singular values alone, so it is done there.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import numpy as np

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def polynomial(s, steps, coefficients=COEFFICIENTS):
    a, b, c = coefficients
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


def orthogonalise(U, steps, eps=1e-7, coefficients=COEFFICIENTS):
    """The iteration on one matrix, by its singular values."""
    left, s, right = np.linalg.svd(U, full_matrices=False)
    return (left * polynomial(s / (np.sqrt((s ** 2).sum()) + eps), steps, coefficients)) @ right


def iterate(U, steps, eps=1e-7, coefficients=COEFFICIENTS):
    """The iteration on one matrix, as it is defined."""
    a, b, c = coefficients
    X = U / (np.sqrt((U ** 2).sum()) + eps)
    turned = X.shape[0] > X.shape[1]
    X = X.T if turned else X
    for _ in range(steps):
        S = X @ X.T
        X = a * X + (b * S + c * S @ S) @ X
    return X.T if turned else X


def step(G, M, W, *, mu=0.95, nesterov=True, steps=5, eps=1e-7, rate=0.02, decay=0.0, scale=1.0, coefficients=COEFFICIENTS, form=orthogonalise):
    """Momentum, update and weight after a step; batches [count][rows][cols], M or W may be None."""
    if M is not None:
        M = mu * M + G
    U = G if M is None else G + mu * M if nesterov else M
    X = np.stack([form(u, steps, eps, coefficients) for u in U])
    return M, X, None if W is None else (1 - rate * decay) * W - rate * scale * X
