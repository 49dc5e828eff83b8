"""fp64 oracle of the global gradient norm and clipping.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import math

import numpy as np


def clip(tensors, max_norm: float, eps: float):
    """norm, coefficient, clipped tensors."""
    norm = math.sqrt(math.fsum(float(v) * float(v) for x in tensors for v in np.asarray(x, np.float64).ravel()))
    coefficient = min(1.0, max_norm / (norm + eps)) if norm + eps > 0 else 1.0
    return norm, coefficient, [coefficient * np.asarray(x, np.float64) for x in tensors]
