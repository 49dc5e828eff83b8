"""Pins of the oracles of the dense layer, the element embedding and the gradient clipping (CPU)."""
import math

import numpy as np
import pytest

from oracle import dense_layer as od
from oracle import element_embedding as oe
from oracle import gradient_clipping as og


@pytest.mark.parametrize("act", od.ACTIVATIONS)
def test_activation_values_and_derivatives(act):
    z = np.concatenate([np.linspace(-8, 8, 41) + 0.013, [-60.0, 45.0]])
    f = {"none": lambda v: v, "relu": lambda v: max(v, 0.0), "silu": lambda v: v / (1 + math.exp(-v)),
         "gelu": lambda v: v / (1 + math.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))) if abs(v) < 12 else max(v, 0.0)}[act]
    value, first, second = od.activation(act, z)
    assert np.abs(value - [f(v) for v in z]).max() < 1e-13
    h = 1e-5
    up, down = od.activation(act, z + h), od.activation(act, z - h)
    assert np.abs((up[0] - down[0]) / (2 * h) - first).max() < 1e-9     # h^2 |act'''| / 6 and 1e-15 * 60 / h
    assert np.abs((up[1] - down[1]) / (2 * h) - second).max() < 1e-9


def _layer(act, seed=3):
    rng = np.random.default_rng(seed)
    X, W, b, R = rng.standard_normal((5, 4)), rng.standard_normal((4, 3)), rng.standard_normal(3), rng.standard_normal((5, 3))
    return rng, X, W, b, R


@pytest.mark.parametrize("act", od.ACTIVATIONS)
def test_gradients_are_finite_differences(act):
    rng, X, W, b, R = _layer(act)
    dY, HX = rng.standard_normal((5, 3)), rng.standard_normal((5, 4))
    Z = od.forward(act, X, W, b, R)[1]
    dX, dW, db = od.backward(act, X, W, Z, dY)
    ddY, X2, W2, b2 = od.double_backward(act, X, W, Z, dY, HX)
    first = lambda X, W, b, dY: float((dY * od.forward(act, X, W, b, R)[0]).sum())                            # noqa: E731
    second = lambda X, W, b, dY: float((HX * od.backward(act, X, W, od.forward(act, X, W, b, R)[1], dY)[0]).sum())  # noqa: E731
    for f, grads in ((first, (dX, dW, db, None)), (second, (X2, W2, b2, ddY))):
        args = [X, W, b, dY]
        for n, grad in enumerate(grads):
            if grad is None:
                continue
            for at in np.ndindex(grad.shape):
                h = 1e-5
                lo, hi = [a.copy() for a in args], [a.copy() for a in args]
                lo[n][at] -= h
                hi[n][at] += h
                assert abs((f(*hi) - f(*lo)) / (2 * h) - grad[at]) < 1e-7


def test_embedding_is_the_product_with_one_hot_rows():
    rng = np.random.default_rng(5)
    z = np.array([2, 0, -1, 2, 4, 5, 2], dtype=np.int32)      # -1 and 5 are outside of a table of 5 rows
    T, dY = rng.standard_normal((5, 6)), rng.standard_normal((7, 6))
    hot = (z[:, None] == np.arange(5)[None, :]).astype(float)
    assert np.abs(oe.forward(z, T, 0.3) - 0.3 * hot @ T).max() < 1e-15
    assert np.abs(oe.backward(z, dY, 5, 0.3) - 0.3 * hot.T @ dY).max() < 1e-15


def test_clipping():
    x = [np.array([3.0, 0.0]), np.zeros(0), np.array([[4.0]])]
    norm, c, out = og.clip(x, 1.0, 0.0)
    assert norm == 5.0 and c == 0.2 and np.abs(out[2] - 0.8).max() < 1e-15
    assert og.clip(x, 10.0, 0.0)[1] == 1.0 and og.clip([], 1.0, 0.0) == (0.0, 1.0, [])
