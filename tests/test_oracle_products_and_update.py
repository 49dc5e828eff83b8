"""Pins of the oracles of the products by element and of the orthogonalised update (CPU)."""
import numpy as np
import pytest

from oracle import orthogonalised_update as oo
from oracle import products_by_element as op


def test_products_by_hand():
    W = np.array([[[1.0, 2.0], [3.0, 4.0]], [[0.0, 1.0], [1.0, 0.0]]])
    X = np.array([[[1.0, 1.0]], [[2.0, 5.0]], [[7.0, 7.0]]])
    z = [0, 1, -1]
    assert op.forward(z, X, W).tolist() == [[[4.0, 6.0]], [[5.0, 2.0]], [[0.0, 0.0]]]
    assert op.forward(z, X, W, np.ones((3, 1, 2))).tolist() == [[[5.0, 7.0]], [[6.0, 3.0]], [[1.0, 1.0]]]
    dX, dW = op.backward(z, X, W, np.array([[[1.0, 0.0]], [[0.0, 1.0]], [[9.0, 9.0]]]))
    assert dX.tolist() == [[[1.0, 3.0]], [[1.0, 0.0]], [[0.0, 0.0]]]
    assert dW.tolist() == [[[1.0, 0.0], [1.0, 0.0]], [[0.0, 2.0], [0.0, 5.0]]]


def test_products_gradients_are_differences():
    rng = np.random.default_rng(3)
    z, X, W, dY = rng.integers(-1, 4, 9), rng.normal(size=(9, 3, 5)), rng.normal(size=(4, 5, 2)), rng.normal(size=(9, 3, 2))
    dX, dW = op.backward(z, X, W, dY)
    loss = lambda x, w: (op.forward(z, x, w) * dY).sum()  # noqa: E731
    for grad, value, f in ((dX, X, lambda v: loss(v, W)), (dW, W, lambda v: loss(X, v))):
        for _ in range(20):
            at = tuple(rng.integers(0, s) for s in value.shape)
            up, down = value.copy(), value.copy()
            up[at] += 0.5
            down[at] -= 0.5
            assert abs(f(up) - f(down) - grad[at]) < 1e-12   # the loss is linear in each


def test_products_second_order_is_made_of_the_same_calls():
    """Gradients of sum(HX * dX): forward of HX, and dW with HX in the place of X."""
    rng = np.random.default_rng(4)
    z, X, W, dY, HX = rng.integers(0, 3, 6), rng.normal(size=(6, 1, 4)), rng.normal(size=(3, 4, 5)), rng.normal(size=(6, 1, 5)), rng.normal(size=(6, 1, 4))
    value = lambda w, g: (HX * op.backward(z, X, w, g)[0]).sum()  # noqa: E731
    ddY, W2 = op.forward(z, HX, W), op.backward(z, HX, W, dY)[1]
    for grad, base, f in ((ddY, dY, lambda v: value(W, v)), (W2, W, lambda v: value(v, dY))):
        for _ in range(10):
            at = tuple(rng.integers(0, s) for s in base.shape)
            up, down = base.copy(), base.copy()
            up[at] += 0.5
            down[at] -= 0.5
            assert abs(f(up) - f(down) - grad[at]) < 1e-12


@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (7, 1), (6, 6), (4, 11), (11, 4)])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_the_two_forms_of_the_iteration(shape, steps):
    U = np.random.default_rng(5).normal(size=shape)
    assert np.abs(oo.orthogonalise(U, steps) - oo.iterate(U, steps)).max() < 1e-12


def test_the_update_is_nearly_orthogonal():
    X = oo.orthogonalise(np.random.default_rng(6).normal(size=(24, 64)), 5)
    s = np.linalg.svd(X, compute_uv=False)
    assert 0.6 < s.min() and s.max() < 1.3
    assert (oo.orthogonalise(np.zeros((3, 4)), 5) == 0).all()


def test_step_by_hand():
    G, M, W = np.full((1, 1, 1), 2.0), np.full((1, 1, 1), 1.0), np.full((1, 1, 1), 3.0)
    M2, X, W2 = oo.step(G, M, W, mu=0.5, steps=0, rate=0.1, decay=0.2, scale=4.0)
    assert M2[0, 0, 0] == 2.5 and abs(X[0, 0, 0] - 3.25 / (3.25 + 1e-7)) < 1e-15
    assert abs(W2[0, 0, 0] - (0.98 * 3.0 - 0.4 * X[0, 0, 0])) < 1e-15
    assert oo.step(G, None, None, steps=0)[0] is None
    assert abs(oo.step(G, -M, W, mu=0.5, nesterov=False, steps=0)[1][0, 0, 0] - 1.0) < 1e-6
