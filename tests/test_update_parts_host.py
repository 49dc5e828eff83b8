"""The limit that tests/test_gpu_orthogonalised_update_exactness.py holds the update's products to, against the arithmetic of parts in numpy (no GPU): two fp16 parts of every operand stay
inside it, a product that loses one is far outside, with every set of coefficients that the test has."""
import numpy as np
import pytest

from oracle import orthogonalised_update as oo
from test_gpu_orthogonalised_update_exactness import HELD, decaying, in_fp32


def parts(v, top, number):
    """v as fp16 values times a power of two that brings `top` to 2^14."""
    up = np.float32(2.0 ** (14 - np.ceil(np.log2(max(top, 1e-3)))))
    h = (v * up).astype(np.float16)
    low = (v * up - h.astype(np.float32)).astype(np.float16) if number == 2 else np.zeros_like(h)
    return h.astype(np.float64), low.astype(np.float64), np.float64(up)


def product(x, y):
    """Rows with rows; the product of the second parts is left out."""
    return ((x[0] @ y[0].T + x[0] @ y[1].T + x[1] @ y[0].T) / (x[2] * y[2])).astype(np.float32)


def iterate(U, steps, coefficients, number):
    a, b, c = (np.float32(v) for v in coefficients)
    X = (U / np.sqrt((U ** 2).sum())).astype(np.float32)
    turned = X.shape[0] > X.shape[1]
    X = X.T if turned else X
    top, x = 1.0, np.linspace(0, 1, 1001)
    for _ in range(steps):
        bound = abs(coefficients[1]) * top ** 2 + abs(coefficients[2]) * top ** 4
        p = parts(X, top, number)
        S = product(p, p)
        s = parts(S, top ** 2, number)
        P = b * S + c * product(s, s)
        X = a * X + product(parts(P, bound, number), parts(X.T, top, number))
        top = np.abs(np.polyval([coefficients[2], 0, coefficients[1], 0, coefficients[0], 0], x * top)).max()
    return X.T if turned else X


@pytest.mark.parametrize("coefficients,steps", HELD, ids=str)
@pytest.mark.parametrize("shape", [(64, 64), (33, 50), (128, 100), (64, 300), (150, 200)], ids=str)
def test_a_lost_part_is_seen(shape, coefficients, steps):
    rng = np.random.default_rng(7)
    norm = lambda x: np.sqrt((x ** 2).sum())  # noqa: E731
    for U in (rng.normal(size=shape), decaying(rng, (1,) + shape)[0]):
        want = oo.iterate(U, steps, 0.0, coefficients)
        plain = max(norm(in_fp32(U, steps, coefficients, 0.0) - want), steps * 2.0 ** -24 * norm(want))
        assert norm(iterate(U, steps, coefficients, 2) - want) <= 8 * plain
        lost = norm(iterate(U, steps, coefficients, 1) - want) / plain
        assert lost > 16, lost
