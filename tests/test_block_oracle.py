"""Pins of oracle/block_oracle.py: gradients against central differences, the polynomial against singular values, the order of
rows against a plain sort."""
import numpy as np
import pytest

from oracle import block_oracle as K

STEP = 1e-6   # central differences of fp64 functions of order 1: error about 1e-6^2 and 1e-16 / 1e-6


def differences(f, a):
    d = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        up, down = a.copy(), a.copy()
        up[i] += STEP
        down[i] -= STEP
        d[i] = (f(up) - f(down)) / (2 * STEP)
    return d


@pytest.mark.parametrize("ptr", [None, [0, 3, 3, 7]])
@pytest.mark.parametrize("groups", [1, 2, 6])
def test_group_norm_gradients(ptr, groups):
    rng = np.random.default_rng([1, groups])
    x, dy = rng.standard_normal((7, 6)) + 0.5, rng.standard_normal((7, 6))
    gamma, beta = 1 + 0.3 * rng.standard_normal(6), 0.3 * rng.standard_normal(6)
    f = lambda x=x, gamma=gamma, beta=beta: (K.group_norm(x, groups, gamma, beta, ptr)[0] * dy).sum()
    dx, dgamma, dbeta, _, _ = K.group_norm_backward(x, dy, groups, gamma, beta, ptr)
    assert np.abs(dx - differences(lambda a: f(x=a), x)).max() < 1e-7
    assert np.abs(dgamma - differences(lambda a: f(gamma=a), gamma)).max() < 1e-7
    assert np.abs(dbeta - differences(lambda a: f(beta=a), beta)).max() < 1e-7


def test_group_norm_statistics():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((50, 12)) * 3 + 7
    one, zero = np.ones(12), np.zeros(12)
    y, mean, rstd = K.group_norm(x, 4, one, zero, [0, 0, 20, 50], eps=0.0)
    assert mean.shape == (3, 4) and not mean[0].any() and not rstd[0].any()
    part = x[20:50, 3:6]
    assert abs(mean[2, 1] - part.mean()) < 1e-12 and abs(rstd[2, 1] * part.std() - 1) < 1e-12
    z = (part - part.mean()) / part.std()
    assert np.allclose(y[20:50, 3:6], z / (1 + np.exp(-z)))


def test_group_rows_order():
    key = np.array([2, 0, 7, -3, 2, 1])
    ptr, perm = K.group_rows(key, 3)
    assert ptr.tolist() == [0, 2, 3, 6] and perm.tolist() == [1, 3, 5, 0, 2, 4]
    ptr, perm = K.group_rows(np.array([1, 0, 1]), 2, lmax=1)
    assert ptr.tolist() == [0, 1, 4, 6, 12]
    assert perm.tolist() == [4, 5, 6, 7, 0, 8, 1, 2, 3, 9, 10, 11]


def test_grouped_linear_gradients():
    rng = np.random.default_rng(3)
    key = np.array([0, 2, 2, 0, 2])
    ptr, perm = K.group_rows(key, 4)
    x, W, b, dy = (rng.standard_normal(s) for s in ((5, 3), (4, 2, 3), (4, 2), (5, 2)))
    y, _ = K.grouped_linear(x, W, ptr, perm, b)
    for r in range(5):
        assert np.allclose(y[r], W[key[r]] @ x[r] + b[key[r]])
    f = lambda x=x, W=W, b=b: (K.grouped_linear(x, W, ptr, perm, b)[0] * dy).sum()
    dx, dW, db = K.grouped_linear_backward(x, W, dy, ptr, perm)[:3]
    assert np.abs(dx - differences(lambda a: f(x=a), x)).max() < 1e-8
    assert np.abs(dW - differences(lambda a: f(W=a), W)).max() < 1e-8
    assert np.abs(db - differences(lambda a: f(b=a), b)).max() < 1e-8


@pytest.mark.parametrize("shape", [(1, 1), (5, 5), (4, 9), (9, 4)])
@pytest.mark.parametrize("steps", [1, 5])
def test_orthogonalise_acts_on_singular_values(shape, steps):
    rng = np.random.default_rng(4)
    g = rng.standard_normal((2, *shape))
    q = K.orthogonalise(g, steps)
    for i in range(2):
        u, s, v = np.linalg.svd(g[i], full_matrices=False)
        s = s / (np.linalg.norm(g[i]) + 1e-7)
        for _ in range(steps):
            s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
        assert np.abs(q[i] - (u * s) @ v).max() < 1e-12


def test_muon_step():
    rng = np.random.default_rng(5)
    W, g, m = (rng.standard_normal((1, 8, 2)) for _ in range(3))
    W2, m2 = K.muon_step(W, g, m, 0.1, beta=0.9, weight_decay=0.5)
    assert np.allclose(m2, 0.9 * m + g)
    assert np.allclose(W2, 0.95 * W - 0.2 * K.orthogonalise(g + 0.9 * (0.9 * m + g)))
