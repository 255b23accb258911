"""The oracle of the training operators against its own definition: gradients against central
differences in 64 bits, and properties that hold exactly."""
import numpy as np
import pytest

from oracle import training as tr

# A central difference with step e errs by e^2 / 6 times a third derivative (of the order of one
# here) and by rounding, 2^-53 |f| / e: 1e-10 at e = 1e-5.
STEP, TOL = 1e-5, 1e-8


def differences(f, x):
    d = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += STEP
        down[i] -= STEP
        d[i] = (f(up) - f(down)) / (2 * STEP)
    return d


@pytest.mark.parametrize("rows,channels", [(1, 2), (3, 5), (2, 16)])
def test_layer_norm_gradients(rows, channels):
    rng = np.random.default_rng(1)
    x, weight = rng.standard_normal((2, rows, channels))
    gamma, beta = rng.standard_normal((2, channels))
    eps = 0.1
    _, mean, rstd = tr.layer_norm(x, gamma, beta, eps)
    dx, dgamma, dbeta = tr.layer_norm_backward(weight, x, gamma, mean, rstd)
    value = lambda x, g, b: (tr.layer_norm(x, g, b, eps)[0] * weight).sum()
    assert np.abs(dx - differences(lambda v: value(v, gamma, beta), x)).max() < TOL
    assert np.abs(dgamma - differences(lambda v: value(x, v, beta), gamma)).max() < TOL
    assert np.abs(dbeta - differences(lambda v: value(x, gamma, v), beta)).max() < TOL


@pytest.mark.parametrize("bias", [False, True])
def test_cross_entropy_gradients(bias):
    rng = np.random.default_rng(2)
    h, w, b = rng.standard_normal((5, 4)), rng.standard_normal((7, 4)), rng.standard_normal(7)
    b = b if bias else None
    target = np.array([0, 6, -100, 3, 9])      # the third is ignored, the last is no class
    dloss = rng.random(5)
    value = lambda h, w, b: (tr.cross_entropy(h, w, b, target)[0] * dloss).sum()
    dh, dw, db, _ = tr.cross_entropy_backward(h, w, b, target, dloss)
    assert np.abs(dh - differences(lambda v: value(v, w, b), h)).max() < TOL
    assert np.abs(dw - differences(lambda v: value(h, v, b), w)).max() < TOL
    if bias:
        assert np.abs(db - differences(lambda v: value(h, w, v), b)).max() < TOL
    assert not dh[2].any() and not dh[4].any()


def test_cross_entropy_of_masked_classes():
    h, w = np.ones((3, 2)), np.ones((3, 2))
    bias = np.array([0.0, -np.inf, 0.0])
    loss, lse = tr.cross_entropy(h, w, bias, np.array([0, 1, 2]))
    assert np.allclose(lse, 2 + np.log(2)) and loss[1] == np.inf
    loss, lse = tr.cross_entropy(h, w, np.full(3, -np.inf), np.array([0, 1, -100]))
    assert np.isneginf(lse).all() and (loss == [np.inf, np.inf, 0]).all()
    dh, dw, db, _ = tr.cross_entropy_backward(h, w, np.full(3, -np.inf), np.array([0, 1, 2]), np.ones(3))
    assert not dh.any() and not dw.any() and not db.any()


def test_update_keeps_singular_vectors():
    rng = np.random.default_rng(3)
    u, _ = np.linalg.qr(rng.standard_normal((4, 4)))
    v, _ = np.linalg.qr(rng.standard_normal((6, 4)))
    s = np.array([3.0, 2.0, 1.0, 0.5])
    o, _ = tr.orthogonalise((u * s) @ v.T)
    x = s / (np.linalg.norm(s) + np.float64(np.float32(1e-7)))
    a, b, c = (np.float64(np.float32(q)) for q in (3.4445, -4.7750, 2.0315))
    for _ in range(5):
        x = a * x + b * x ** 3 + c * x ** 5
    assert np.abs(o - (u * x) @ v.T).max() < 1e-12
    tall, _ = tr.orthogonalise(((u * s) @ v.T).T)
    assert np.abs(tall.T - o).max() < 1e-12
    assert not tr.orthogonalise(np.zeros((2, 3)))[0].any()
