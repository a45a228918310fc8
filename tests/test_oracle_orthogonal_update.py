"""Pins of the orthogonalised update's float64 reference: what the formula must give whatever computes it."""

import numpy as np
import pytest

import oracle.orthogonal_update as O


def _f(x):
    a, b, c = (float(np.float32(k)) for k in O.NS_COEF)
    return a * x + b * x ** 3 + c * x ** 5


@pytest.mark.parametrize("m,n", [(1, 1), (3, 7), (7, 3), (8, 8), (1, 9), (9, 1)])
def test_singular_values_go_through_the_polynomial(m, n):
    rng = np.random.default_rng(m * 31 + n)
    U = rng.normal(size=(m, n))
    u, s, vt = np.linalg.svd(U, full_matrices=False)
    x = s / (np.sqrt((s * s).sum()) + float(np.float32(1e-7)))
    for _ in range(5):
        x = _f(x)
    assert np.abs(O.newton_schulz(U) - (u * x) @ vt).max() < 1e-12


def test_the_polynomial_keeps_its_interval():
    x = np.linspace(0.0, 1.25, 100001)
    assert _f(x).min() >= -1e-12 and _f(x).max() < 1.25


def test_equivariance_and_scale():
    rng = np.random.default_rng(5)
    U = rng.normal(size=(5, 9))
    q = np.linalg.qr(rng.normal(size=(5, 5)))[0]
    X = O.newton_schulz(U, eps=0.0)
    assert np.abs(O.newton_schulz(q @ U, eps=0.0) - q @ X).max() < 1e-12
    assert np.abs(O.newton_schulz(U * 1e9, eps=0.0) - X).max() < 1e-12
    assert np.abs(O.newton_schulz(U.T, eps=0.0) - X.T).max() < 1e-12
    assert not O.newton_schulz(np.zeros((4, 6))).any()


def test_momentum_and_weights():
    rng = np.random.default_rng(6)
    G, M, W = rng.normal(size=(3, 2, 4, 6))
    buf, X, upd, w = O.muon_update(G, M, W, lr=0.5, mu=0.5, weight_decay=0.25, update_scale=2.0)
    assert np.allclose(buf, 0.5 * M + G) and np.allclose(X, [O.newton_schulz(g + 0.5 * b) for g, b in zip(G, buf)])
    assert np.allclose(upd, 2 * X) and np.allclose(w, 0.875 * W - X)
    _, Xn, _, _ = O.muon_update(G, M, None, mu=0.5, nesterov=False)
    assert np.allclose(Xn, [O.newton_schulz(b) for b in buf])
    assert O.muon_update(G, None, None, mu=0.0)[0] is None
