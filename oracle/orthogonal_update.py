"""Float64 reference of the orthogonalised update (momentum, Newton-Schulz steps, step on the weights).

Written from the formulas of ``include/rl_loss.h`` (rl_muon_update) in plain NumPy:

    buf = mu buf + G;  U = G + mu buf (nesterov) or buf;  U = G without momentum
    X = U / (|U|_F + eps);  steps times: A = X X^T, X = a X + (b A + c A A) X
    update = s X;  weights = (1 - lr wd) weights - lr s X
"""

import numpy as np

NS_COEF = (3.4445, -4.7750, 2.0315)


def newton_schulz(U, steps=5, coef=NS_COEF, eps=1e-7):
    """X after `steps` steps from one matrix U [m, n] (in either orientation: the steps commute with
    the transpose, which only changes which product is the smaller)."""
    a, b, c = (float(np.float32(k)) for k in coef)
    X = np.asarray(U, np.float64)
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    X = X / (np.sqrt((X * X).sum()) + float(np.float32(eps)))
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if tall else X


def muon_update(grad, momentum=None, weights=None, *, lr=1e-5, mu=0.95, nesterov=True, weight_decay=0.0,
                update_scale=1.0, steps=5, coef=NS_COEF, eps=1e-7):
    """(momentum, X, update, weights) of a batch [batch, m, n], float64 (None where an input is None)."""
    f = lambda x: float(np.float32(x))  # noqa: E731  (the library takes its parameters in float32)
    G = np.asarray(grad, np.float64)
    buf, U = None, G
    if mu > 0:
        buf = f(mu) * np.asarray(momentum, np.float64) + G
        U = G + f(mu) * buf if nesterov else buf
    X = np.stack([newton_schulz(u, steps, coef, eps) for u in U]) if len(U) else np.zeros_like(U)
    W = None
    if weights is not None:
        W = (1.0 - f(lr) * f(weight_decay)) * np.asarray(weights, np.float64) - f(lr) * f(update_scale) * X
    return buf, X, f(update_scale) * X, W
