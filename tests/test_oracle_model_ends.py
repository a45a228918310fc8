"""Pins of the float64 references of the model's ends: against differences, autograd and a sum over all tokens by hand."""

import math

import numpy as np
import torch

import oracle.model_ends as O


def test_layer_norm_and_its_gradient():
    rng = np.random.default_rng(0)
    x, w, b, dy = rng.normal(1, 2, (4, 13)), rng.normal(1, 0.3, 13), rng.normal(0, 0.2, 13), rng.normal(0, 1, (4, 13))
    y, mean, rstd = O.layer_norm(x, w, b, 1e-5)
    t = [torch.tensor(a, requires_grad=True) for a in (x, w, b)]
    ref = torch.nn.functional.layer_norm(t[0], (13,), t[1], t[2], float(np.float32(1e-5)))
    assert np.allclose(y, ref.detach().numpy(), rtol=1e-12, atol=1e-12)
    ref.backward(torch.tensor(dy))
    dx, dw, db = O.layer_norm_grad(dy, x, mean, rstd, w)
    for got, leaf in zip((dx, dw, db), t):
        assert np.allclose(got, leaf.grad.numpy(), rtol=1e-10, atol=1e-12)
    h = 1e-6
    for d in (rng.normal(0, 1, (4, 13)) for _ in range(3)):
        diff = ((O.layer_norm(x + h * d, w, b)[0] - O.layer_norm(x - h * d, w, b)[0]) * dy).sum() / (2 * h)
        assert abs(diff - (dx * d).sum()) < 1e-7
    mask = np.array([1, 0, 1, 0])
    mx, mw, mb = O.layer_norm_grad(dy, x, mean, rstd, w, mask)
    assert (mx[1::2] == 0).all() and np.allclose(mx[::2], dx[::2]) and np.allclose(mb, dy[::2].sum(0))
    assert np.allclose(mw, (dy * ((x - mean[:, None]) * rstd[:, None]))[::2].sum(0))


def test_embedding_and_its_gradient():
    rng = np.random.default_rng(1)
    ids, w, d = np.array([3, 0, 3, 9, -1, 3]), rng.normal(size=(5, 4)), rng.normal(size=(6, 4))
    out = O.embedding(ids, w, 0.5)
    assert (out[3] == 0).all() and (out[4] == 0).all() and np.allclose(out[0], 0.5 * w[3])
    dw, size = O.embedding_grad(ids, d, 5, 0.5)
    assert np.allclose(dw[3], 0.5 * (d[0] + d[2] + d[5])) and np.allclose(dw[0], 0.5 * d[1]) and (dw[[1, 2, 4]] == 0).all()
    assert (size >= np.abs(dw) - 1e-12).all()


def brute(z, u, T, k, p, m):
    """The definition with lists: (token, number kept)."""
    live = [v for v in range(len(z)) if z[v] > -math.inf]
    top = max(z)
    w = {v: math.exp((z[v] - top) / T) for v in live}
    order = sorted(live, key=lambda v: (-z[v], v))
    of_k = order[:k] if k else order
    total, before, keep = math.fsum(w[v] for v in of_k), 0.0, []
    for v in of_k:
        if p < 1 and not before < p * total:
            break
        if m > 0 and keep and w[v] < m * w[order[0]]:
            break
        keep.append(v)
        before += w[v]
    goal, run = u * math.fsum(w[v] for v in keep), 0.0
    for v in sorted(keep):
        run += w[v]
        if run > goal:
            return v, len(keep)


def test_sampling_by_hand():
    rng = np.random.default_rng(2)
    for trial in range(400):
        V = int(rng.integers(1, 12))
        z = np.rint(rng.normal(0, 2, V)) if trial % 2 else rng.normal(0, 2, V)
        z[rng.random(V) < 0.2] = -np.inf
        z[rng.integers(0, V)] = 1.0
        T, k = float(rng.choice([0.5, 1.0, 2.0])), int(rng.choice([0, 1, 3, 100]))
        p, m = float(rng.choice([1.0, 0.83, 0.31])), float(rng.choice([0.0, 0.07, 0.9]))
        u = float(rng.random())
        tok, lp, among, n = O.sample(z, u, T, k, p, m)
        assert (tok, n) == brute(list(z), u, T, k, p, m), (z, T, k, p, m, u)
        soft = np.exp(z / T) / np.exp(z / T).sum()
        assert math.isclose(lp, math.log(soft[tok]), abs_tol=1e-12) and among >= lp - 1e-12
    assert O.sample([1.0, 3.0, 3.0], 0.9, 0.0)[0] == 1  # greedy: the lowest index of the largest
