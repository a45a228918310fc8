"""Float64 references of the operators at the ends of the policy model: layer norm, the embedding, sampling.

TEST INFRASTRUCTURE, written from the statements in ``include/rl_loss.h`` in plain NumPy.
"""

import numpy as np


# ----------------------------------------------------------------------------- rl_layer_norm_fwd, rl_layer_norm_bwd

def layer_norm(x, w=None, b=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + float(np.float32(eps)))
    y = (x - mean[:, None]) * rstd[:, None]
    if w is not None:
        y = y * np.asarray(w, np.float64)
    if b is not None:
        y = y + np.asarray(b, np.float64)
    return y, mean, rstd


def layer_norm_grad(dy, x, mean, rstd, w=None, mask=None):
    """(dx, dw, db): the formula's, for the mean and rstd given."""
    dy, x = np.array(dy, np.float64), np.array(x, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    on = np.ones(len(x), bool) if mask is None else np.asarray(mask) != 0
    dy[~on] = 0.0
    x[~on] = 0.0
    h = np.where(on[:, None], (x - mean) * rstd, 0.0)
    g = dy if w is None else dy * np.asarray(w, np.float64)
    dx = rstd * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return np.where(on[:, None], dx, 0.0), (dy * h).sum(0), dy.sum(0)


# ----------------------------------------------------------------------------- rl_embedding_fwd, rl_embedding_bwd

def embedding(ids, w, scale=1.0):
    ids, w = np.asarray(ids, np.int64), np.asarray(w, np.float64)
    ok = (ids >= 0) & (ids < len(w))
    out = np.zeros((len(ids), w.shape[1]))
    out[ok] = w[ids[ok]] * float(np.float32(scale))
    return out


def embedding_grad(ids, d, V, scale=1.0):
    """(d W, sum of |scale d| of each element): the second bounds the roundings of a sum."""
    ids, d = np.asarray(ids, np.int64), np.asarray(d, np.float64) * float(np.float32(scale))
    ok = (ids >= 0) & (ids < V)
    dw, size = np.zeros((V, d.shape[1])), np.zeros((V, d.shape[1]))
    np.add.at(dw, ids[ok], d[ok])
    np.add.at(size, ids[ok], np.abs(d[ok]))
    return dw, size


# ----------------------------------------------------------------------------- rl_sample_tokens

def kept_tokens(z, T, top_k=0, top_p=1.0, min_p=0.0):
    """(p, indices of the kept tokens in vocabulary order) of a row with a finite largest entry: p = softmax(z / T)."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore"):
        p = np.exp((z - z.max()) / T)
    p /= p.sum()
    order = np.argsort(-z, kind="stable")
    order = order[: int((z > -np.inf).sum())]
    n = len(order)
    if top_k > 0:
        n = min(n, top_k)
    of_k = np.cumsum(p[order[:n]])
    least = n
    if top_p < 1:
        least = min(least, 1 + int((of_k < top_p * of_k[-1]).sum()))
    if min_p > 0:
        least = min(least, max(1, int((p[order] >= min_p * p[order[0]]).sum())))
    return p, np.sort(order[:least])


def sample(z, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability under softmax(z / T), log-probability among the kept ones, number kept) of one row."""
    z = np.asarray(z, np.float64)
    if T == 0:
        tok = int(np.argmax(z))
        p, _ = kept_tokens(z, 1.0)
        return tok, float(np.log(p[tok])), 0.0, 1
    p, left = kept_tokens(z, T, top_k, top_p, min_p)
    c = np.cumsum(p[left])
    hit = np.nonzero((c > u * c[-1]) & (p[left] > 0))[0]
    tok = int(left[hit[0]])
    return tok, float(np.log(p[tok])), float(np.log(p[tok] / c[-1])), len(left)
