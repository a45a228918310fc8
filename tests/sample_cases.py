"""Rows of logits with settings for the tests of rl_sample_tokens. top_p, min_p and the given numbers are kept away from the
edges at which a whole number of the result changes, as far as fp32 sums can be off."""

import numpy as np

import oracle.model_ends as O
from verify_cases import values

EDGE = 2e-5    # distance of u and top_p from the edges of their token's interval
LEAST = 1e-4   # mass of a token at which top_p ends, or that u selects, if any has as much


def rows(law, n, V, dtype, rng):
    z = rng.normal(0, 2.0, (n, V))
    if law == "likely":
        z[np.arange(n), rng.integers(0, V, n)] += np.log(V) + 2.0
    elif law == "ties":  # few different values
        z = np.rint(z)
    elif law == "equal":
        z = np.full((n, V), 3.0)
    elif law == "signed_zero":
        z = np.where(rng.random((n, V)) < 0.5, 0.0, -0.0) - 4.0 * (rng.random((n, V)) < 0.5)
    elif law == "negative":
        z = z - 60.0
    elif law == "masked":
        z[rng.random((n, V)) < 0.5] = -np.inf
        z[np.arange(n), rng.integers(0, V, n)] = 4.0
    elif law == "one_left":
        z[:] = -np.inf
        z[np.arange(n), rng.integers(0, V, n)] = -3.0
    elif law == "finite_masks":  # of the type's lowest value, and of a large one
        z = np.where(rng.random((n, V)) < 0.6, np.where(rng.random((n, V)) < 0.5, -3.38e38, -1e10), z)
        z[np.arange(n), rng.integers(0, V, n)] = 5.0
    elif law == "far":  # borders many powers of two below the largest entry
        z = np.where(rng.random((n, V)) < 0.5, 1.0, -1.0) * np.exp2(rng.uniform(-40, 0, (n, V)))
    elif law == "close":  # fp32 entries that differ in their last bits
        z = 1.0 + rng.integers(0, 40, (n, V)) * 2.0 ** -23
    elif law == "large":
        z = z * 1e4
    return values(z, dtype)


def away_from_edges(z, T, top_k, top_p, min_p, s):
    """(top_p, min_p, u) near those given, at which the row's result does not hang on rounding."""
    if T == 0:
        return float(np.float32(top_p)), float(np.float32(min_p)), float(np.float32(s))
    if top_p < 1:
        p, left = O.kept_tokens(z, T, top_k)
        o = left[np.argsort(-z[left], kind="stable")]
        m = p[o] / p[o].sum()
        c = np.cumsum(m)
        at = min(int((c < top_p).sum()), max(0, int((m >= LEAST).sum()) - 1), len(m) - 1)
        top_p = c[at] - 0.5 * m[at]
        if top_p >= 1 - 1e-6:
            top_p = 0.999
    if min_p > 0:
        r = np.sort(np.unique(z[z > -np.inf]))[::-1]
        rel = np.exp((r - r[0]) / T)
        at = int((rel >= min_p).sum())
        pairs = [(rel[i - 1], rel[i]) for i in range(max(1, at - 8), min(len(rel), at + 9))] or [(1.0, 0.0)]
        hi, lo = max(pairs, key=lambda x: x[0] / max(x[1], 1e-300))
        min_p = np.sqrt(hi * max(lo, hi * 0.25))
    top_p, min_p = float(np.float32(top_p)), float(np.float32(min_p))
    p, left = O.kept_tokens(z, T, top_k, top_p, min_p)
    c = np.cumsum(p[left]) / p[left].sum()
    m = p[left] / p[left].sum()
    at = min(int((c <= s).sum()), len(c) - 1)
    if m[at] < LEAST:
        at = int(np.argmax(m))
    return top_p, min_p, min(float(np.float32(c[at] - m[at] * (0.3 + 0.4 * s))), 1 - 2.0 ** -24)


def solid(z, T, top_k, top_p, min_p, u):
    """Whether the row's result does not hang on rounding: the masses at its borders are large enough."""
    if T == 0:
        return True
    p, left = O.kept_tokens(z, T, top_k)
    o = left[np.argsort(-z[left], kind="stable")]
    if top_p < 1:
        m = p[o] / p[o].sum()
        c = np.cumsum(m)
        if np.abs(c - top_p).min() < EDGE * 0.5:
            return False
    if min_p > 0:
        rel = np.exp((z[left] - z.max()) / T)
        if np.abs(rel / min_p - 1).min() < 1e-5:
            return False
    p, left = O.kept_tokens(z, T, top_k, top_p, min_p)
    c = np.cumsum(p[left]) / p[left].sum()
    return np.abs(c[:-1] - u).min(initial=1.0) > EDGE * 0.5
