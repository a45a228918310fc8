"""Packed sequences with drafted tokens for the tests of rl_verify_drafts, with their random numbers kept
away from the edges at which a whole number of the result changes (as far as float32 sums can be off)."""

import numpy as np

import oracle.draft_verification as O
from paper_2608_16798_gb300 import workloads as W

ACCEPT_BAND = 1e-4  # relative distance of u from p(x) / q(x)
CDF_BAND = 2e-5     # distance of s from the edges of its token's interval


def values(x, dtype):
    """x rounded to dtype, as float64."""
    x = np.asarray(x, np.float32)
    if dtype == "bf16":
        bits = W.bf16_bits_from_f32(x)
        x = (bits.astype(np.uint32) << 16).view(np.float32)
    return x.astype(np.float64)


def inside(weights, s):
    """A number near s that lies well inside the interval of a token of these weights."""
    w = weights / weights.sum()
    c = np.cumsum(w)
    v = O.draw(w, s)
    if w[v] < 3 * CDF_BAND:
        v = int(np.argmax(w))
    lo = c[v] - w[v]
    return float(np.float32(lo + CDF_BAND + s * (w[v] - 2 * CDF_BAND)))


def make(counts, V, dtype="f32", draft=True, T=1.0, std=2.0, noise=0.7, masked=0.0, mask_value=-np.inf, seed=0,
         likely=0.5, mask_from=None, shift=None):
    """dict(target, draft, ids, offsets, u, s, T): float64 rows with exactly representable entries. Entries are masked at
    random and, with mask_from, from there on; with shift they are whole numbers around it."""
    rng = np.random.default_rng(seed)
    K = np.asarray(counts, np.int64)
    offsets = np.concatenate([[0], np.cumsum(K)]).astype(np.int32)
    nd, n = int(K.sum()), len(K)
    z = rng.normal(0, std, (nd + n, V))
    zd = z[[r for b in range(n) for r in range(offsets[b] + b, offsets[b + 1] + b)]] + rng.normal(0, noise, (nd, V))
    hot = rng.integers(0, V, nd + n)
    z[np.arange(nd + n), hot] += np.where(rng.random(nd + n) < likely, np.log(V) + std * std / 2, 0)
    if shift is not None:
        z, zd = np.rint(z) + shift, np.rint(zd) + shift
    if masked:
        off = rng.random(z.shape) < masked
        if mask_from is not None:
            off[:, mask_from:] = True
        off[np.arange(nd + n), hot] = False
        z = np.where(off, mask_value, z)
        if nd:
            t_row = np.concatenate([np.arange(offsets[b], offsets[b + 1]) + b for b in range(n)])
            zd = np.where(off[t_row], mask_value, zd)
    z, zd = values(z, dtype), values(zd, dtype)
    scale = T if T > 0 else 1.0
    ids, u, s = np.zeros(nd, np.int32), np.zeros(nd, np.float32), np.zeros(n, np.float32)
    for b in range(n):
        weights = None
        for j in range(K[b]):
            i, r = offsets[b] + j, offsets[b] + b + j
            p = O.softmax(z[r], scale)
            if draft:
                q = O.softmax(zd[i], scale)
                ids[i] = O.draw(q, rng.random())
            else:
                q = np.zeros(V)
                ids[i] = hot[r] if rng.random() < 0.7 else O.draw(p, rng.random())
                q[ids[i]] = 1.0
            if T == 0 and rng.random() < 0.7:
                ids[i] = int(np.argmax(z[r]))
            ratio = p[ids[i]] / max(q[ids[i]], 1e-300)
            x = rng.random()
            if abs(x - ratio) <= ACCEPT_BAND * ratio:
                x = ratio * (1 + 4 * ACCEPT_BAND) if ratio < 0.9 else ratio * (1 - 4 * ACCEPT_BAND)
            u[i] = min(x, 1 - 2.0 ** -24)
            if weights is None and not float(u[i]) * q[ids[i]] < p[ids[i]]:
                weights = O.residual(p, q)
        if weights is None:
            weights = O.softmax(z[offsets[b + 1] + b], scale)
        s[b] = inside(weights, rng.random())
    return dict(target=z, draft=zd if draft and nd else None, ids=ids, offsets=offsets, u=u, s=s, T=T, dtype=dtype,
                max_draft=int(K.max(initial=0)))


def expected(c):
    return O.verify(c["target"], c["draft"], c["ids"], c["offsets"], c["u"], c["s"], c["T"])
