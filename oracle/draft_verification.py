"""Float64 reference of the verification of drafted tokens (speculative decoding's acceptance test).

TEST INFRASTRUCTURE, written from the statement in ``include/rl_loss.h`` (rl_verify_drafts): token j is
accepted while u_j q(x_j) < p(x_j); the first refused token is replaced by the draw from max(p - q, 0),
and without a refusal one more is drawn from the last row's p. A draw is the lowest v at which the running
sum of the weights, in vocabulary order, passes s times their total.
"""

import numpy as np


def softmax(z, T):
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.exp((z - z.max()) / T)
    return e / e.sum()


def draw(weights, s):
    c = np.cumsum(weights)
    hit = np.nonzero((c > s * c[-1]) & (weights > 0))[0]
    return int(hit[0]) if len(hit) else int(np.nonzero(weights > 0)[0][-1])


def residual(p, q):
    r = np.maximum(p - q, 0.0)
    return r if r.any() else p


def verify_one(target, draft, ids, u, s, T):
    """(accepted tokens and the one drawn, their log-probabilities) of one sequence: target [K + 1, V],
    draft [K, V] or None."""
    out, logp = [], []
    scale = T if T > 0 else 1.0
    for j in range(len(ids) + 1):
        p = softmax(target[j], scale)
        with np.errstate(divide="ignore"):
            lp = np.log(p)
        if T == 0:
            tok = int(np.argmax(target[j]))
            more = j < len(ids) and ids[j] == tok
        elif j < len(ids):
            x = int(ids[j])
            if draft is None:
                q = np.zeros_like(p)
                q[x] = 1.0
            else:
                q = softmax(draft[j], scale)
            more = float(u[j]) * q[x] < p[x]
            tok = x if more else draw(residual(p, q), float(s))
        else:
            more, tok = False, draw(p, float(s))
        out.append(tok)
        logp.append(lp[tok])
        if not more:
            return out, logp


def verify(target, draft, ids, offsets, u, s, T):
    """(out_ids, n_accepted, out_logp) of packed sequences, laid out as the target rows."""
    n = len(offsets) - 1
    rows = int(offsets[-1]) + n
    out, lp, acc = np.full(rows, -1, np.int64), np.zeros(rows), np.zeros(n, np.int64)
    for b in range(n):
        o, o1 = int(offsets[b]), int(offsets[b + 1])
        r = o + b
        got, l = verify_one(target[r:r + o1 - o + 1], None if draft is None else draft[o:o1], ids[o:o1], u[o:o1], s[b], T)
        out[r:r + len(got)], lp[r:r + len(got)], acc[b] = got, l, len(got) - 1
    return out, acc, lp
