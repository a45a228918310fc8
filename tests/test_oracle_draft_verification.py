"""Pins of the draft verification's float64 reference: what speculative sampling has to give whatever
computes it."""

import numpy as np
import pytest

import oracle.draft_verification as O
import verify_cases as V


def first_token_distribution(target, draft, T, with_rows, n=400):
    """The distribution of the first emitted token over all drafts x ~ q and stratified numbers."""
    p, q = O.softmax(target[0], T), O.softmax(draft[0], T)
    grid = (np.arange(n) + 0.5) / n
    got = np.zeros(len(p))
    for x in range(len(p)):
        for u in grid:
            a = np.array([x], np.int32)
            out, _ = O.verify_one(target, draft if with_rows else None, a, [u], 0.5, T)
            if len(out) > 1:
                got[x] += q[x] / n
            else:  # refused: the draw's distribution
                one = np.zeros_like(p)
                one[x] = 1.0
                r = O.residual(p, q if with_rows else one)
                got += q[x] / n * r / r.sum()
    return p, got


@pytest.mark.parametrize("with_rows", [True, False])
@pytest.mark.parametrize("T", [1.0, 0.5])
def test_the_emitted_token_follows_the_target(T, with_rows):
    rng = np.random.default_rng(3)
    target, draft = rng.normal(0, 1.5, (2, 6)), rng.normal(0, 1.5, (1, 6))
    p, got = first_token_distribution(target, draft, T, with_rows)
    assert np.abs(got - p).max() < 1.0 / 400


def test_draws_cover_their_intervals():
    w = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [O.draw(w, s) for s in (0.0, 0.2499, 0.25, 0.7499, 0.75, 0.9999, 1.0)] == [1, 1, 3, 3, 4, 4, 4]


def test_equal_rows_accept_everything():
    c = V.make([3, 0, 2], 11, noise=0.0, likely=0.0, seed=1)
    c["draft"] = c["target"][[0, 1, 2, 5, 6]]
    out, n, lp = V.expected(c)
    assert n.tolist() == [3, 0, 2]
    assert (out[[0, 1, 2]] == c["ids"][:3]).all() and np.isfinite(lp).all()


def test_greedy_takes_the_first_largest():
    z = np.array([[0.0, 2.0, 2.0], [1.0, 0.0, 1.0]])
    assert O.verify_one(z, None, [1], [0.9], 0.9, 0.0)[0] == [1, 0]
    assert O.verify_one(z, None, [2], [0.0], 0.0, 0.0)[0] == [1]


def test_layout_and_masks():
    c = V.make([2, 0, 4, 1], 40, masked=0.5, seed=2)
    out, n, lp = V.expected(c)
    assert len(out) == 7 + 4 and (n <= [2, 0, 4, 1]).all()
    for b in range(4):
        r = c["offsets"][b] + b
        k = c["offsets"][b + 1] - c["offsets"][b]
        assert (out[r:r + n[b] + 1] >= 0).all() and (out[r + n[b] + 1:r + k + 1] == -1).all()
        for j in range(n[b] + 1):
            assert np.isfinite(c["target"][r + j, out[r + j]])
