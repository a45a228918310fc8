"""The example's iterations: rollouts by verified drafts, the loss, and the orthogonalised updates together."""

import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_reward_rises_and_the_drafter_falls_behind():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import rl_iteration as E

    rewards, accepted = E.train(iterations=12)
    # 64 rollouts of 24 tokens at reward 1/2 each: a standard error of 0.013, the first mean within five of them
    assert abs(rewards[0] - 0.5) < 0.07
    # the drafter is the policy at the start: equal rows accept every token
    assert accepted[0] == 1.0
    assert sum(rewards[-3:]) / 3 > rewards[0] + 0.1
    assert accepted[-1] < 1.0
    # the same seed, the same run
    again, _ = E.train(iterations=2)
    assert again == rewards[:2]
