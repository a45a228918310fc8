"""The ends of the model and the loss together, as a training step uses them: tokens drawn by rl_sample_tokens from a policy whose
embedding is tied to its LM head, hidden = layer norm(scale embedding), the loss through the fused head, and its gradient back
through the norm into the matrix to which the head has added its own.

The whole gradient is compared with the loss's differences along it, in float64 without any rounding between the stages. The step
rounds five times to bf16 on the way (embedding, hidden, gradient of the logits, d hidden, d embedding), each by at most half a
step, 2^-8 relative: 5 / 256 of the gradient's norm, and 2^-5 is allowed. Where a tied head makes the policy certain (entries of 0.3:
a token's own logit is 128 x 0.3), the gradient is c A (1 - p) h with 1 - p far below p's rounding in fp32: it is off by up to
2^-23 c |A| |h| |d| for every token and each of the places where its row of the matrix enters, |h| about 12 and the norm's and the
scale's factors in d at most 40. Each stage is held to its own reference, at its own tolerance, in the tests of its operator.
"""

import numpy as np
import pytest
import torch

import oracle.grpo_objective as G
import oracle.model_ends as O

pytestmark = pytest.mark.gpu

V, D, T, SCALE = 700, 128, 96, 3.0


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R

    R.lib()
    return R


class Step:
    """One step's buffers, as a program keeps them."""

    def __init__(self, R, seed, size=0.3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.R = R
        self.w = (torch.randn(V, D, generator=g, device="cuda") * size).bfloat16()
        self.ln = 1 + 0.2 * torch.randn(D, generator=g, device="cuda")
        self.bias = 0.1 * torch.randn(D, generator=g, device="cuda")
        self.before = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        self.u = torch.rand(T, generator=g, device="cuda")
        self.mask = (torch.rand(T, generator=g, device="cuda") < 0.7).to(torch.uint8)
        self.adv, self.coef = torch.tensor([0.7, -0.4, 1.1], device="cuda"), torch.tensor([0.02, 0.03, 0.01], device="cuda")
        self.traj = (torch.arange(T, device="cuda") % 3).int()
        self.shift = torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, 0.05, -0.05)
        self.ws, self.head = R.new_workspace(T, V), R.new_workspace(T, V, D)
        self.ews, self.nws = R.new_embedding_workspace(T, V, D), R.new_layer_norm_workspace(T, D)
        self.d_w, self.d_ln, self.d_bias = (torch.zeros(V, D, device="cuda"), torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda"))
        self.loss = torch.zeros(1, dtype=torch.float64, device="cuda")
        self.params = R.make_params(loss_agg=R.AGG_TOKEN_SUM)

    def hidden(self):
        R = self.R
        self.x = R.rl_embedding_fwd(self.before, self.w, self.ews, scale=SCALE)
        self.h, self.mean, self.rstd = R.rl_layer_norm_fwd(self.x, weight=self.ln, bias=self.bias)
        return self.h

    def draw(self):
        """Tokens, and the log-probabilities that the loss calls old."""
        R = self.R
        logits = (self.hidden().float() @ self.w.float().T).contiguous()
        self.ids, self.rollout = R.rl_sample_tokens(logits, self.u, R.make_sample_params(1.0, 100, 0.95, 0.0), self.ws)
        self.old = self.rollout - self.shift

    def train(self):
        R = self.R
        h = self.hidden()
        d_h = R.rl_fused_head_loss_fwd_bwd(h, self.w, self.ids, self.mask, self.traj, self.adv, self.coef, self.old, self.params,
                                           self.head, self.loss, self.d_w, d_hidden_dtype=torch.bfloat16)
        d_x = R.rl_layer_norm_bwd(d_h, self.x, self.mean, self.rstd, self.nws, weight=self.ln, mask=self.mask,
                                  d_weight=self.d_ln, d_bias=self.d_bias)
        R.rl_embedding_bwd(self.before, d_x, self.d_w, self.ews, scale=SCALE)

    def checked(self):
        for ws in (self.ws, self.head, self.ews, self.nws):
            assert self.R.rl_query_status(ws)[1] == 0


def exact_loss(s, w, ln, bias):
    h, _, _ = O.layer_norm(O.embedding(s.before.cpu().numpy(), w, SCALE), ln, bias)
    P = G.LossParams(loss_agg=G.AGG_TOKEN_SUM)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    z = h @ w.T
    loss = 0.0
    for t in range(T):
        if s.mask[t]:
            lp = z[t] - z[t].max()
            lp = float(lp[int(s.ids[t])] - np.log(np.exp(lp).sum()))
            rho, A, c = np.exp(lp - float(s.old[t])), f(s.adv)[int(s.traj[t])], f(s.coef)[int(s.traj[t])]
            loss -= c * min(rho * A, np.clip(rho, 1 - P.clip_eps_low, 1 + P.clip_eps_high) * A)
    return loss


@pytest.mark.parametrize("size", [0.3, 0.04, 0.02])
def test_a_step_with_a_tied_head(R, size):
    s = Step(R, 3, size)
    s.draw()
    assert (s.ids >= 0).all() and len(set(s.ids.tolist())) > 10
    # the drawn tokens' log-probabilities are the loss's own
    again, _, _ = R.rl_fused_head_token_logprobs(s.h, s.w, s.ids, s.head)
    # (two sums of 128 products of bf16 numbers each of up to 4 in size, in other orders)
    assert (again - s.rollout).abs().max() < 1e-3
    s.train()
    s.checked()
    grads = [t.double().cpu().numpy() for t in (s.d_w, s.d_ln, s.d_bias)]
    at = [t.double().cpu().numpy() for t in (s.w, s.ln, s.bias)]
    assert abs(float(s.loss) - exact_loss(s, *at)) <= 2.0 ** -5 * float(s.coef.sum()) * T
    for k in range(3):
        n = np.linalg.norm(grads[k])
        assert n > 0
        h = 1e-4 / max(1.0, np.abs(grads[k] / n).max())
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + h * grads[k] / n, at[k] - h * grads[k] / n
        diff = (exact_loss(s, *up) - exact_loss(s, *down)) / (2 * h)
        rounding = 2.0 ** -23 * 12 * 40 * float((s.coef[s.traj.long()] * s.adv[s.traj.long()].abs()).sum())
        assert abs(diff - n) <= 2.0 ** -5 * n + rounding, (k, diff, n)
        assert size == 0.3 or n > 100 * rounding


def test_the_step_repeats_in_a_graph_and_on_another_stream(R):
    s = Step(R, 5)
    s.draw()
    s.train()
    torch.cuda.synchronize()
    first = [t.clone() for t in (s.ids, s.rollout, s.h, s.d_w, s.d_ln, s.d_bias)]

    def clear():
        for t in (s.d_w, s.d_ln, s.d_bias, s.loss):
            t.zero_()

    side = torch.cuda.Stream()
    clear()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.draw()
        s.train()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (s.ids, s.rollout, s.h, s.d_w, s.d_ln, s.d_bias)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.draw()
        s.train()
    for _ in range(2):
        clear()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (s.ids, s.rollout, s.h, s.d_w, s.d_ln, s.d_bias)))
    s.checked()


def test_two_steps_at_once(R):
    """Two programs on two streams with workspaces of their own."""
    a, b = Step(R, 7), Step(R, 8)
    alone = []
    for s in (a, b):
        s.draw()
        s.train()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (s.ids, s.d_w, s.d_ln)])
        for t in (s.d_w, s.d_ln, s.d_bias, s.loss):
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, st in zip((a, b), streams):
        with torch.cuda.stream(st):
            s.draw()
            s.train()
    torch.cuda.synchronize()
    for s, ref in zip((a, b), alone):
        assert all(torch.equal(x, y) for x, y in zip(ref, (s.ids, s.d_w, s.d_ln)))
        s.checked()
