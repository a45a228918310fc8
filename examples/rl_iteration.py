"""Iterations of RL on a toy policy, with the library on both sides of the loss.

The policy sees the last token only: hidden = tanh(embedding[token] W1^T), logits = hidden W^T. A smaller
model (the policy's own matrices as they were at the start) drafts ``DRAFTED`` tokens at a time,
``rl_verify_drafts`` accepts or replaces them by the policy's probabilities, and the log-probabilities it
emits are the rollout's. The reward is the share of tokens from the lower half of the vocabulary. Then
group advantages, the loss through the fused head with the truncated importance weight against the rollout's
log-probabilities, and ``rl_muon_update`` on both matrices, W in fp32 with the bf16 copy that the next
iteration's products read.

    python examples/rl_iteration.py
"""

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_16798_gb300.rl_loss as R  # noqa: E402

VOCAB, HIDDEN, PROMPTS, GROUP, TOKENS, DRAFTED = 1000, 128, 4, 16, 24, 3


def hidden_of(tokens, embedding, w1):
    return torch.tanh(embedding[tokens.long()].float() @ w1.float().T).bfloat16()


def rollout(policy, drafter, embedding, start, g):
    """(tokens before and at each place, their rollout log-probabilities), [sequences, TOKENS] each, and the
    share of drafted tokens that were accepted."""
    n, dev = start.numel(), start.device
    tokens = torch.full((n, TOKENS + DRAFTED + 1), -1, dtype=torch.int32, device=dev)
    logp = torch.zeros(n, TOKENS + DRAFTED + 1, device=dev)
    at, last, accepted, drafted = torch.zeros(n, dtype=torch.int64, device=dev), start.clone(), 0, 0
    one, params = R.make_verify_params(1.0), R.make_verify_params(1.0)
    no_offsets = torch.zeros(n + 1, dtype=torch.int32, device=dev)
    offsets = torch.arange(0, n * DRAFTED + 1, DRAFTED, dtype=torch.int32, device=dev)
    none_i, none_f = torch.empty(0, dtype=torch.int32, device=dev), torch.empty(0, device=dev)
    ws = R.new_workspace(n * (DRAFTED + 1), VOCAB, device=dev)
    while int(at.min()) < TOKENS:
        # the drafter's tokens, one draw after the other
        ids = torch.empty(n, DRAFTED, dtype=torch.int32, device=dev)
        draft = torch.empty(n, DRAFTED, VOCAB, dtype=torch.bfloat16, device=dev)
        prev = last
        for j in range(DRAFTED):
            draft[:, j] = hidden_of(prev, embedding, drafter[0]) @ drafter[1].T
            z = draft[:, j].contiguous()
            prev, _, _ = R.rl_verify_drafts(z, none_i, no_offsets, none_f, torch.rand(n, generator=g, device=dev), 0, one, ws)
            ids[:, j] = prev
        # the policy's rows at all places at once
        before = torch.cat([last[:, None], ids], 1).reshape(-1)
        target = hidden_of(before, embedding, policy[0]) @ policy[1].T
        out, acc, lp = R.rl_verify_drafts(target, ids.reshape(-1), offsets,
                                          torch.rand(n * DRAFTED, generator=g, device=dev),
                                          torch.rand(n, generator=g, device=dev), DRAFTED, params, ws,
                                          draft_logits=draft.view(-1, VOCAB))
        if R.rl_query_status(ws)[1]:
            raise RuntimeError("a device check failed in the verification")
        out, lp, acc = out.view(n, -1), lp.view(n, -1), acc.long()
        accepted, drafted = accepted + int(acc.sum()), drafted + n * DRAFTED
        for j in range(DRAFTED + 1):
            on = (j <= acc) & (at + j < tokens.shape[1])
            tokens[on, (at + j)[on]] = out[on, j]
            logp[on, (at + j)[on]] = lp[on, j]
        last = out.gather(1, acc[:, None])[:, 0].contiguous()
        at = at + acc + 1
    tokens = tokens[:, :TOKENS].contiguous()
    before = torch.cat([start[:, None], tokens[:, :-1]], 1)
    return before, tokens, logp[:, :TOKENS].contiguous(), accepted / drafted


def train(iterations=12, seed=0, device="cuda"):
    """The mean reward of each iteration, and the share of drafted tokens accepted in it."""
    g = torch.Generator(device=device).manual_seed(seed)
    n = PROMPTS * GROUP
    embedding = torch.randn(VOCAB, HIDDEN, generator=g, device=device).bfloat16()
    w1 = torch.randn(HIDDEN, HIDDEN, generator=g, device=device) / math.sqrt(HIDDEN)
    head = torch.randn(VOCAB, HIDDEN, generator=g, device=device) * (1.5 / math.sqrt(HIDDEN))
    copies = [w1.bfloat16(), head.bfloat16()]
    drafter = [w1.bfloat16().clone(), head.bfloat16().clone()]
    momenta = [torch.zeros_like(w1), torch.zeros_like(head)]
    spaces = [R.new_muon_workspace(1, *w.shape) for w in (w1, head)]
    steps = [R.make_muon_params(lr=lr, momentum=0.9, update_scale=0.2 * math.sqrt(max(w.shape)))
             for lr, w in ((0.05, w1), (0.15, head))]
    group_offsets = torch.arange(0, n + 1, GROUP, dtype=torch.int32, device=device)
    traj_offsets = torch.arange(0, n * TOKENS + 1, TOKENS, dtype=torch.int64, device=device)
    mask = torch.ones(n * TOKENS, dtype=torch.uint8, device=device)
    params = R.make_params(tis_cap=2.0)
    ws = R.new_workspace(n * TOKENS, VOCAB, HIDDEN, device=device)
    rewards_seen, accepted_seen = [], []
    for _ in range(iterations):
        start = torch.randint(0, VOCAB, (PROMPTS,), generator=g, device=device, dtype=torch.int32).repeat_interleave(GROUP)
        before, tokens, rollout_logp, accepted = rollout(copies, drafter, embedding, start, g)
        rewards = (tokens < VOCAB // 2).float().mean(1)
        rewards_seen.append(float(rewards.mean()))
        accepted_seen.append(accepted)
        # the policy gradient through the head
        adv, coef, _, owner = R.rl_group_advantages(group_offsets, rewards, traj_offsets, mask, params, ws)
        ids, h = tokens.reshape(-1), hidden_of(before.reshape(-1), embedding, copies[0])
        old_logp, _, _ = R.rl_fused_head_token_logprobs(h, copies[1], ids, ws)
        loss = torch.zeros(1, dtype=torch.float64, device=device)
        d_head = torch.zeros(VOCAB, HIDDEN, device=device)
        d_h = R.rl_fused_head_loss_fwd_bwd(h, copies[1], ids, mask, owner, adv, coef, old_logp, params, ws, loss, d_head,
                                           d_hidden_dtype=torch.float32, rollout_logp=rollout_logp.reshape(-1))
        d_pre = d_h * (1.0 - h.float() ** 2)
        d_w1 = d_pre.T @ embedding[before.reshape(-1).long()].float()
        # the updates
        for k, (w, grad) in enumerate(((w1, d_w1), (head, d_head))):
            R.rl_muon_update(grad.contiguous(), steps[k], spaces[k], momentum=momenta[k], weights=w, weights_bf16=copies[k])
            if R.rl_query_status(spaces[k])[1]:
                raise RuntimeError("a device check failed in the update")
        if R.rl_query_status(ws)[1]:
            raise RuntimeError("a device check failed in the loss")
    return rewards_seen, accepted_seen


if __name__ == "__main__":
    for i, (r, a) in enumerate(zip(*train())):
        print(f"iteration {i}: mean reward {r:.3f}, {100 * a:.0f}% of the drafted tokens accepted")
