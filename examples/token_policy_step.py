"""A policy step from token ids to clipped gradients, on one GPU: both ends around examples/replay_policy_step.py.

    python examples/token_policy_step.py

Rollout: `score` embeds the batch's tokens, evaluates the layer and the head, and logs of each next token what the trainer will need: its log-probability, the
policy's entropy and the most likely alternatives.  Trainer: `train` evaluates the same tokens from the routing log (Router Replay, section 2.4.4), takes the policy
loss against the logged log-probabilities, walks back to the embedding table, and scales all gradients down to a largest norm, as the optimizer will take them.
"""
from __future__ import annotations

import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)

import replay_policy_step as replay  # noqa: E402
from replay_policy_step import moe  # noqa: E402


class TokenPolicyStep:
    """Buffers and calls of one step: T tokens of a vocabulary of V, a layer (d, E, k, F); `top` alternatives are logged."""

    def __init__(self, T, d, E, k, F, V, top=8, device="cuda:0"):
        self.step = step = replay.ReplayPolicyStep(T, d, E, k, F, V, device)
        self.V, self.ctx, self.scale = V, step.ctx, d ** 0.5
        new = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device=device)  # noqa: E731
        self.x, self.dtable = new(T, d, t=torch.bfloat16), new(V, d)
        self.logp, self.entropy, self.top_idx, self.top_logp = new(T), new(T), new(T, top, t=torch.int32), new(T, top)
        self.sum_sq, self.norm = new(1, t=torch.float64), new(1)
        # the buffers stay where they are: their list is made once
        self.grads = moe.GradList([step.dW1, step.dW3, step.dW2, step.dgain, step.dhead, self.dtable])

    def close(self):
        self.step.close()

    def score(self, ids, next_ids, table, log_ids, log_w, w, gain, head_q, head_s, temperature=1.0):
        """(log-probability of next_ids, entropy, alternatives and theirs), of rows without a next token (an id outside the vocabulary) the latter three."""
        s, c = self.step, self.ctx
        moe.moe_embed(c, ids, table, self.scale, self.x)
        y = s.layer.forward_replay(self.x, log_ids, log_w, w)
        moe.moe_add_rmsnorm(c, y, self.x, gain, replay.EPS, sum=s.h, q=s.n_q, scales=s.n_s, rstd=s.rstd)
        moe.moe_linear_fp8(c, s.n_q, s.n_s, s.T, s.d, head_q, head_s, s.wide, s.logits)
        moe.moe_token_logp(c, s.logits[:, :self.V], next_ids, self.logp, self.entropy, self.top_idx, self.top_logp, temperature=temperature)
        return self.logp, self.entropy, self.top_idx, self.top_logp

    def train(self, ids, table, log_ids, log_w, w, gain, head_q, head_s, batch, max_norm):
        """The loss; all gradients, scaled down where their norm is above max_norm, are in the step's buffers and dtable."""
        s, c = self.step, self.ctx
        moe.moe_embed(c, ids, table, self.scale, self.x)
        loss = s.forward(self.x, log_ids, log_w, w, gain, head_q, head_s, batch)
        dx = s.backward(self.x, w, gain, head_q, head_s)
        moe.moe_embed_backward(c, dx, ids, self.scale, self.dtable)
        moe.moe_grad_norm(c, self.grads, self.sum_sq, self.norm)
        moe.moe_clip_grads(c, self.grads, self.sum_sq, max_norm)
        return loss


def main():
    T, d, E, k, F, V = 512, 1024, 16, 4, 512, 4000
    _, log_ids, log_w, w, gain, head_q, head_s, batch = replay.make_batch(T, d, E, k, F, V)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    table = (torch.randn((V, d), generator=g, device="cuda:0") * d ** -0.5).to(torch.bfloat16)
    tokens = torch.randint(0, V, (T + 1,), generator=g, device="cuda:0", dtype=torch.int32)
    ids, batch["target"] = tokens[:-1].contiguous(), tokens[1:].contiguous()
    step = TokenPolicyStep(T, d, E, k, F, V)
    args = (table, log_ids, log_w, w, gain, head_q, head_s)
    logp, entropy, top_idx, _ = step.score(ids, batch["target"], *args)
    batch["old_logp"] = batch["ref_logp"] = logp.clone()
    print(f"mean log-probability {float(logp.mean()):.4f}, mean entropy {float(entropy.mean()):.4f}, first alternatives {top_idx[0].tolist()}")
    loss = step.train(ids, *args, batch, max_norm=1.0)
    torch.cuda.synchronize()
    print(f"loss {float(loss):.6f}, norm of the gradients {float(step.norm):.4e}")
    step.close()


if __name__ == "__main__":
    main()
