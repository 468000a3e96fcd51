"""One policy-gradient step through a replayed MoE layer, forward and backward, on one GPU.

    python examples/replay_policy_step.py

The trainer's second evaluation of the rollout's tokens (Router Replay, section 2.4.4): the layer runs from the routing log, its output
joins the residual stream, is normalised and coded for the FP8 head, and the clipped policy loss is taken on the head's logits.  Then
everything is walked back to the tokens, the experts' matrices, the router, the norm's gain and the head.

Router Replay comes in two forms.  With a router, the log's expert ids are replayed and the gates are this policy's own, a softmax over its logits of those
experts: they depend on the tokens and on the router, and the gradient goes on into both.  Without one, the logged gates are replayed too and are constants;
`drouter` is then the gradient that logits behind such gates would receive, and goes no further.

The 8-bit activations that the forward pass made are the checkpoints of the backward pass: no activation is kept in bf16 but the
norm's input.  SwiGLU's own derivative, which is elementwise, and the router's two products are written in torch here; SwiGLU's and the gate and up
projections that it needs are recomputed from the codes, expert by expert, for which the experts' bounds come to the host: that, and the layer's
`hidden()`, which waits for its copies, are what a captured graph could not take.
"""
from __future__ import annotations

import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2512_07710_amd as moe  # noqa: E402

BLOCK = 128
EPS = 1e-6
LOSS = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.02, entropy_coef=0.001, temperature=1.0)


def values(codes, scales, rows_per_block):
    """What e4m3 codes and their scales stand for, in fp32.  rows_per_block 1: activations, scales [cols/128, rows]; 128: weights."""
    v = codes.view(torch.float8_e4m3fn).float()
    if rows_per_block == 1:
        return (v.unflatten(-1, (-1, BLOCK)) * scales.t()[:, :, None]).flatten(-2)
    return v * scales.repeat_interleave(BLOCK, -2).repeat_interleave(BLOCK, -1)


class ReplayPolicyStep:
    """Buffers and calls of one step: T tokens, a layer (d, E, k, F) and a head of V logits."""

    def __init__(self, T, d, E, k, F, V, device="cuda:0"):
        self.T, self.d, self.E, self.k, self.F, self.V = T, d, E, k, F, V
        self.wide = (V + BLOCK - 1) // BLOCK * BLOCK           # the head's rows come in blocks of 128
        self.layer = moe.MoELayer(T, d, E, k, F, device)
        self.ctx = self.layer.ctx
        moe.moe_reserve_gradients(self.ctx)
        new = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device=device)  # noqa: E731
        b16, u8, N = torch.bfloat16, torch.uint8, T * k
        self.h, self.n_q, self.n_s, self.rstd = new(T, d, t=b16), new(T, d, t=u8), new(d // BLOCK, T), new(T)
        self.logits, self.dlogits = new(T, self.wide), torch.zeros((T, self.wide), dtype=b16, device=device)
        self.logp, self.entropy, self.row_loss, self.loss = new(T), new(T), new(T), new(1)
        self.dn, self.dh, self.dgain = new(T, d, t=b16), new(T, d, t=b16), new(d)
        self.dhead = new(self.wide, d)
        self.dy_perm, self.dgate, self.drouter = new(N, d, t=b16), new(T, k), new(T, E)
        self.dhidden, self.dW2 = new(N, F, t=b16), new(E, d, F)
        self.x_perm, self.xq, self.xs = new(N, d, t=b16), new(N, d, t=u8), new(d // BLOCK, N)
        self.dx_gate, self.dx_up, self.dx = new(N, d, t=b16), new(N, d, t=b16), new(T, d, t=b16)
        self.dW_router = new(E, d)
        self.dW1, self.dW3 = new(E, F, d), new(E, F, d)

    def close(self):
        self.layer.close()

    def forward(self, x, log_ids, log_w, w, gain, head_q, head_s, batch, router=None):
        """The loss [1] of this batch: target, old_logp, ref_logp, advantage, weight.  router [E, d]: log_w is not read, the gates are computed."""
        L, c = self.layer, self.ctx
        if router is None:
            y = L.forward_replay(x, log_ids, log_w, w)
        else:
            L.route_replay_ids(x, router, log_ids)
            L.quantize_tokens(x)
            L.expert_ffn_gather(w)
            L.combine()
            y = L.y
        moe.moe_add_rmsnorm(c, y, x, gain, EPS, sum=self.h, q=self.n_q, scales=self.n_s, rstd=self.rstd)
        moe.moe_linear_fp8(c, self.n_q, self.n_s, self.T, self.d, head_q, head_s, self.wide, self.logits)
        moe.moe_policy_loss(c, self.logits[:, :self.V], batch["target"], batch["old_logp"], batch["ref_logp"], batch["advantage"], batch["weight"],
                            self.logp, self.entropy, self.row_loss, self.loss, self.dlogits[:, :self.V], **LOSS)
        return self.loss

    def backward(self, x, w, gain, head_q, head_s, router=None):
        """Gradients of the last forward pass, in this object's buffers: dx, dW1, dW3, dW2, drouter, dgain, dhead, and with the forward pass's router
        dW_router."""
        L, c = self.layer, self.ctx
        moe.moe_linear_fp8_dgrad(c, self.dlogits, head_q, head_s, None, self.dn)
        moe.moe_linear_fp8_wgrad(c, self.dlogits, self.n_q, self.n_s, None, self.dhead)
        moe.moe_add_rmsnorm_backward(c, self.dn, self.h, self.rstd, gain, None, self.dh, self.dgain)
        moe.moe_combine_backward(c, self.dh, L.y_perm, L.inv_perm, L.topk_w, L.topk_idx, self.dy_perm, self.dgate, self.drouter)
        hq, hs = L.hidden()
        moe.moe_linear_fp8_dgrad(c, self.dy_perm, w["W2q"], w["s2"], L.offsets, self.dhidden)
        moe.moe_linear_fp8_wgrad(c, self.dy_perm, hq, hs, L.offsets, self.dW2)
        # the experts' inputs again, in their order: the same codes that the layer's gate and up projections read
        moe.moe_dispatch(c, x, L.inv_perm, self.x_perm)
        moe.moe_quantize_fp8(c, self.x_perm, self.T * self.k, self.d, BLOCK, None, 1, self.xq, self.xs)
        dg, du = self._swiglu_backward(w, L.offsets.tolist())
        moe.moe_linear_fp8_dgrad(c, dg, w["W1q"], w["s1"], L.offsets, self.dx_gate)
        moe.moe_linear_fp8_dgrad(c, du, w["W3q"], w["s3"], L.offsets, self.dx_up)
        moe.moe_linear_fp8_wgrad(c, dg, self.xq, self.xs, L.offsets, self.dW1)
        moe.moe_linear_fp8_wgrad(c, du, self.xq, self.xs, L.offsets, self.dW3)
        beside = self.dh                                       # the residual's own way
        if router is not None:                                 # and the gates'
            beside = (self.dh.float() + self.drouter @ router).to(torch.bfloat16)
            torch.matmul(self.drouter.t(), x.float(), out=self.dW_router)
        moe.moe_dispatch_backward(c, self.dx_gate.add_(self.dx_up), L.inv_perm, beside, self.dx)
        return self.dx

    def _swiglu_backward(self, w, bounds):
        x = values(self.xq, self.xs, 1)
        dg, du = torch.zeros_like(self.dhidden), torch.zeros_like(self.dhidden)
        for e in range(self.E):
            at = slice(bounds[e], bounds[e + 1])
            g = x[at] @ values(w["W1q"][e], w["s1"][e], BLOCK).t()
            u = x[at] @ values(w["W3q"][e], w["s3"][e], BLOCK).t()
            s, dh = torch.sigmoid(g), self.dhidden[at].float()
            dg[at] = (dh * u * (s + g * s * (1 - s))).to(torch.bfloat16)
            du[at] = (dh * g * s).to(torch.bfloat16)
        return dg, du


def make_batch(T, d, E, k, F, V, seed=0, device="cuda:0"):
    """Random tokens, log, weights (coded by the library's own weight quantisation) and rollout statistics."""
    g = torch.Generator(device=device).manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
    x = randn(T, d).to(torch.bfloat16)
    ids = torch.topk(randn(T, E), k, dim=1).indices.to(torch.int32).contiguous()
    log_w = torch.softmax(randn(T, k), dim=1).contiguous()
    ctx = moe.moe_create(0, d, E, k, F)

    def coded(rows, cols, std, *lead):
        w = (randn(*lead, rows, cols) * std).to(torch.bfloat16)
        q = torch.empty(w.shape, dtype=torch.uint8, device=device)
        s = torch.empty((*lead, rows // BLOCK, cols // BLOCK), device=device)
        moe.moe_quantize_weights_fp8(ctx, w, w.numel() // cols, cols, q, s)
        return q, s
    w = {}
    w["W1q"], w["s1"] = coded(F, d, d ** -0.5, E)
    w["W3q"], w["s3"] = coded(F, d, d ** -0.5, E)
    w["W2q"], w["s2"] = coded(d, F, F ** -0.5, E)
    head_q, head_s = coded((V + BLOCK - 1) // BLOCK * BLOCK, d, 2 * d ** -0.5)
    torch.cuda.synchronize()
    moe.moe_destroy(ctx)
    gain = 1 + 0.2 * randn(d)
    weight = (torch.rand(T, generator=g, device=device) > 0.2).float()
    guess = -float(torch.log(torch.tensor(float(V))))
    batch = dict(target=torch.randint(0, V, (T,), generator=g, device=device, dtype=torch.int32), old_logp=guess + randn(T),
                 ref_logp=guess + randn(T), advantage=randn(T), weight=weight / weight.sum())
    return x, ids, log_w, w, gain, head_q, head_s, batch


def main():
    T, d, E, k, F, V = 512, 1024, 16, 4, 512, 4000
    x, ids, log_w, w, gain, head_q, head_s, batch = make_batch(T, d, E, k, F, V)
    step = ReplayPolicyStep(T, d, E, k, F, V)
    # the rollout's log: ids of its own router, which the present one has moved away from
    router = torch.randn(E, d, generator=torch.Generator(device=x.device).manual_seed(1), device=x.device) * 2 * d ** -0.5
    step.layer.route(x, router, None)
    ids, router = step.layer.topk_idx.clone(), router + 0.02 * torch.randn_like(router)
    # its log-probabilities: the old policy is the present one, the reference near it
    step.forward(x, ids, None, w, gain, head_q, head_s, batch, router)
    batch["old_logp"] = step.logp.clone()
    batch["ref_logp"] = step.logp + 0.1 * torch.randn_like(step.logp)
    loss = step.forward(x, ids, None, w, gain, head_q, head_s, batch, router).clone()
    step.backward(x, w, gain, head_q, head_s, router)
    torch.cuda.synchronize()
    print(f"loss {float(loss):.6f}, mean log-probability {float(step.logp.mean()):.4f}, mean entropy {float(step.entropy.mean()):.4f}")
    for name in ("dx", "dW1", "dW3", "dW2", "drouter", "dW_router", "dgain", "dhead"):
        print(f"  |{name}| = {float(getattr(step, name).float().norm()):.4e}")
    step.close()


if __name__ == "__main__":
    main()
