"""One policy step with the gates of the policy's own router on replayed ids (examples/replay_policy_step.py): the gradient goes through the gates into the
router and the tokens, against torch's own differentiation of the same step on the values that the codes stand for."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import replay_policy_step
    return replay_policy_step


def _reference(ex, step, x, ids, w, gain, head_q, head_s, batch, router):
    """Gradients by torch in fp32; where the forward pass codes or rounds, the coded value with the gradient passed straight through"""
    T, E, k, V = step.T, step.E, step.k, step.V
    through = lambda v, coded: v + (coded - v).detach()  # noqa: E731
    X, R = x.float().requires_grad_(), router.clone().requires_grad_()
    W = {n: ex.values(w[n + "q"], w["s" + n[1]], 128).requires_grad_() for n in ("W1", "W3", "W2")}
    head, G = ex.values(head_q, head_s, 128).requires_grad_(), gain.clone().requires_grad_()
    logits = X @ R.t()
    logits.retain_grad()
    gates = torch.softmax(logits.gather(1, ids.long()), dim=1)
    assert (gates - step.layer.topk_w).abs().max() <= 1e-5
    hq, hs = step.layer.hidden()
    hidden, codes_x = ex.values(hq, hs, 1), ex.values(step.xq, step.xs, 1)                     # in expert order
    inv = step.layer.inv_perm.long().view(T, k)
    y = torch.zeros_like(X)
    for e in range(E):
        for j in range(k):
            t = (ids[:, j] == e).nonzero()[:, 0]
            p = inv[t, j]
            xe = through(X[t], codes_x[p])
            h = through(torch.nn.functional.silu(xe @ W["W1"][e].t()) * (xe @ W["W3"][e].t()), hidden[p])
            y = y.index_add(0, t, gates[t, j][:, None] * (h @ W["W2"][e].t()))
    h = through(y + X, step.h.float())
    n = through(h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + ex.EPS) * G, ex.values(step.n_q, step.n_s, 1))
    z = through(n @ head[:V].t(), step.logits[:, :V])
    logp = torch.log_softmax(z / ex.LOSS["temperature"], dim=1)
    lp = logp.gather(1, batch["target"].long()[:, None])[:, 0]
    H = -(logp.exp() * logp).sum(dim=1)
    A, r, q = batch["advantage"], torch.exp(lp - batch["old_logp"]), batch["ref_logp"] - lp
    pg = -torch.minimum(r * A, r.clamp(1 - ex.LOSS["clip_low"], 1 + ex.LOSS["clip_high"]) * A)
    loss = (batch["weight"] * (pg + ex.LOSS["kl_coef"] * (torch.exp(q) - q - 1) - ex.LOSS["entropy_coef"] * H)).sum()
    loss.backward()
    return loss.detach(), dict(dx=X.grad, dW1=W["W1"].grad, dW3=W["W3"].grad, dW2=W["W2"].grad, drouter=logits.grad, dW_router=R.grad, dgain=G.grad,
                               dhead=head.grad)


@pytest.mark.parametrize("shape", [(96, 256, 8, 2, 256, 1000), (130, 384, 12, 3, 128, 517)], ids=str)
def test_step_with_the_routers_own_gates(gpu_lib, example, shape):
    T, d, E = shape[:3]
    x, ids, _, w, gain, head_q, head_s, batch = example.make_batch(*shape, seed=4)
    router = torch.randn(E, d, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * 4 * d ** -0.5
    step = example.ReplayPolicyStep(*shape)
    try:
        step.forward(x, ids, None, w, gain, head_q, head_s, batch, router)
        batch["old_logp"] = step.logp + 0.05 * torch.randn_like(step.logp)
        loss = step.forward(x, ids, None, w, gain, head_q, head_s, batch, router).clone()
        step.backward(x, w, gain, head_q, head_s, router)
        torch.cuda.synchronize()
        want, grads = _reference(example, step, x, ids, w, gain, head_q, head_s, batch, router)
        assert abs(float(loss[0]) - float(want)) <= 1e-4 * (1 + abs(float(want)))
        # a chain of at most seven arrays rounded to bf16 (2^-8 of a value at most, 0.4 of that in the mean square), errors that add up in squares
        limit = 7 ** 0.5 * 2.0 ** -8
        for name, g in grads.items():
            rel = float((getattr(step, name).float() - g).norm() / g.norm())
            assert rel <= limit, (name, rel)
        # the gates' part of dx is no small one: without it the check above would have failed
        assert float((grads["drouter"] @ router).norm() / grads["dx"].norm()) > 3 * limit
    finally:
        step.close()


def test_the_example_runs(gpu_lib, example, capsys):
    example.main()
    out = capsys.readouterr().out
    assert "dW_router" in out and "nan" not in out
