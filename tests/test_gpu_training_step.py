"""One policy step through a replayed layer (examples/replay_policy_step.py) against torch's own differentiation in fp32 of the same step on the
values that the codes stand for (and on the head's logits as moe_linear_fp8 summed them), and the operators inside captured graphs and on streams of the caller's."""
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


def _reference(ex, step, x, ids, log_w, w, gain, head_q, head_s, batch):
    """Gradients by torch in fp32; where the forward pass codes or rounds, the coded value with the gradient passed straight through"""
    T, d, E, k, V = step.T, step.d, step.E, step.k, step.V
    through = lambda v, coded: v + (coded - v).detach()  # noqa: E731
    X = x.float().requires_grad_()
    W = {n: ex.values(w[n + "q"], w["s" + n[1]], 128).requires_grad_() for n in ("W1", "W3", "W2")}
    head, G = ex.values(head_q, head_s, 128).requires_grad_(), gain.clone().requires_grad_()
    raw = torch.log(log_w).requires_grad_()                   # softmax over the chosen logits gives the logged weights
    gates = torch.softmax(raw, dim=1)
    hq, hs = step.layer.hidden()
    hidden = ex.values(hq, hs, 1)                              # in expert order
    inv = step.layer.inv_perm.long().view(T, k)
    codes_x = ex.values(step.xq, step.xs, 1)
    y = torch.zeros((T, d), device=x.device)
    for e in range(E):
        for j in range(k):
            t = (ids[:, j] == e).nonzero()[:, 0]
            p = inv[t, j]
            xe = through(X[t], codes_x[p])
            h = torch.nn.functional.silu(xe @ W["W1"][e].t()) * (xe @ W["W3"][e].t())
            h = through(h, hidden[p])
            y = y.index_add(0, t, gates[t, j][:, None] * (h @ W["W2"][e].t()))
    h = through(y + X, step.h.float())
    n = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + ex.EPS) * G
    n = through(n, ex.values(step.n_q, step.n_s, 1))
    z = through(n @ head[:V].t(), step.logits[:, :V])         # the FP8 product's own sums
    logp = torch.log_softmax(z / ex.LOSS["temperature"], dim=1)
    lp = logp.gather(1, batch["target"].long()[:, None])[:, 0]
    H = -(logp.exp() * logp).sum(dim=1)
    A, r, z = batch["advantage"], torch.exp(lp - batch["old_logp"]), batch["ref_logp"] - lp
    pg = -torch.minimum(r * A, r.clamp(1 - ex.LOSS["clip_low"], 1 + ex.LOSS["clip_high"]) * A)
    loss = (batch["weight"] * (pg + ex.LOSS["kl_coef"] * (torch.exp(z) - z - 1) - ex.LOSS["entropy_coef"] * H)).sum()
    loss.backward()
    router = torch.zeros((T, E), device=x.device).scatter_add_(1, ids.long(), raw.grad)
    return loss.detach(), dict(dx=X.grad, dW1=W["W1"].grad, dW3=W["W3"].grad, dW2=W["W2"].grad, drouter=router, dgain=G.grad, dhead=head.grad), lp.detach()


@pytest.mark.parametrize("shape", [(96, 256, 8, 2, 256, 1000), (130, 384, 12, 3, 128, 517)], ids=str)
def test_step_against_autograd(gpu_lib, example, shape):
    x, ids, log_w, w, gain, head_q, head_s, batch = example.make_batch(*shape, seed=3)
    step = example.ReplayPolicyStep(*shape)
    try:
        step.forward(x, ids, log_w, w, gain, head_q, head_s, batch)
        batch["old_logp"] = step.logp + 0.05 * torch.randn_like(step.logp)
        loss = step.forward(x, ids, log_w, w, gain, head_q, head_s, batch).clone()
        step.backward(x, w, gain, head_q, head_s)
        torch.cuda.synchronize()
        want, grads, lp = _reference(example, step, x, ids, log_w, w, gain, head_q, head_s, batch)
        assert (step.logp - lp).abs().max() <= 1e-4
        assert abs(float(loss[0]) - float(want)) <= 1e-4 * (1 + abs(float(want)))
        for name, g in grads.items():
            got = getattr(step, name).float()
            # a chain of at most six arrays rounded to bf16 (2^-8 of a value at most, 0.4 of that in the mean square), errors that add up in squares
            rel = float((got - g).norm() / g.norm())
            assert rel <= 6 ** 0.5 * 2.0 ** -8, (name, rel)
    finally:
        step.close()


def test_backward_calls_in_a_captured_graph(gpu_lib, example):
    """No call allocates or synchronises: a captured forward and backward replays to the same bits, several times, between other work."""
    shape = (64, 256, 8, 2, 256, 1000)
    x, ids, log_w, w, gain, head_q, head_s, batch = example.make_batch(*shape, seed=5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step = example.ReplayPolicyStep(*shape)
        c, L = step.ctx, step.layer

        def calls():
            step.forward(x, ids, log_w, w, gain, head_q, head_s, batch)
            gpu_lib.moe_linear_fp8_dgrad(c, step.dlogits, head_q, head_s, None, step.dn)
            gpu_lib.moe_linear_fp8_wgrad(c, step.dlogits, step.n_q, step.n_s, None, step.dhead)
            gpu_lib.moe_add_rmsnorm_backward(c, step.dn, step.h, step.rstd, gain, None, step.dh, step.dgain)
            gpu_lib.moe_combine_backward(c, step.dh, L.y_perm, L.inv_perm, L.topk_w, L.topk_idx, step.dy_perm, step.dgate, step.drouter)
            gpu_lib.moe_linear_fp8_dgrad(c, step.dy_perm, w["W2q"], w["s2"], L.offsets, step.dhidden)
            gpu_lib.moe_dispatch(c, x, L.inv_perm, step.x_perm)
            gpu_lib.moe_dispatch_backward(c, step.x_perm, L.inv_perm, step.dh, step.dx)
        names = ("loss", "logp", "dlogits", "dn", "dhead", "dh", "dgain", "dy_perm", "dgate", "drouter", "dhidden", "x_perm", "dx")
        calls()
        stream.synchronize()
        want = {n: getattr(step, n).clone() for n in names}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls()
        for turn in range(3):
            for n in names:
                getattr(step, n).fill_(7)
            step.dlogits[:, step.V:] = 0
            graph.replay()
            stream.synchronize()
            for n in names:
                assert torch.equal(getattr(step, n), want[n]), (turn, n)
            calls()                                            # eager work in between
            stream.synchronize()
            assert torch.equal(step.dx, want["dx"])
        step.close()


def test_reserving_twice_and_contexts_side_by_side(gpu_lib):
    """A context's workspace is its own: two contexts on two streams do not disturb each other."""
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    ctxs = []
    for s in (a, b):
        c = gpu_lib.moe_create(0, 128, 1, 1, 128, s)
        gpu_lib.moe_reserve_gradients(c)
        gpu_lib.moe_reserve_gradients(c)
        ctxs.append(c)
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = [torch.randn((300, 1024), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    h = [torch.randn((300, 1024), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    gain, rstd = torch.ones(1024, device="cuda"), torch.ones(300, device="cuda")
    out = [(torch.empty_like(h[0]), torch.empty(1024, device="cuda")) for _ in range(4)]
    torch.cuda.synchronize()
    for i in (0, 1):
        gpu_lib.moe_add_rmsnorm_backward(ctxs[i], dy[i], h[i], rstd, gain, None, *out[i])
        torch.cuda.synchronize()
    for _ in range(20):
        for i in (0, 1):
            gpu_lib.moe_add_rmsnorm_backward(ctxs[i], dy[i], h[i], rstd, gain, None, *out[2 + i])
    torch.cuda.synchronize()
    for i in (0, 1):
        assert torch.equal(out[i][0], out[2 + i][0]) and torch.equal(out[i][1], out[2 + i][1])
        gpu_lib.moe_destroy(ctxs[i])
