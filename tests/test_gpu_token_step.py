"""A policy step from token ids to clipped gradients (examples/token_policy_step.py), and its two ends together: in captured graphs, on streams of the caller's,
with other work on the same workspace in between."""
import os
import sys

import pytest
import torch

from test_gpu_training_step import _reference
from training_common import F32

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import token_policy_step
    return token_policy_step


@pytest.mark.parametrize("shape", [(96, 256, 8, 2, 256, 1000), (130, 384, 12, 3, 128, 517)], ids=str)
def test_step(gpu_lib, example, shape):
    T, d, E, k, F, V = shape
    ex = example.replay
    _, log_ids, log_w, w, gain, head_q, head_s, batch = ex.make_batch(*shape, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    table = (torch.randn((V, d), generator=g, device="cuda") * d ** -0.5).to(torch.bfloat16)
    ids = torch.randint(0, V // 8, (T,), generator=g, device="cuda", dtype=torch.int32)    # tokens come again
    s = example.TokenPolicyStep(*shape)
    try:
        args = (table, log_ids, log_w, w, gain, head_q, head_s)
        logp, H, top_idx, top_logp = s.score(ids, batch["target"], *args)
        z = torch.log_softmax(s.step.logits[:, :V].double(), dim=1)
        # fp32 sums over at most 1000 logits, exponents of at most 40: see the operator's own tests
        bound = 300 * F32 * (1 + z.gather(1, batch["target"].long()[:, None])[:, 0].abs())
        assert ((logp.double() - z.gather(1, batch["target"].long()[:, None])[:, 0]).abs() <= bound).all()
        assert ((H.double() + (z.exp() * z).sum(dim=1)).abs() <= 1000 * F32 * (1 + H)).all()
        assert torch.equal(top_idx.long(), torch.sort(s.step.logits[:, :V], dim=1, descending=True, stable=True).indices[:, :8])
        batch["old_logp"] = logp + 0.05 * torch.randn_like(logp)
        loss = s.train(ids, *args, batch, max_norm=1e9)
        torch.cuda.synchronize()
        assert torch.equal(s.x, (table[ids.long()].float() * torch.tensor(d ** 0.5, device="cuda")).bfloat16())
        want, grads, _ = _reference(ex, s.step, s.x, log_ids, log_w, w, gain, head_q, head_s, batch)
        assert abs(float(loss) - float(want)) <= 1e-4 * (1 + abs(float(want)))
        dtable = torch.zeros((V, d), device="cuda").index_add_(0, ids.long(), grads["dx"] * d ** 0.5)
        # as dx itself: a chain of at most six arrays rounded to bf16
        assert float((s.dtable - dtable).norm() / dtable.norm()) <= 6 ** 0.5 * 2.0 ** -8
        whole = [t.clone() for t in s.grads.tensors]
        norm = sum(t.double().square().sum() for t in whole).sqrt()
        assert abs(float(s.norm) - float(norm)) <= 2 * F32 * float(norm)
        s.train(ids, *args, batch, max_norm=float(norm) / 4)
        for t, u in zip(s.grads.tensors, whole):
            assert ((t.double() - u.double() / 4).abs() <= 4 * F32 * u.double().abs() + 1e-38).all()
    finally:
        s.close()


class _Ends:
    """Ids to rows, logits to log-probabilities and back, rows' gradients to the table's, norm and clipping; the logits are a plain product of the rows."""

    def __init__(self, moe, T, V, d, seed, frequent=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
        self.moe, self.d = moe, d
        self.ctx = moe.moe_create(0, 128, 1, 1, 128)
        moe.moe_reserve_gradients(self.ctx)
        self.ids = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        self.ids[:frequent] = V // 3
        self.table = torch.randn((V, d), generator=g, device="cuda").bfloat16()
        self.logits = (torch.randn((T, V), generator=g, device="cuda") * 3).bfloat16()
        self.given = torch.randint(0, V, (T, 2), generator=g, device="cuda", dtype=torch.int32)
        self.dlogp, self.dH = torch.randn((T, 2), generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
        self.dx = torch.randn((T, d), generator=g, device="cuda").bfloat16()
        self.x, self.logp, self.H, self.top, self.top_logp, self.stats = new(T, d, t=torch.bfloat16), new(T, 2), new(T), new(T, 5, t=torch.int32), new(T, 5), new(T, 2)
        self.dlogits, self.dtable, self.sum_sq, self.norm = new(T, V, t=torch.bfloat16), new(V, d), new(1, t=torch.float64), new(1)
        self.many = [new(7 + i % 5).fill_(0.1) for i in range(150)]            # a list longer than a launch's arguments
        self.list = moe.GradList([self.dtable, self.dlogits, *self.many])
        self.clipped = [torch.empty_like(t) for t in self.list.tensors]
        self.outs = moe.GradList(self.clipped)

    def calls(self):
        m, c = self.moe, self.ctx
        m.moe_embed(c, self.ids, self.table, 2.0, self.x)
        m.moe_token_logp(c, self.logits, self.given, self.logp, self.H, self.top, self.top_logp, self.stats)
        m.moe_token_logp_backward(c, self.logits, self.given, self.dlogp, self.dH, self.stats, self.H, self.dlogits)
        m.moe_embed_backward(c, self.dx, self.ids, 2.0, self.dtable)
        m.moe_grad_norm(c, self.list, self.sum_sq, self.norm)
        m.moe_clip_grads(c, self.list, self.sum_sq, 1.0, self.outs)

    def outputs(self):
        return [self.x, self.logp, self.H, self.top, self.top_logp, self.stats, self.dlogits, self.dtable, self.sum_sq, self.norm, *self.clipped]

    def close(self):
        self.moe.moe_destroy(self.ctx)


@pytest.mark.parametrize("T,V,d,frequent", [(33, 3000, 256, 20), (1500, 700, 136, 900), (3, 70000, 64, 0)])
def test_captured_and_replayed(gpu_lib, T, V, d, frequent):
    """No call allocates or synchronises; a replay gives the eager calls' bits, several times, between other calls on the same workspace."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        e = _Ends(gpu_lib, T, V, d, 1, frequent)
        e.calls()
        stream.synchronize()
        want = [t.clone() for t in e.outputs()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            e.calls()
        other = torch.empty((V, d), device="cuda")
        for turn in range(3):
            for t in e.outputs():
                t.fill_(7)
            graph.replay()
            stream.synchronize()
            for a, b in zip(e.outputs(), want):
                assert torch.equal(a, b), turn
            gpu_lib.moe_embed_backward(e.ctx, e.dx, e.ids.flip(0), 1.0, other)             # eager work on the same workspace
            e.calls()
            stream.synchronize()
            for a, b in zip(e.outputs(), want):
                assert torch.equal(a, b), turn
        # inputs are read again in every replay
        e.ids.copy_(e.ids.roll(1))
        e.logits.mul_(0.5)
        graph.replay()
        stream.synchronize()
        got = [t.clone() for t in e.outputs()]
        e.calls()
        stream.synchronize()
        for a, b in zip(e.outputs(), got):
            assert torch.equal(a, b)
        assert not torch.equal(got[1], want[1])
        e.close()


def test_contexts_side_by_side(gpu_lib):
    """Two contexts on two streams do not disturb each other."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    ends, want = [], []
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            ends.append(_Ends(gpu_lib, 1200 + 300 * i, 500, 200, i, 600))
            ends[i].calls()
            s.synchronize()
            want.append([t.clone() for t in ends[i].outputs()])
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                ends[i].calls()
    torch.cuda.synchronize()
    for i in (0, 1):
        for a, b in zip(ends[i].outputs(), want[i]):
            assert torch.equal(a, b)
        ends[i].close()


def test_after_the_policy_loss_and_before_it(gpu_lib):
    """The calls share tickets and workspace with the training side's: any order gives the same."""
    moe = gpu_lib
    rows, V = 40, 40000
    z = torch.randn((rows, V), device="cuda")
    target, f = torch.arange(rows, device="cuda", dtype=torch.int32), lambda: torch.randn(rows, device="cuda")  # noqa: E731
    fixed = [f(), f(), f().abs()]
    out = [torch.empty(rows, device="cuda") for _ in range(3)] + [torch.empty(1, device="cuda")]
    e = _Ends(moe, 1300, 600, 144, 5, 700)

    def loss():
        moe.moe_policy_loss(e.ctx, z, target, fixed[0], None, fixed[1], fixed[2], *out)
    loss()
    e.calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (*out, *e.outputs())]
    for order in ((e.calls, loss), (loss, e.calls, loss), (e.calls, e.calls, loss)):
        for call in order:
            call()
        torch.cuda.synchronize()
        for a, b in zip((*out, *e.outputs()), want):
            assert torch.equal(a, b)
    e.close()
