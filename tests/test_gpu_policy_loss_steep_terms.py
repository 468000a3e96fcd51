"""moe_policy_loss where a term of the row's gradient is very steep: masked logits stay without one, and an infinite loss keeps the gradient that it has."""
import pytest
import torch

from training_common import TYPES, Context, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(6, 900), (6, 40003), (140, 70001)], ids=str)
def test_masked_logits_under_a_steep_entropy_term(gpu_lib, shape, type):
    """entropy_coef * weight / temperature = 1e16, next to logits of -inf"""
    rows, V = shape
    z = randn(shape, type, 1, 2e-6)
    z[:, ::5] = float("-inf")
    f = lambda v: torch.full((rows,), float(v), device="cuda")  # noqa: E731
    out, g = [f(9), f(9), f(9), torch.full((1,), 9.0, device="cuda")], torch.full(shape, 9.0, dtype=TYPES[type], device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_policy_loss(ctx, z.cuda(), torch.ones(rows, dtype=torch.int32, device="cuda"), f(-7), None, f(0.5), f(1e10), *out, g, entropy_coef=1.0,
                                temperature=1e-6)
    assert all(o.isfinite().all() for o in out) and g.isfinite().all()
    assert (g[:, ::5] == 0).all() and (g[:, 1] != 0).all()


@pytest.mark.parametrize("shape", [(6, 900), (6, 40003)], ids=str)
def test_reference_policy_without_the_token(gpu_lib, shape):
    """ref_logp = -inf: the KL term is infinite, its slope kl_coef * (1 - 0)"""
    rows, V = shape
    z = randn(shape, "f32", 2, 2.0)
    f = lambda v: torch.full((rows,), float(v), device="cuda")  # noqa: E731
    ref = f(-8)
    ref[2] = float("-inf")
    out, g = [f(9), f(9), f(9), torch.full((1,), 9.0, device="cuda")], torch.full(shape, 9.0, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_policy_loss(ctx, z.cuda(), torch.ones(rows, dtype=torch.int32, device="cuda"), f(-7), ref, f(0), f(1), *out, g, kl_coef=0.25)
    loss = out[2].cpu()
    assert loss[2] == float("inf") and out[3][0] == float("inf") and loss[[0, 1, 3, 4, 5]].isfinite().all()
    p = torch.softmax(z[2].double(), dim=0)
    want = -0.25 * p
    want[1] += 0.25
    # p: an exponent of at most 16 nats, off by five roundings of itself, and the sum's roundings
    assert ((g[2].cpu().double() - want).abs() <= (80 + 300) * 2.0 ** -24 * want.abs()).all()
    assert g.isfinite().all()
