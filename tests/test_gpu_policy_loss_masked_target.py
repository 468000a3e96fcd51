"""moe_policy_loss on rows whose target is masked while other logits are not: no effect, whatever the row's other inputs are."""
import numpy as np
import pytest
import torch

from training_common import TYPES, Context, randn

pytestmark = pytest.mark.gpu
SHAPES = [(12, 900), (12, 40003), (140, 70001)]                # a row in registers, rows in parts, a row read twice


def _row(v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


@pytest.mark.parametrize("params", [dict(kl_coef=0.05, entropy_coef=0.01), dict(kl_coef=0.0, entropy_coef=0.01), dict(kl_coef=0.05, entropy_coef=0.0)],
                         ids=str)
@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_masked_target_has_no_effect(gpu_lib, shape, type, params):
    rows, V = shape
    z = randn(shape, type, 1, 2.5)
    target = (np.arange(rows) * 7 % V).astype(np.int32)
    masked = np.arange(rows) % 3 == 1
    low = [float("-inf"), torch.finfo(TYPES[type]).min, -2e30]
    for i, r in enumerate(np.flatnonzero(masked)):
        z[r, target[r]] = low[i % 3]
    rng = np.random.default_rng(2)
    old, ref, A = -8 + rng.normal(size=rows), -8 + rng.normal(size=rows), rng.normal(size=rows)
    ref[1] = -np.inf                                           # masked by the reference policy too
    w = np.ones(rows)
    arg = [torch.from_numpy(target).cuda(), _row(old), _row(ref), _row(A), _row(w)]
    for grad in (None, type):
        for with_ref in (True, False):
            out = [torch.full((rows,), 9.0, device="cuda") for _ in range(3)] + [torch.full((1,), 9.0, device="cuda")]
            g = None if grad is None else torch.full(shape, 9.0, dtype=TYPES[type], device="cuda")
            use = [a if with_ref or i != 2 else None for i, a in enumerate(arg)]
            with Context(gpu_lib) as ctx:
                gpu_lib.moe_policy_loss(ctx, z.cuda(), *use, *out, g, **params)
            logp, H, loss, total = (o.cpu() for o in out)
            m = torch.from_numpy(masked)
            assert (logp[m] == float("-inf")).all() and (loss[m] == 0).all() and H.isfinite().all()
            assert logp[~m].isfinite().all() and (loss[~m] != 0).all() and total.isfinite().all()
            if g is not None:
                assert (g[m.cuda()] == 0).all() and g.isfinite().all()
                if params["entropy_coef"]:                     # (otherwise a ratio beyond its bound may leave nothing)
                    assert (g[~m.cuda()] != 0).any(dim=1).all()
