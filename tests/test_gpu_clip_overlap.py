"""moe_clip_grads with outputs in the memory of other gradients is refused, and with outputs between the gradients it is right."""
import math

import pytest
import torch

from training_common import Context

pytestmark = pytest.mark.gpu


def test_outputs_over_other_gradients(gpu_lib):
    whole = torch.randn(4096, device="cuda")
    a, b, c, d = whole[:1000], whole[1000:2000], whole[2000:3000], whole[3000:4000]
    before, s = whole.clone(), torch.empty(1, dtype=torch.float64, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_grad_norm(ctx, [a, c], s)
        for outs in ([c, a], [b, a], [c, d], [a, whole[1500:2500]], [whole[4:1004], c]):
            with pytest.raises(gpu_lib.MoEError):
                gpu_lib.moe_clip_grads(ctx, [a, c], s, 1.0, outs)
        torch.cuda.synchronize()
        assert torch.equal(whole, before)
        factor = float(torch.tensor(1.0 / math.sqrt(float(s)), dtype=torch.float32))
        gpu_lib.moe_clip_grads(ctx, [a, c], s, 1.0, [b, d])
        assert torch.equal(b, before[:1000] * factor) and torch.equal(d, before[2000:3000] * factor) and torch.equal(a, before[:1000])
        gpu_lib.moe_clip_grads(ctx, [c, a], s, 1.0, [d, a])    # one of them in place
        assert torch.equal(a, before[:1000] * factor) and torch.equal(d, before[2000:3000] * factor)
