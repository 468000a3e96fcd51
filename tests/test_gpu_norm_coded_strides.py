"""moe_add_rmsnorm with codes takes every stride whose rows lie at multiples of 16 bytes: four elements of f32, eight of bf16."""
import pytest
import torch

from training_common import TYPES, Context, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [7, 9000])
@pytest.mark.parametrize("type,step", [("f32", 4), ("bf16", 8)])
def test_strides_of_16_bytes(gpu_lib, type, step, rows):
    cols, ld_x, ld_r = 256, 256 + step, 256 + 3 * step
    x, res = randn((rows, ld_x), type, 1).cuda()[:, :cols], randn((rows, ld_r), type, 2).cuda()[:, step:step + cols]
    gain = (1 + randn((cols,), "f32", 3, 0.3)).cuda()
    outs = []
    with Context(gpu_lib, reserve=False) as ctx:
        for a, b in ((x, res), (x.contiguous(), res.contiguous())):
            h, q = torch.empty((rows, cols), dtype=TYPES[type], device="cuda"), torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
            s, r = torch.empty((cols // 128, rows), device="cuda"), torch.empty(rows, device="cuda")
            gpu_lib.moe_add_rmsnorm(ctx, a, b, gain, 1e-6, h, None, q, s, r)
            outs.append((h, q, s, r))
        for a, b in zip(*outs):
            assert torch.equal(a, b)
        for a, b in ((x[:, :128], None), (res[:, :128], None)):             # a part of the columns
            gpu_lib.moe_add_rmsnorm(ctx, a, b, gain[:128], 1e-6, q=q[:, :128].contiguous(), scales=s[:1])
        wide = torch.zeros((rows, ld_x + step // 2), dtype=TYPES[type], device="cuda")
        with pytest.raises(gpu_lib.MoEError):                  # rows that begin between
            gpu_lib.moe_add_rmsnorm(ctx, wide[:, :cols], None, gain, 1e-6, q=q, scales=s)
