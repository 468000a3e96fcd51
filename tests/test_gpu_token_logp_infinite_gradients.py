"""moe_token_logp_backward of rows whose gradients are infinite or NaN: masked logits have none all the same."""
import pytest
import torch

from training_common import TYPES, Context, guarded, randn

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("type,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("rows,V", [(9, 43), (9, 5003), (9, 100001), (2061, 43)])
def test_masked_logits_of_spoiled_rows(gpu_lib, rows, V, type, out):
    g = torch.Generator().manual_seed(1)
    z = randn((rows, V), type, 2, 2.0)
    closed = torch.rand((rows, V), generator=g) < 0.4
    closed[:, :2], closed[:, V - 2], closed[:, V - 1] = False, True, False                     # (a masked one and an open one behind the vectors)
    z[closed] = torch.where(torch.rand((rows, V), generator=g)[closed] < 0.5, -INF, torch.finfo(TYPES[type]).min).to(TYPES[type])
    z[6, 1] = NAN
    z[7, 0] = INF
    ids = torch.zeros((rows, 2), dtype=torch.int32)
    ids[:, 1] = V - 1
    dlogp, dH = randn((rows, 2), "f32", 3), randn((rows,), "f32", 4)
    z, ids, dlogp, dH = z.cuda(), ids.cuda(), dlogp.cuda(), dH.cuda()
    logp, H, stats = torch.empty((rows, 2), device="cuda"), torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    clean, check_clean = guarded((rows, V), TYPES[out])
    got, check = guarded((rows, V), TYPES[out])
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_token_logp(ctx, z, ids, logp, H, stats=stats)
        gpu_lib.moe_token_logp_backward(ctx, z, ids, dlogp, dH, stats, H, clean)
        dlogp[0, 0], dlogp[1, 1], dlogp[2, 0] = INF, -INF, NAN
        dlogp[3] = torch.tensor([INF, -INF])
        dH[4], dH[5] = INF, NAN
        gpu_lib.moe_token_logp_backward(ctx, z, ids, dlogp, dH, stats, H, got)
        check_clean()
        check()
        assert (got[closed.cuda()] == 0).all() and (clean[closed.cuda()] == 0).all()
        others = torch.arange(rows, device="cuda") > 7
        assert torch.equal(got[others], clean[others]) and torch.isfinite(got[others]).all()
        for r in range(8):                                     # what is spoiled does not look sound
            assert not torch.isfinite(got[r, :2]).any(), r
        if type == out:
            gpu_lib.moe_token_logp_backward(ctx, z, ids, dlogp, dH, stats, H, z)
            assert torch.equal(z.view(torch.int16 if out == "bf16" else torch.int32), got.view(torch.int16 if out == "bf16" else torch.int32))
