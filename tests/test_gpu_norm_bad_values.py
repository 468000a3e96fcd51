"""moe_add_rmsnorm with codes: what is not finite leaves as what is not finite, in its own groups of columns only."""
import pytest
import torch

from training_common import TYPES, Context, randn

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(6, 384), (6, 7168), (9000, 1024)])                  # one row and several to a block
def test_codes_keep_nan_and_infinity(gpu_lib, rows, cols, type):
    x = randn((rows, cols), type, 1)
    gain = 1 + randn((cols,), "f32", 2, 0.2)
    clean, clean_gain = x.clone(), gain.clone()
    x[1, 7], x[3, 200], x[4, 0] = NAN, INF, -NAN
    gain[130] = INF                                            # of every row one group has an infinite y
    outs = []
    with Context(gpu_lib, reserve=False) as ctx:
        for v, g in ((x, gain), (clean, clean_gain)):
            q, s = torch.empty((rows, cols), dtype=torch.uint8, device="cuda"), torch.empty((cols // 128, rows), device="cuda")
            y = torch.empty((rows, cols), dtype=TYPES[type], device="cuda")
            gpu_lib.moe_add_rmsnorm(ctx, v.cuda(), None, g.cuda(), 1e-6, y=y, q=q, scales=s)
            outs.append((q.cpu(), s.cpu(), y.cpu()))
    (q, s, y), (q0, s0, _) = outs
    for r in (1, 4):                                           # NaN: the whole row is
        assert y[r].isnan().all() and s[:, r].isnan().all() and (q[r] & 0x7F == 0x7F).all()
    # an infinity: 1/rms is 0, the row 0 but for NaN where it stood, and 0 * inf under the infinite gain
    assert s[1, 3].isnan() and (q[3, 128:256] & 0x7F == 0x7F).all()
    other = [g for g in range(cols // 128) if g != 1]
    assert (s[other, 3] == 1).all() and (q[3].view(-1, 128)[other] & 0x7F == 0).all()
    # the infinite gain: scale inf, NaN there, signed zeros in the rest of its group
    for r in [0, 2, 5, rows - 1]:
        assert s[1, r] == INF and q[r, 130] & 0x7F == 0x7F
        rest = torch.cat([q[r, 128:130], q[r, 131:256]])
        assert (rest & 0x7F == 0).all()
        assert torch.equal(rest >> 7, torch.cat([q0[r, 128:130], q0[r, 131:256]]) >> 7)
        value = q[r, 128:256].view(torch.float8_e4m3fn).float() * s[1, r]
        assert value.isnan().all()
    # everything else as it is without them
    fine = [r for r in range(rows) if r not in (1, 3, 4)]
    assert torch.equal(q.view(rows, -1, 128)[fine][:, other], q0.view(rows, -1, 128)[fine][:, other]) and torch.equal(s[other][:, fine], s0[other][:, fine])


def test_the_linear_behind_it_sees_them(gpu_lib):
    """A bad row is a row of NaN in the products that read the codes, and no other row's."""
    x = randn((5, 256), "bf16", 3)
    x[2, 9] = NAN
    q, s = torch.empty((5, 256), dtype=torch.uint8, device="cuda"), torch.empty((2, 5), device="cuda")
    Wq = torch.full((128, 256), 0x38, dtype=torch.uint8, device="cuda")
    ws, y = torch.ones((1, 2), device="cuda"), torch.empty((5, 128), device="cuda")
    with Context(gpu_lib, T=5, d=256) as ctx:
        gpu_lib.moe_add_rmsnorm(ctx, x.cuda(), None, torch.ones(256, device="cuda"), 1e-6, q=q, scales=s)
        gpu_lib.moe_linear_fp8(ctx, q, s, 5, 256, Wq, ws, 128, y)
        torch.cuda.synchronize()
    assert y[2].isnan().all() and y[[0, 1, 3, 4]].isfinite().all()
