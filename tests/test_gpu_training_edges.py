"""Very many rows, for which one grid is too small, and matrices too wide for a tile's 32-bit offsets."""
import pytest
import torch

from training_common import F32, HALF_ULP, Context, randn

pytestmark = pytest.mark.gpu
MANY = 2 ** 26 + 5                                             # times 64 threads: past 2^32


def test_norm_of_very_many_rows(gpu_lib):
    x = randn((4096, 2), "bf16", 1).cuda().repeat(MANY // 4096 + 1, 1)[:MANY].contiguous()
    gain = torch.tensor([0.5, 2.0], device="cuda")
    y, rstd = torch.full_like(x, 9.0), torch.full((MANY,), 9.0, device="cuda")
    with Context(gpu_lib, reserve=False) as ctx:
        gpu_lib.moe_add_rmsnorm(ctx, x, None, gain, 1e-6, None, y, None, None, rstd)
        few, r = torch.empty_like(x[:4096]), torch.empty_like(rstd[:4096])
        gpu_lib.moe_add_rmsnorm(ctx, x[:4096], None, gain, 1e-6, None, few, None, None, r)
    exact = torch.rsqrt(x[:4096].double().square().mean(dim=1) + 1e-6)
    assert ((r.double() - exact).abs() <= 8 * F32 * exact).all()
    whole = MANY // 4096 * 4096
    assert (y[:whole].view(-1, 4096, 2) == few).all() and (rstd[:whole].view(-1, 4096) == r).all()
    assert torch.equal(y[whole:], few[:MANY - whole]) and torch.equal(rstd[whole:], r[:MANY - whole])


def test_loss_of_very_many_rows(gpu_lib):
    n, few = MANY, 1024
    tile = lambda t: t.cuda().repeat(n // few + 1, *[1] * (t.dim() - 1))[:n].contiguous()  # noqa: E731
    z = tile(randn((few, 2), "f32", 2))
    target = tile((torch.arange(few) % 2).to(torch.int32))
    old, adv = tile(randn((few,), "f32", 3) - 1), tile(randn((few,), "f32", 4))
    weight = torch.full((n,), 2.0 ** -26, device="cuda")
    out = [torch.full((n,), 9.0, device="cuda") for _ in range(3)]
    short = [torch.empty(few, device="cuda") for _ in range(3)]
    loss, grad, part, g = torch.empty(1, device="cuda"), torch.full_like(z, 9.0), torch.empty(1, device="cuda"), torch.empty_like(z[:few])
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_policy_loss(ctx, z, target, old, None, adv, weight, *out, loss, grad)
        gpu_lib.moe_policy_loss(ctx, z[:few], target[:few], old[:few], None, adv[:few], weight[:few], *short, part, g)
    logp = torch.log_softmax(z[:few].double(), dim=1).gather(1, target[:few, None].long())[:, 0]
    assert ((short[0].double() - logp).abs() <= 8 * F32 * (1 + logp.abs())).all()
    whole = n // few * few
    for a, b in [*zip(out, short), (grad, g)]:
        assert (a[:whole].view(-1, *b.shape) == b).all() and torch.equal(a[whole:], b[:n - whole])
    total = out[2].double().sum()
    assert abs(loss.double() - total) <= F32 * total.abs() + 1e-12 * out[2].double().abs().sum()


def test_matrices_too_wide_for_a_tile(gpu_lib):
    t = torch.zeros(64, device="cuda")                         # (refused before anything is read)
    lib, p, wide = gpu_lib.load_library(), t.data_ptr(), 2 ** 24 + 128
    with Context(gpu_lib) as ctx:
        for NOUT, K in [(wide, 128), (128, wide)]:
            assert lib.moe_linear_fp8_dgrad(ctx, p, 1, NOUT, p, p, K, None, 1, p) == -1
            assert lib.moe_linear_fp8_wgrad(ctx, p, 1, NOUT, p, p, K, None, 1, 0, 0, p) == -1


@pytest.mark.parametrize("rows,NOUT,K", [(1, 128, 4096), (7, 640, 4224), (30, 1024, 4096), (45, 384, 6144), (64, 16384, 4096), (33, 2048, 640),
                                         (16, 192 * 128, 128), (48, 256, 3968), (90, 896, 1152), (128, 2048, 1024), (113, 128, 4096), (200, 4096, 512)])
def test_dgrad_of_few_rows(gpu_lib, rows, NOUT, K):
    """The forms for few rows: 64 and 128 columns, one to four tiles of rows, sums in one part and in many."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    dy = torch.randn((rows, NOUT), generator=g, device="cuda").bfloat16()
    Wq = torch.randint(0, 256, (NOUT, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    Wq[(Wq & 127) == 127] = 0                                  # (NaN)
    ws = torch.exp2(torch.randint(-20, 20, (NOUT // 128, K // 128), generator=g, device="cuda").float()) * (
        1 + torch.rand((NOUT // 128, K // 128), generator=g, device="cuda"))
    ws[0, 0] = 0
    whole = torch.full((rows + 2, K), 37.0, dtype=torch.bfloat16, device="cuda")
    again = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_linear_fp8_dgrad(ctx, dy, Wq, ws, None, whole[1:-1])
        gpu_lib.moe_linear_fp8_dgrad(ctx, dy, Wq, ws, None, again)
    assert (whole[0] == 37).all() and (whole[-1] == 37).all() and torch.equal(whole[1:-1], again)
    W = Wq.view(torch.float8_e4m3fn).double().view(NOUT // 128, 128, K // 128, 128) * ws.double()[:, None, :, None]
    W = W.view(NOUT, K)
    exact, size = dy.double() @ W, dy.double().abs() @ W.abs()
    # fp32 sums of exact products in chains of at most NOUT / 32 matrix instructions, a rescaling each 64, and the result's own rounding
    bound = (NOUT / 16 + 64) * F32 * size + HALF_ULP["bf16"] * 1.01 * exact.abs()
    assert ((again.double() - exact).abs() <= bound).all()
