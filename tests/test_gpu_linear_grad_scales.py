"""moe_linear_fp8_dgrad with block scales anywhere in fp32's range, its ends among them, against fp64."""
import pytest
import torch

from training_common import F32, HALF_ULP, Context

pytestmark = pytest.mark.gpu
# exponents of the block scales from .. to, and of dy
RANGES = {"large": (116, 127, -60), "largest": (127, 127, -40), "small": (-126, -112, 60), "below-normal": (-147, -126, 70), "mixed": (-147, 20, -4),
          "all": (-140, 127, -50)}


def _inputs(rows, E, NOUT, K, low, high, power, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dy = (torch.randn((rows, NOUT), generator=g, device="cuda") * 2.0 ** power).bfloat16()
    Wq = torch.randint(0, 256, (E, NOUT, K), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    Wq[(Wq & 127) == 127] = 1                                  # (NaN; in its place the smallest code)
    n = (E, NOUT // 128, K // 128)
    ws = torch.ldexp(1 + torch.rand(n, generator=g, device="cuda").double() * 0.99, torch.randint(low, high + 1, n, generator=g, device="cuda")).float()
    return dy, Wq, torch.where(torch.rand(n, generator=g, device="cuda") < 0.3, -ws, ws)


def _exact(dy, Wq, ws):
    NOUT, K = Wq.shape
    W = (Wq.view(torch.float8_e4m3fn).double().view(NOUT // 128, 128, K // 128, 128) * ws.double()[:, None, :, None]).view(NOUT, K)
    return dy.double() @ W, dy.double().abs() @ W.abs()


def _check(got, exact, size, NOUT):
    # fp32 sums of exact products in chains of at most NOUT / 32 matrix instructions, a rescaling each 64, and the result's own rounding
    bound = (NOUT / 16 + 64) * F32 * size + HALF_ULP["bf16"] * 1.01 * exact.abs() + 2.0 ** -133
    assert exact.abs().max() < 3e38 and (exact != 0).any()
    assert ((got.double() - exact).abs() <= bound).all(), float(((got.double() - exact).abs() / bound).max())


# few rows in 64 and 128 columns, tiles of 128 rows, tiles cut into parts
@pytest.mark.parametrize("rows,NOUT,K", [(5, 640, 1024), (30, 1024, 4096), (300, 512, 384), (1100, 2048, 1152)])
@pytest.mark.parametrize("range", RANGES)
def test_dense(gpu_lib, range, rows, NOUT, K):
    dy, Wq, ws = _inputs(rows, 1, NOUT, K, *RANGES[range], rows)
    dx = torch.full((rows, K), 9.0, dtype=torch.bfloat16, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_linear_fp8_dgrad(ctx, dy, Wq[0], ws[0], None, dx)
    _check(dx, *_exact(dy, Wq[0], ws[0]), NOUT)


@pytest.mark.parametrize("range", RANGES)
def test_by_expert(gpu_lib, range):
    rows, E, NOUT, K = 700, 5, 640, 512
    bounds = [0, 3, 3, 260, 500, 700]
    dy, Wq, ws = _inputs(rows, E, NOUT, K, *RANGES[range], 7)
    dx = torch.full((rows, K), 9.0, dtype=torch.bfloat16, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_linear_fp8_dgrad(ctx, dy, Wq, ws, torch.tensor(bounds, dtype=torch.int32, device="cuda"), dx)
    for e in (0, 2, 3, 4):
        at = slice(bounds[e], bounds[e + 1])
        _check(dx[at], *_exact(dy[at], Wq[e], ws[e]), NOUT)
