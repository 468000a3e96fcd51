"""Arrays of more than 2^32 elements: what lies behind them is read and written where it belongs."""
import pytest
import torch

from training_common import F32, HALF_ULP, Context

pytestmark = pytest.mark.gpu
BF16, U8, CUDA = torch.bfloat16, torch.uint8, "cuda"


@pytest.fixture(autouse=True)
def _empty_cache():
    yield
    torch.cuda.empty_cache()


def _codes(shape):
    q = torch.randint(0, 126, shape, device=CUDA, dtype=U8)
    return q.add_(torch.randint(0, 2, shape, device=CUDA, dtype=U8).mul_(128))


def _values(q):
    return q.view(torch.float8_e4m3fn).double()


def test_policy_loss(gpu_lib):
    moe = gpu_lib
    rows, V, last = 33000, 131072, 600
    z = torch.empty((rows, V), dtype=BF16, device=CUDA).normal_()
    tail = z[-last:].clone()
    target = torch.randint(0, V, (rows,), device=CUDA, dtype=torch.int32)
    old, adv, w = torch.full((rows,), -11.0, device=CUDA), torch.randn(rows, device=CUDA), torch.full((rows,), 1.0, device=CUDA)
    out, short = [torch.empty(rows, device=CUDA) for _ in range(3)], [torch.empty(last, device=CUDA) for _ in range(3)]
    total, part, grad = torch.empty(1, device=CUDA), torch.empty(1, device=CUDA), torch.empty_like(tail)
    at = slice(rows - last, rows)
    with Context(moe) as ctx:
        moe.moe_policy_loss(ctx, z, target, old, None, adv, w, *out, total, z, entropy_coef=0.01)
        moe.moe_policy_loss(ctx, tail, target[at], old[at], None, adv[at], w[at], *short, part, grad, entropy_coef=0.01)
    for a, b in zip(out, short):
        assert torch.equal(a[at], b)
    assert torch.equal(z[at], grad)


def test_norm_and_its_gradient(gpu_lib):
    moe = gpu_lib
    rows, cols, last = 600000, 7168, 100
    x, gain = torch.empty((rows, cols), dtype=BF16, device=CUDA).normal_(), torch.rand(cols, device=CUDA) + 0.5
    y, rstd, y_s, r_s = torch.empty_like(x), torch.empty(rows, device=CUDA), torch.empty((last, cols), dtype=BF16, device=CUDA), torch.empty(last, device=CUDA)
    dgain, dg_s = torch.empty(cols, device=CUDA), torch.empty(cols, device=CUDA)
    with Context(moe) as ctx:
        moe.moe_add_rmsnorm(ctx, x, None, gain, 1e-6, None, y, None, None, rstd)
        moe.moe_add_rmsnorm(ctx, x[-last:], None, gain, 1e-6, None, y_s, None, None, r_s)
        assert torch.equal(y[-last:], y_s) and torch.equal(rstd[-last:], r_s)
        dx, dx_s = torch.empty_like(x), torch.empty_like(y_s)
        moe.moe_add_rmsnorm_backward(ctx, y, x, rstd, gain, None, dx, dgain)
        moe.moe_add_rmsnorm_backward(ctx, y[-last:], x[-last:], rstd[-last:], gain, None, dx_s, dg_s)
        assert torch.equal(dx[-last:], dx_s) and torch.isfinite(dgain).all()


def test_rows_by_expert(gpu_lib):
    moe = gpu_lib
    T, d, E, k = 100000, 7168, 16, 8
    N = T * k
    inv = torch.randperm(N, device=CUDA).to(torch.int32).view(T, k)
    inv[-1, 0], inv[-1, 1] = N - 1, N - 2                      # (rows written by two tokens: the last token's are not looked at below)
    idx = torch.arange(k, device=CUDA, dtype=torch.int32).repeat(T, 1)
    w = torch.softmax(torch.randn((T, k), device=CUDA), dim=1)
    dy, y = torch.empty((T, d), dtype=BF16, device=CUDA).normal_(), torch.empty((N, d), device=CUDA).normal_()
    rows, dw, dl = torch.empty((N, d), dtype=BF16, device=CUDA), torch.empty((T, k), device=CUDA), torch.empty((T, E), device=CUDA)
    behind = (inv >= N - 2000) & (torch.arange(T, device=CUDA) < T - 1)[:, None]
    t, j = behind.nonzero(as_tuple=True)
    p = inv[t, j].long()
    keep = p < N - 2
    t, j, p = t[keep], j[keep], p[keep]
    with Context(moe, T, d, E, k, reserve=False) as ctx:
        moe.moe_combine_backward(ctx, dy, y, inv, w, idx, rows, dw, dl)
        assert torch.equal(rows[p], (w[t, j][:, None] * dy[t].float()).to(BF16))
        exact, size = (dy[t].double() * y[p].double()).sum(1), (dy[t].double() * y[p].double()).abs().sum(1)
        assert ((dw[t, j].double() - exact).abs() <= (d / 256 + 16) * F32 * size).all()
        del y
        moe.moe_dispatch(ctx, dy, inv, rows)
        assert torch.equal(rows[p], dy[t])
        dx = torch.empty_like(dy)
        moe.moe_dispatch_backward(ctx, rows, inv, None, dx)
        some = t[:64]
        exact = rows[inv[some].long()].double().sum(1)
        assert ((dx[some].double() - exact).abs() <= HALF_ULP["bf16"] * 1.01 * exact.abs() + 16 * F32 * rows[inv[some].long()].double().abs().sum(1)).all()


def test_linear_gradients_of_many_experts(gpu_lib):
    moe = gpu_lib
    E, NOUT, K, rows = 128, 7168, 5120, 400
    Wq, ws = _codes((E, NOUT, K)), torch.rand((E, NOUT // 128, K // 128), device=CUDA) + 0.5
    off = torch.full((E + 1,), 200, dtype=torch.int32, device=CUDA)
    off[0], off[-1] = 0, rows
    dy, xq, xs = torch.randn((rows, NOUT), device=CUDA).to(BF16), _codes((rows, K)), torch.rand((K // 128, rows), device=CUDA) + 0.5
    dx, dW = torch.empty((rows, K), dtype=BF16, device=CUDA), torch.empty((E, NOUT, K), dtype=BF16, device=CUDA)
    with Context(moe) as ctx:
        moe.moe_linear_fp8_dgrad(ctx, dy, Wq, ws, off, dx)
        moe.moe_linear_fp8_wgrad(ctx, dy, xq, xs, off, dW)
    W = (_values(Wq[-1]).view(NOUT // 128, 128, K // 128, 128) * ws[-1].double()[:, None, :, None]).view(NOUT, K)
    g = dy[200:].double()
    exact, size = g @ W, g.abs() @ W.abs()
    assert ((dx[200:].double() - exact).abs() <= (NOUT / 16 + 64) * F32 * size + HALF_ULP["bf16"] * 1.01 * exact.abs()).all()
    x = (_values(xq[200:]).view(-1, K // 128, 128) * xs[:, 200:].t().double()[:, :, None]).view(-1, K)
    exact, size = g.t() @ x, g.abs().t() @ x.abs()
    assert ((dW[-1].double() - exact).abs() <= (HALF_ULP["bf16"] * 1.01 + 256 * F32) * size + HALF_ULP["bf16"] * 1.01 * exact.abs()).all()
    assert (dW[1:-1] == 0).all()


@pytest.mark.parametrize("NOUT,K", [(32768, 128), (128, 32768)])
def test_linear_gradients_of_many_rows(gpu_lib, NOUT, K):
    moe = gpu_lib
    rows, last = 140000, 300
    dy = torch.empty((rows, NOUT), dtype=BF16, device=CUDA).normal_()
    Wq, ws = _codes((NOUT, K)), torch.rand((NOUT // 128, K // 128), device=CUDA) + 0.5
    xq, xs = _codes((rows, K)), torch.rand((K // 128, rows), device=CUDA) + 0.5
    dx, dW = torch.empty((rows, K), dtype=BF16, device=CUDA), torch.empty((NOUT, K), device=CUDA)
    with Context(moe) as ctx:
        moe.moe_linear_fp8_dgrad(ctx, dy, Wq, ws, None, dx)
        moe.moe_linear_fp8_wgrad(ctx, dy, xq, xs, None, dW)
    W = (_values(Wq).view(NOUT // 128, 128, K // 128, 128) * ws.double()[:, None, :, None]).view(NOUT, K)
    g = dy[-last:].double()
    exact, size = g @ W, g.abs() @ W.abs()
    assert ((dx[-last:].double() - exact).abs() <= (NOUT / 16 + 64) * F32 * size + HALF_ULP["bf16"] * 1.01 * exact.abs()).all()
    x = _values(xq[:, -128:]) * xs[-1].double()[:, None]
    g = dy[:, -128:].t().double()
    exact, size = g @ x, g.abs() @ x.abs()
    assert ((dW[-128:, -128:].double() - exact).abs() <= (rows / 16 + 64) * F32 * size).all()
