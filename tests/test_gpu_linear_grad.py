"""moe_linear_fp8_dgrad and moe_linear_fp8_wgrad against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import fp_formats as ff
from oracle import training as tr
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded, randn

pytestmark = pytest.mark.gpu


def _inputs(rows, E, NOUT, K, seed):
    rng = np.random.default_rng(seed)
    code = lambda *s: ff.e4m3_encode(rng.normal(size=s) * 60)  # noqa: E731
    return dict(dy=randn((rows, NOUT), "bf16", seed), Wq=code(E, NOUT, K), ws=(2.0 ** rng.uniform(-12, -6, (E, NOUT // 128, K // 128))).astype(np.float32),
                xq=code(rows, K), xs=(2.0 ** rng.uniform(-9, -5, (K // 128, rows))).astype(np.float32))


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _bounds(E, rows, seed, kind):
    rng = np.random.default_rng(seed)
    if kind == "even":
        return np.linspace(0, rows, E + 1).astype(np.int32)
    p = (np.arange(E) + 1.0) ** -1.2
    counts = np.bincount(rng.choice(E, rows, p=p / p.sum()), minlength=E)
    return np.concatenate([[0], np.cumsum(rng.permutation(counts))]).astype(np.int32)


def _check(n, offsets, grouped, moe, types=("bf16", "f32")):
    E, NOUT, K = n["Wq"].shape
    rows = n["dy"].shape[0]
    dx_o, dW_o = tr.linear_backward(f64(n["dy"]), n["Wq"], n["ws"], n["xq"], n["xs"], offsets)
    dx_s, dW_s = tr.linear_backward(np.abs(f64(n["dy"])), n["Wq"] & 0x7F, np.abs(n["ws"]), n["xq"] & 0x7F, np.abs(n["xs"]), offsets)
    dev = {k: v.cuda() if k == "dy" else _dev(v) for k, v in n.items()}
    off = _dev(offsets) if grouped else None
    Wq, ws = (dev["Wq"], dev["ws"]) if grouped else (dev["Wq"][0], dev["ws"][0])
    end = int(offsets[-1])
    dx, check_x = guarded((rows, K), torch.bfloat16)
    with Context(moe) as ctx:
        moe.moe_linear_fp8_dgrad(ctx, dev["dy"], Wq, ws, off, dx)
        torch.cuda.synchronize()
        check_x()
        # products exact, sums of NOUT terms in fp32 (with an fp32 scale for each block of 128)
        assert (np.abs(f64(dx) - dx_o)[:end] <= HALF_ULP["bf16"] * 1.01 * np.abs(dx_o)[:end] + (NOUT / 8 + 16) * F32 * dx_s[:end]).all()
        assert (f64(dx)[end:] == 37.0).all()
        for type in types:
            dW, check_W = guarded((E, NOUT, K) if grouped else (NOUT, K), TYPES[type])
            moe.moe_linear_fp8_wgrad(ctx, dev["dy"], dev["xq"], dev["xs"], off, dW)
            torch.cuda.synchronize()
            check_W()
            got = f64(dW).reshape(dW_o.shape)
            # operand: rounded to bf16 for a bf16 result (each product off by 2^-8 at most), exact but for 2^-24 otherwise
            operand = 2.0 ** -8 if type == "bf16" else 4 * F32
            bound = HALF_ULP[type] * 1.01 * np.abs(dW_o) + (operand * 1.01 + (rows / 8 + 16) * F32) * dW_s
            assert (np.abs(got - dW_o) <= bound).all(), (type, np.abs(got - dW_o).max())
            # added to what is there
            start = randn(tuple(dW.shape), type, 5, float(dW_s.mean())).cuda()
            total = start.clone()
            moe.moe_linear_fp8_wgrad(ctx, dev["dy"], dev["xq"], dev["xs"], off, total, accumulate=True)
            o = dW_o + f64(start).reshape(dW_o.shape)
            assert (np.abs(f64(total).reshape(dW_o.shape) - o) <= HALF_ULP[type] * 1.01 * np.abs(o) + (operand * 1.01 + (rows / 8 + 16) * F32) * dW_s
                    + F32 * np.abs(f64(start).reshape(dW_o.shape))).all()
            again = torch.empty_like(dW)
            moe.moe_linear_fp8_wgrad(ctx, dev["dy"], dev["xq"], dev["xs"], off, again)
            assert torch.equal(again, dW)
        dx2 = torch.full_like(dx, 37.0)
        moe.moe_linear_fp8_dgrad(ctx, dev["dy"], Wq, ws, off, dx2)
        assert torch.equal(dx2, dx)


@pytest.mark.parametrize("rows,NOUT,K", [(1, 128, 128), (5, 128, 384), (63, 256, 128), (64, 256, 256), (65, 384, 640), (127, 128, 256), (129, 640, 256),
                                         (255, 256, 384), (257, 512, 128), (300, 1408, 512), (40, 1024, 2176), (1000, 256, 256), (520, 896, 2176),
                                         (2100, 128, 128)])
def test_dense(gpu_lib, rows, NOUT, K):
    _check(_inputs(rows, 1, NOUT, K, rows), np.array([0, rows], np.int32), False, gpu_lib)


@pytest.mark.parametrize("rows,E,NOUT,K,kind", [(100, 4, 128, 256, "even"), (1, 8, 256, 128, "zipf"), (333, 60, 128, 128, "zipf"), (700, 256, 128, 128, "zipf"),
                                                (900, 3, 384, 256, "zipf"), (600, 1, 256, 384, "even"), (1500, 16, 256, 128, "zipf")])
def test_grouped(gpu_lib, rows, E, NOUT, K, kind):
    _check(_inputs(rows, E, NOUT, K, rows + E), _bounds(E, rows, E, kind), True, gpu_lib)


def test_rows_behind_the_last_expert_are_left_alone(gpu_lib):
    """Assignments with invalid ids leave rows behind offsets[E]: not written by dgrad, no part of wgrad's sums, whatever they hold."""
    n = _inputs(300, 4, 256, 256, 77)
    offsets = np.array([0, 100, 100, 130, 171], np.int32)
    clean = dict(n)
    _check(clean, offsets, True, gpu_lib)
    n["dy"][171:] = float("nan")
    n["xq"][171:] = 0x7F
    n["xs"][:, 171:] = np.nan
    with np.errstate(invalid="ignore"):
        _check(n, offsets, True, gpu_lib)


def test_a_neighbours_bad_rows_stay_with_it(gpu_lib):
    """Infinities and NaN in one expert's rows reach that expert's gradients only (tiles end inside the segments)."""
    n = _inputs(200, 3, 128, 128, 78)
    offsets = np.array([0, 70, 133, 200], np.int32)
    bad = {k: (v.clone() if k == "dy" else v.copy()) for k, v in n.items()}
    bad["dy"][70:133] = float("inf")
    bad["xq"][100] = 0x7F
    out = []
    with Context(gpu_lib) as ctx:
        for v in (n, bad):
            dev = {k: t.cuda() if k == "dy" else _dev(t) for k, t in v.items()}
            dx, dW, dWf = (torch.empty(s, dtype=t, device="cuda") for s, t in (((200, 128), torch.bfloat16), ((3, 128, 128), torch.bfloat16),
                                                                              ((3, 128, 128), torch.float32)))
            gpu_lib.moe_linear_fp8_dgrad(ctx, dev["dy"], dev["Wq"], dev["ws"], _dev(offsets), dx)
            gpu_lib.moe_linear_fp8_wgrad(ctx, dev["dy"], dev["xq"], dev["xs"], _dev(offsets), dW)
            gpu_lib.moe_linear_fp8_wgrad(ctx, dev["dy"], dev["xq"], dev["xs"], _dev(offsets), dWf)
            out.append((dx, dW, dWf))
    for a, b in zip(*out):
        keep = [0, 2] if a.dim() == 3 else list(range(70)) + list(range(133, 200))
        assert torch.equal(a[keep], b[keep])
        assert not torch.isfinite(b[1 if a.dim() == 3 else 90]).all()


def test_an_infinite_last_row_is_not_a_nan(gpu_lib):
    """Rows that pad the last step of a sum must not turn an infinity into a NaN."""
    n = _inputs(70, 1, 128, 128, 79)
    n["xq"][:] = 0x38                                          # 1.0
    n["dy"][:] = 1.0
    n["dy"][69, 5] = float("inf")
    for type in ("bf16", "f32"):
        dW = torch.empty((128, 128), dtype=TYPES[type], device="cuda")
        with Context(gpu_lib) as ctx:
            gpu_lib.moe_linear_fp8_wgrad(ctx, n["dy"].cuda(), _dev(n["xq"]), _dev(n["xs"]), None, dW)
        assert (dW[5] == float("inf")).all() and torch.isfinite(dW[6]).all()


def test_extreme_and_zero_scales(gpu_lib):
    """Block scales far apart, negative, one and zero: each block's sum counts with its own."""
    n = _inputs(50, 1, 768, 256, 80)
    n["ws"][0, :, 0] = [1e-30, 1.0, 0.0, 3e20, -2.5, 1e-12]
    n["ws"][0, :, 1] = [1.0, 1e-30, 1e-30, 0.0, 1e-25, 0.0]
    n["xs"][0, :] = np.where(np.arange(50) % 3 == 0, 0.0, n["xs"][0])
    n["xs"][1, :] = -n["xs"][1]
    _check(n, np.array([0, 50], np.int32), False, gpu_lib)


def test_the_forward_passes_own_checkpoint(gpu_lib):
    """Codes and scales as moe_quantize_fp8 and moe_quantize_weights_fp8 write them, the pair that moe_linear_fp8 multiplies."""
    rows, NOUT, K = 77, 384, 256
    x, w = randn((rows, K), "bf16", 1), randn((NOUT, K), "bf16", 2, 0.05)
    xq, xs = torch.empty((rows, K), dtype=torch.uint8, device="cuda"), torch.empty((K // 128, rows), device="cuda")
    Wq, ws = torch.empty((NOUT, K), dtype=torch.uint8, device="cuda"), torch.empty((NOUT // 128, K // 128), device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_quantize_fp8(ctx, x.cuda(), rows, K, 128, None, 1, xq, xs)
        gpu_lib.moe_quantize_weights_fp8(ctx, w.cuda(), NOUT, K, Wq, ws)
    n = dict(dy=randn((rows, NOUT), "bf16", 3), Wq=Wq.cpu().numpy()[None], ws=ws.cpu().numpy()[None], xq=xq.cpu().numpy(), xs=xs.cpu().numpy())
    _check(n, np.array([0, rows], np.int32), False, gpu_lib)


def test_no_rows_and_refusals(gpu_lib):
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    u = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    with Context(gpu_lib) as ctx:
        dW, was = torch.full((128, 256), 3.0, device="cuda"), torch.full((128, 256), 3.0, device="cuda")
        gpu_lib.moe_linear_fp8_wgrad(ctx, b(0, 128), u(0, 256), f(2, 0), None, dW)
        assert (dW == 0).all()
        gpu_lib.moe_linear_fp8_wgrad(ctx, b(0, 128), u(0, 256), f(2, 0), None, was, accumulate=True)
        assert (was == 3).all()
        gpu_lib.moe_linear_fp8_dgrad(ctx, b(0, 128), u(128, 256), f(1, 2), None, b(0, 256))
        d, w = gpu_lib.moe_linear_fp8_dgrad, gpu_lib.moe_linear_fp8_wgrad
        for call, args in [(d, (b(4, 100), u(100, 256), f(0, 2), None, b(4, 256))), (d, (b(4, 128), u(128, 200), f(1, 1), None, b(4, 200))),
                           (d, (f(4, 128), u(128, 256), f(1, 2), None, b(4, 256))), (d, (b(4, 128), u(128, 256), f(1, 3), None, b(4, 256))),
                           (d, (b(4, 128), u(128, 256), f(1, 2), None, f(4, 256))), (d, (b(4, 128), u(2, 128, 256), f(2, 1, 2), None, b(4, 256))),
                           (d, (b(4, 128), u(2, 128, 256), f(2, 1, 2), i(2), b(4, 256))), (d, (b(4, 128), u(300, 128, 128), f(300, 1, 1), i(301), b(4, 128))),
                           (w, (b(4, 128), u(5, 256), f(2, 4), None, f(128, 256))), (w, (b(4, 128), u(4, 256), f(4, 2), None, f(128, 256))),
                           (w, (b(4, 128), u(4, 256), f(2, 4), None, f(128, 256).half())), (w, (b(4, 128), u(4, 256), f(2, 4), i(2), f(128, 256)))]:
            with pytest.raises(gpu_lib.MoEError):
                call(ctx, *args)
        with pytest.raises(gpu_lib.MoEError):                  # 16-byte addresses
            d(ctx, b(4 * 128 + 1)[1:].view(4, 128), u(128, 256), f(1, 2), None, b(4, 256))
    with Context(gpu_lib, reserve=False) as ctx:
        for call, args in [(d, (b(4, 128), u(128, 256), f(1, 2), None, b(4, 256))), (w, (b(4, 128), u(4, 256), f(2, 4), None, f(128, 256)))]:
            with pytest.raises(gpu_lib.MoEError):
                call(ctx, *args)
