"""moe_add_rmsnorm and its gradient against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import fp_formats as ff
from oracle import training as tr
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded, keep, randn

pytestmark = pytest.mark.gpu
EPS = 1e-6
# rows, cols: one row, whole groups, odd widths, widths beyond one block's registers
SHAPES = [(1, 128), (1, 4096), (3, 1), (5, 7), (2, 257), (67, 384), (130, 1408), (33, 2176), (9, 5120), (4, 7168), (3, 16384), (2, 32768), (2, 65536),
          (2, 40001)]


def _sum_error(cols):
    """Relative error of an fp32 sum of squares over a row: a thread's chain of cols/64 additions at most, and a tree"""
    return (cols / 64 + 16) * F32


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(gpu_lib, shape, residual, type):
    rows, cols = shape
    x, res = randn(shape, type, 1), randn(shape, type, 2, 3.0) if residual else None
    gain = 1 + randn((cols,), "f32", 3, 0.3)
    h_o, y_o, r_o = tr.add_rmsnorm(f64(x), f64(res) if residual else None, f64(gain), EPS, keep(type))
    t = TYPES[type]
    s, check_s = guarded(shape, t)
    y, check_y = guarded(shape, t)
    rstd, check_r = guarded((rows,), torch.float32)
    coded = cols % 128 == 0 and cols <= 32768
    q, check_q = guarded(shape, torch.uint8)
    scales, check_c = guarded((cols // 128, rows), torch.float32)
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_add_rmsnorm(ctx, x.cuda(), res.cuda() if residual else None, gain.cuda(), EPS, s, y, q if coded else None,
                                scales if coded else None, rstd)
        torch.cuda.synchronize()
    for check in (check_s, check_y, check_r, check_q, check_c):
        check()
    assert np.array_equal(f64(s), h_o)
    rel = _sum_error(cols) + 4 * F32
    assert (np.abs(f64(rstd) - r_o) <= rel * r_o).all()
    assert (np.abs(f64(y) - y_o) <= (rel + HALF_ULP[type] * 1.01) * np.abs(y_o)).all()
    if coded:
        s_o = tr.group_scales(y_o)
        assert (np.abs(f64(scales) - s_o) <= (rel + 2 * F32) * s_o).all()
        s_g = np.repeat(f64(scales), 128, axis=0).T
        value = ff.e4m3_decode(q.cpu().numpy()) * s_g
        # nearest of values 1/8 of a binade apart, or 2^-9 below the normal range
        assert (np.abs(value - y_o) <= np.maximum(np.abs(y_o) * (2.0 ** -4 + 2 * rel), s_g * 2.0 ** -10 * 1.001)).all()


def test_codes_without_other_outputs_and_zero_groups(gpu_lib):
    """Codes alone; groups of zeros have scale 1 and codes 0; a row of zeros with eps > 0."""
    x = randn((6, 512), "bf16", 5)
    x[:, 128:256] = 0
    x[2] = 0
    gain = torch.ones(512)
    q, scales = torch.empty((6, 512), dtype=torch.uint8, device="cuda"), torch.empty((4, 6), device="cuda")
    with Context(gpu_lib, reserve=False) as ctx:
        gpu_lib.moe_add_rmsnorm(ctx, x.cuda(), None, gain.cuda(), EPS, q=q, scales=scales)
    assert (scales[1] == 1).all() and (q[:, 128:256] & 0x7F == 0).all()
    assert (scales[:, 2] == 1).all() and (q[2] & 0x7F == 0).all()
    y_o = tr.add_rmsnorm(f64(x), None, f64(gain), EPS, None)[1]
    assert (np.abs(f64(scales) - tr.group_scales(y_o)) <= 1e-5 * tr.group_scales(y_o)).all()


@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_rows_with_strides_and_sum_in_place(gpu_lib, type):
    t = TYPES[type]
    wide, res = randn((20, 1000), type, 7).cuda(), randn((20, 640), type, 8).cuda()
    x = wide[:, 64:64 + 640]                                   # 16-byte aligned rows
    odd = wide[:, 3:3 + 640]                                   # and others
    gain = (1 + randn((640,), "f32", 9, 0.3)).cuda()
    with Context(gpu_lib, reserve=False) as ctx:
        for v in (x, odd):
            h, y, r = torch.empty((20, 640), dtype=t, device="cuda"), torch.empty((20, 640), dtype=t, device="cuda"), torch.empty(20, device="cuda")
            gpu_lib.moe_add_rmsnorm(ctx, v, res, gain, EPS, h, y, rstd=r)
            h2, y2, r2 = torch.empty_like(h), torch.empty_like(y), torch.empty_like(r)
            gpu_lib.moe_add_rmsnorm(ctx, v.contiguous(), res, gain, EPS, h2, y2, rstd=r2)
            assert torch.equal(h, h2)
            assert (np.abs(f64(y) - f64(y2)) <= (2 * HALF_ULP[type] + 30 * F32) * np.abs(f64(y2))).all()
            inplace = res.clone()
            gpu_lib.moe_add_rmsnorm(ctx, v, inplace, gain, EPS, inplace, y2)
            assert torch.equal(inplace, h)


def test_bad_values_stay_in_their_rows(gpu_lib):
    x = randn((5, 384), "bf16", 11)
    clean = x.clone()
    x[1, 7], x[3, 200] = float("nan"), float("inf")
    gain = torch.ones(384, device="cuda")
    out = []
    with Context(gpu_lib) as ctx:
        for v in (x, clean):
            y = torch.empty((5, 384), dtype=torch.bfloat16, device="cuda")
            r = torch.empty(5, device="cuda")
            gpu_lib.moe_add_rmsnorm(ctx, v.cuda(), None, gain, EPS, y=y, rstd=r)
            out.append((y, r))
    for a, b in zip(*out):
        assert torch.equal(a[[0, 2, 4]], b[[0, 2, 4]])
    assert out[0][0][1].isnan().all() and out[0][0][3, 200].isnan()


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [True, False])
@pytest.mark.parametrize("shape", SHAPES + [(1100, 640), (2500, 136)], ids=str)
def test_backward(gpu_lib, shape, dh, type):
    rows, cols = shape
    h, dy, e = randn(shape, type, 21, 2.0), randn(shape, type, 22), randn(shape, type, 23) if dh else None
    gain = 1 + randn((cols,), "f32", 24, 0.3)
    rstd = torch.rsqrt(h.double().square().mean(dim=1) + EPS).float()
    dx_o, dg_o = tr.add_rmsnorm_backward(f64(dy), f64(h), f64(rstd), f64(gain), f64(e) if dh else None)
    dx, check_x = guarded(shape, TYPES[type])
    dg, check_g = guarded((cols,), torch.float32)
    with Context(gpu_lib) as ctx:
        args = (dy.cuda(), h.cuda(), rstd.cuda(), gain.cuda(), e.cuda() if dh else None)
        gpu_lib.moe_add_rmsnorm_backward(ctx, *args, dx, dg)
        torch.cuda.synchronize()
        check_x()
        check_g()
        u, H, r = np.abs(f64(dy) * f64(gain)), np.abs(f64(h)), f64(rstd)[:, None]
        size = r * u + H * r ** 3 * ((u * H).sum(axis=1, keepdims=True) / cols) + (np.abs(f64(e)) if dh else 0)
        assert (np.abs(f64(dx) - dx_o) <= HALF_ULP[type] * 1.01 * np.abs(dx_o) + (_sum_error(cols) + 8 * F32) * size).all()
        size = (np.abs(f64(dy)) * H * r).sum(axis=0)
        assert (np.abs(f64(dg) - dg_o) <= (rows / 256 + 80) * F32 * size).all()
        # in place, and the same bits again
        for k in (0, 4):
            if args[k] is None:
                continue
            again = [None if v is None else v.clone() for v in args]
            dg2 = torch.empty_like(dg)
            gpu_lib.moe_add_rmsnorm_backward(ctx, *again, again[k], dg2)
            assert torch.equal(again[k], dx) and torch.equal(dg2, dg)


def test_empty_batches(gpu_lib):
    z = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    gain, dg = torch.ones(256, device="cuda"), torch.full((256,), 3.0, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_add_rmsnorm(ctx, z, z, gain, EPS, y=z)
        gpu_lib.moe_add_rmsnorm_backward(ctx, z, z, torch.empty(0, device="cuda"), gain, None, z, dg)
    assert (dg == 0).all()


def test_refusals(gpu_lib):
    E = gpu_lib.MoEError
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    u = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    x, g = b(4, 256), f(256)
    with Context(gpu_lib) as ctx:
        call = lambda *a, **k: gpu_lib.moe_add_rmsnorm(ctx, *a, **k)  # noqa: E731
        for args, kw in [((x, None, g, EPS), {}),                                    # nothing to write
                         ((x, None, g, -1.0), dict(y=b(4, 256))), ((x, None, g, float("nan")), dict(y=b(4, 256))),
                         ((x, None, f(255), EPS), dict(y=b(4, 256))), ((x, b(4, 255), g, EPS), dict(y=b(4, 256))),
                         ((x, f(4, 256), g, EPS), dict(y=b(4, 256))), ((x, None, g, EPS), dict(y=f(4, 256))),
                         ((x, None, g, EPS), dict(q=u(4, 256))), ((x, None, g, EPS), dict(q=u(4, 256), scales=f(4, 2))),
                         ((b(4, 200), None, f(200), EPS), dict(q=u(4, 200), scales=f(1, 4))),
                         ((b(4, 520)[:, 1:257], None, g, EPS), dict(q=u(4, 256), scales=f(2, 4))),   # codes need aligned rows
                         ((x.half(), None, g, EPS), dict(y=b(4, 256))), ((x.t(), None, f(4), EPS), dict(y=b(256, 4))),
                         ((b(4, 512)[:, :256], None, g, EPS), dict(sum=b(4, 512)[:, :256]))]:
            with pytest.raises(E):
                call(*args, **kw)
        back = lambda *a: gpu_lib.moe_add_rmsnorm_backward(ctx, *a)  # noqa: E731
        for args in [(x, x, f(3), g, None, b(4, 256), f(256)), (x, f(4, 256), f(4), g, None, b(4, 256), f(256)),
                     (x, x, f(4), g, None, b(4, 256), f(255)), (x, x, f(4), g, b(3, 256), b(4, 256), f(256)), (x, x, f(4), g, None, None, f(256))]:
            with pytest.raises(E):
                back(*args)
    with Context(gpu_lib, reserve=False) as ctx, pytest.raises(E):                    # the workspace was not reserved
        gpu_lib.moe_add_rmsnorm_backward(ctx, x, x, f(4), g, None, b(4, 256), f(256))
