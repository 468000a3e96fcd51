"""moe_dispatch, moe_dispatch_backward and moe_combine_backward against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import fp_formats as ff
from oracle import moe_layer as om
from oracle import training as tr
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded, keep, randn

pytestmark = pytest.mark.gpu
# T, d, E, k
SHAPES = [(1, 128, 8, 2), (1, 7168, 256, 8), (3, 128, 1, 1), (64, 256, 8, 3), (33, 2176, 60, 5), (200, 1024, 40, 16), (129, 4096, 5, 4),
          (17, 5120, 128, 7), (700, 384, 30, 6), (1100, 640, 12, 3)]


def _routing(T, E, k, seed, bad=True):
    """ids, inv_perm (with slots of invalid ids at -1) and gate weights"""
    rng = np.random.default_rng(seed)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    if bad and T > 2:
        idx[1, 0], idx[2, k - 1] = E + 3, -1
    flat = idx.reshape(-1)
    valid = (flat >= 0) & (flat < E)
    inv = np.full(T * k, -1, np.int32)
    order = np.flatnonzero(valid)[np.argsort(flat[valid], kind="stable")]
    inv[order] = np.arange(order.size)
    if not bad:
        assert np.array_equal(inv, om.permute(idx, E)[2])
    return idx, inv, rng.dirichlet(np.ones(k), T).astype(np.float32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_dispatch_and_back(gpu_lib, shape, type):
    T, d, E, k = shape
    _, inv, _ = _routing(T, E, k, 1)
    x, g, add = randn((T, d), type, 2), randn((T * k, d), type, 3), randn((T, d), type, 4)
    x_perm, check_p = guarded((T * k, d), TYPES[type], -5.0)
    dx, check_d = guarded((T, d), TYPES[type])
    with Context(gpu_lib, T, d, E, k, reserve=False) as ctx:
        gpu_lib.moe_dispatch(ctx, x.cuda(), _dev(inv), x_perm)
        assert np.array_equal(f64(x_perm), tr.dispatch(f64(x), inv, k, -5.0))
        for extra in (None, add):
            gpu_lib.moe_dispatch_backward(ctx, g.cuda(), _dev(inv), None if extra is None else extra.cuda(), dx)
            o = tr.dispatch_backward(f64(g), inv, k, None if extra is None else f64(extra))
            size = tr.dispatch_backward(np.abs(f64(g)), inv, k, None if extra is None else np.abs(f64(extra)))
            assert (np.abs(f64(dx) - o) <= HALF_ULP[type] * 1.01 * np.abs(o) + (k + 1) * F32 * size).all()
        own = add.cuda()
        gpu_lib.moe_dispatch_backward(ctx, g.cuda(), _dev(inv), own, own)
        assert torch.equal(own, dx)
        torch.cuda.synchronize()
        check_p()
        check_d()


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_combine_backward(gpu_lib, shape, type):
    T, d, E, k = shape
    idx, inv, w = _routing(T, E, k, 5)
    if k > 1 and T > 40:
        idx[40, 1] = idx[40, 0]                                # a repeated id receives the sum of its slots
    dy, y_perm = randn((T, d), type, 6), randn((T * k, d), "f32", 7)
    missing = np.setdiff1d(np.arange(T * k), inv)
    y_perm[missing] = float("nan")                             # rows that no slot names are not read
    dy_perm, check_p = guarded((T * k, d), TYPES[type], -5.0)
    dw, check_w = guarded((T, k), torch.float32)
    dl, check_l = guarded((T, E), torch.float32)
    o_perm, o_w, o_l = tr.combine_backward(f64(dy), f64(y_perm), inv, w.astype(np.float64), idx, E, -5.0)
    with Context(gpu_lib, T, d, E, k, reserve=False) as ctx:
        args = (ctx, dy.cuda(), y_perm.cuda(), _dev(inv), _dev(w))
        gpu_lib.moe_combine_backward(*args, _dev(idx), dy_perm, dw, dl)
        dw2, rows2 = torch.empty_like(dw), torch.full_like(dy_perm, -5.0)
        gpu_lib.moe_combine_backward(*args, None, rows2, dw2, None)
        torch.cuda.synchronize()
    for check in (check_p, check_w, check_l):
        check()
    assert np.array_equal(f64(dy_perm), keep(type)(o_perm))    # one product in fp32, one rounding
    assert torch.equal(rows2, dy_perm) and torch.equal(dw2, dw)
    size = tr.combine_backward(np.abs(f64(dy)), np.abs(f64(y_perm)), inv, w.astype(np.float64), idx, E, 0.0)[1]
    bound = (d / 64 + 16) * F32 * size                         # a thread's chain of d/64 additions at most, and a tree
    assert (np.abs(f64(dw) - o_w) <= bound).all()
    each = w * (bound + (w * bound).sum(axis=1, keepdims=True) + 8 * F32 * (np.abs(o_w) + np.abs(w * o_w).sum(axis=1, keepdims=True)))
    bound_l = np.zeros((T, E))
    for t in range(T):
        for j in range(k):
            if 0 <= idx[t, j] < E:
                bound_l[t, idx[t, j]] += each[t, j]
    assert (np.abs(f64(dl) - o_l) <= bound_l).all()


def test_rows_behind_the_valid_ones_and_wild_entries(gpu_lib):
    """An inv_perm entry beyond the last row is skipped like a negative one."""
    T, d, E, k = 8, 256, 4, 2
    _, inv, w = _routing(T, E, k, 9, bad=False)
    inv[3], inv[9] = T * k, 2 ** 31 - 1
    x, g = randn((T, d), "bf16", 1), randn((T * k, d), "bf16", 2)
    out, check = guarded((T * k, d), torch.bfloat16, -5.0)
    legal = np.where(inv < T * k, inv, -1)
    with Context(gpu_lib, T, d, E, k, reserve=False) as ctx:
        gpu_lib.moe_dispatch(ctx, x.cuda(), _dev(inv), out)
        assert np.array_equal(f64(out), tr.dispatch(f64(x), legal, k, -5.0))
        dx = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
        gpu_lib.moe_dispatch_backward(ctx, g.cuda(), _dev(inv), None, dx)
        o = tr.dispatch_backward(f64(g), legal, k, None)
        assert (np.abs(f64(dx) - o) <= 2.0 ** -8 * np.abs(o) + 1e-6).all()
        dw = torch.empty((T, k), device="cuda")
        gpu_lib.moe_combine_backward(ctx, x.cuda(), torch.ones((T * k, d), device="cuda"), _dev(inv), _dev(w), None, out, dw, None)
        assert dw.view(-1)[3] == 0 and dw.view(-1)[9] == 0
        torch.cuda.synchronize()
        check()


def test_the_layers_own_permutation(gpu_lib):
    """The gradient of a replayed layer's combine, through the routing call's own inv_perm."""
    T, d, E, k = 96, 256, 8, 2
    idx, _, w = _routing(T, E, k, 12, bad=False)
    layer = gpu_lib.MoELayer(T, d, E, k, 128)
    try:
        layer.route_replay(None, _dev(idx), _dev(w))
        layer.y_perm.copy_(randn((T * k, d), "f32", 3).cuda())
        dy = randn((T, d), "bf16", 4)
        dy_perm, dw, dl = (torch.empty(s, dtype=t, device="cuda") for s, t in
                           (((T * k, d), torch.bfloat16), ((T, k), torch.float32), ((T, E), torch.float32)))
        gpu_lib.moe_combine_backward(layer.ctx, dy.cuda(), layer.y_perm, layer.inv_perm, layer.topk_w, layer.topk_idx, dy_perm, dw, dl)
        inv = layer.inv_perm.cpu().numpy()
        o = tr.combine_backward(f64(dy), f64(layer.y_perm), inv, w.astype(np.float64), idx, E, 0.0)
        assert np.array_equal(ff.f64_to_bf16_bits(f64(dy_perm)), ff.f64_to_bf16_bits(o[0].astype(np.float32).astype(np.float64)))
        assert np.abs(f64(dw) - o[1]).max() <= 1e-4 and np.abs(f64(dl) - o[2]).max() <= 1e-4
    finally:
        layer.close()


def test_empty_batch_and_refusals(gpu_lib):
    b, f = torch.bfloat16, torch.float32
    z = lambda *s, t=b: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    with Context(gpu_lib, 0, 128, 4, 2, reserve=False) as ctx:
        gpu_lib.moe_dispatch(ctx, z(0, 128), i(0), z(0, 128))
        gpu_lib.moe_dispatch_backward(ctx, z(0, 128), i(0), None, z(0, 128))
        gpu_lib.moe_combine_backward(ctx, z(0, 128), z(0, 128, t=f), i(0), z(0, 2, t=f), None, z(0, 128), z(0, 2, t=f), None)
    with Context(gpu_lib, 4, 128, 4, 2, reserve=False) as ctx:
        x, r, y, w = z(4, 128), z(8, 128), z(8, 128, t=f), z(4, 2, t=f)
        for call, args in [(gpu_lib.moe_dispatch, (z(5, 128), i(8), r)), (gpu_lib.moe_dispatch, (x, i(7), r)),
                           (gpu_lib.moe_dispatch, (x, i(8), z(7, 128))), (gpu_lib.moe_dispatch, (x, i(8), y)),
                           (gpu_lib.moe_dispatch, (x.half(), i(8), r.half())), (gpu_lib.moe_dispatch_backward, (r, i(8), z(3, 128), x)),
                           (gpu_lib.moe_combine_backward, (x, r, i(8), w, None, r, w, None)),
                           (gpu_lib.moe_combine_backward, (x, y, i(8), w, i(4, 2), r, w, None)),
                           (gpu_lib.moe_combine_backward, (x, y, i(8), w, None, r, w, z(4, 4, t=f))),
                           (gpu_lib.moe_combine_backward, (x, y, i(8), w, i(4, 2), r, w, z(4, 5, t=f)))]:
            with pytest.raises(gpu_lib.MoEError):
                call(ctx, *args)
    with pytest.raises(gpu_lib.MoEError):
        gpu_lib.moe_dispatch(12345, x, i(8), r)
