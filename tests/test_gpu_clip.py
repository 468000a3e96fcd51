"""moe_grad_norm and moe_clip_grads against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import step_ends as ends
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -126


def _list(sizes, types, seed, std=1.0, pad=8):
    """Tensors of these sizes at every alignment that their types have, inside larger ones, and a check that nothing around them was written."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    tensors, checks = [], []
    for i, (n, t) in enumerate(zip(sizes, types)):
        whole = torch.full((n + 2 * pad + 8,), 41.0, dtype=TYPES[t], device="cuda")
        at = pad + i % 8
        whole[at:at + n] = torch.randn(n, generator=g, device="cuda") * std
        tensors.append(whole[at:at + n])
        checks.append((whole, at, n))

    def check():
        for whole, at, n in checks:
            assert (whole[:at] == 41).all() and (whole[at + n:] == 41).all(), "written outside a tensor"
    return tensors, check


def _sum_sq(moe, ctx, grads):
    (s, check_s), (n, check_n) = guarded((1,), torch.float64), guarded((1,), torch.float32)
    moe.moe_grad_norm(ctx, grads, s, n)
    torch.cuda.synchronize()
    check_s()
    check_n()
    return s, n


def _check_sum(tensors, s, n):
    want = sum(float((f64(t) ** 2).sum()) for t in tensors)
    count = sum(t.numel() for t in tensors)
    # squares of fp32 numbers are exact in fp64; at most `count` additions
    assert abs(float(s) - want) <= 2.0 ** -53 * (count + 10) * want
    assert abs(float(n) - np.sqrt(want)) <= 1.01 * F32 * np.sqrt(want) + 1e-45


LISTS = [([1], ["f32"]), ([0, 3, 0], ["bf16", "bf16", "f32"]), ([8, 9, 7, 4096, 1], ["bf16"] * 5), ([100001, 16384, 16385, 5], ["f32", "bf16", "f32", "f32"]),
         ([3000003], ["bf16"]), ([257 + 13 * i for i in range(300)], ["bf16" if i % 3 else "f32" for i in range(300)]), ([], []),
         ([1 + i % 5 for i in range(1000)], ["f32" if i % 2 else "bf16" for i in range(1000)]), ([0] * 200 + [5], ["f32"] * 201)]


@pytest.mark.parametrize("sizes,types", LISTS, ids=lambda v: f"{len(v)}" if v and isinstance(v[0], str) else f"{sum(v)}")
def test_norm_and_clipping(gpu_lib, sizes, types):
    tensors, check = _list(sizes, types, 1)
    before = [f64(t) for t in tensors]
    with Context(gpu_lib) as ctx:
        grads = gpu_lib.GradList(tensors)
        s, n = _sum_sq(gpu_lib, ctx, grads)
        _check_sum(tensors, s, n)
        again, _ = _sum_sq(gpu_lib, ctx, tensors)
        assert torch.equal(s, again)
        norm = float(s) ** 0.5
        # above the norm: nothing changes, neither in place nor elsewhere
        outs, check_outs = _list(sizes, types, 2)
        gpu_lib.moe_clip_grads(ctx, grads, s, norm * 1.5 + 1, outs)
        gpu_lib.moe_clip_grads(ctx, grads, s, norm * 1.5 + 1)
        for o, t, b in zip(outs, tensors, before):
            assert torch.equal(o, t) and np.array_equal(f64(t), b)
        gpu_lib.moe_clip_grads(ctx, grads, s, norm * 0.3, outs)
        gpu_lib.moe_clip_grads(ctx, grads, s, norm * 0.3)
        torch.cuda.synchronize()
        check()
        check_outs()
    want = ends.clip(before, float(np.float32(norm * 0.3)))[1]
    for o, t, w, type in zip(outs, tensors, want, types):
        assert torch.equal(o, t)
        # the factor's rounding and the product's (and its share of fp64's sum)
        assert (np.abs(f64(t) - w) <= (2.02 * F32 + HALF_ULP[type] * 1.01) * np.abs(w) + TINY).all()


def test_squares_beyond_fp32(gpu_lib):
    """Gradients whose squares are no fp32 numbers, and those that cancel nothing: fp64 holds them all."""
    tiny = torch.full((1000,), 2.0 ** -140, device="cuda")
    huge = torch.full((5000,), 3e38, dtype=torch.float32, device="cuda")
    with Context(gpu_lib) as ctx:
        s, n = _sum_sq(gpu_lib, ctx, [tiny])
        assert float(s) == 1000 * 2.0 ** -280
        s, n = _sum_sq(gpu_lib, ctx, [huge, tiny])
        _sum = 5000 * float(huge[0].double() ** 2)
        assert abs(float(s) - _sum) <= 1e-12 * _sum and float(n) == float("inf")          # (the norm is no fp32 number, its square is held)
        gpu_lib.moe_clip_grads(ctx, [huge], s, 1e6)            # (a factor of 5e-35)
    assert (huge.double() * 5000 ** 0.5 / 1e6 - 1).abs().max() <= 3 * F32


def test_zeros_infinities_and_nan(gpu_lib):
    z, o = torch.zeros(100, device="cuda"), torch.full((100,), 9.0, device="cuda")
    with Context(gpu_lib) as ctx:
        s, n = _sum_sq(gpu_lib, ctx, [z])
        assert float(s) == 0 and float(n) == 0
        gpu_lib.moe_clip_grads(ctx, [z], s, 0.0, [o])
        assert (o == 0).all()
        g = torch.randn(1000, device="cuda")
        g[5] = float("inf")
        s, n = _sum_sq(gpu_lib, ctx, [g])
        assert float(s) == float("inf") and float(n) == float("inf")
        gpu_lib.moe_clip_grads(ctx, [g], s, 1.0)
        assert torch.isnan(g[5]) and (g[:5] == 0).all() and (g[6:] == 0).all()
        g = torch.randn(1000, device="cuda").bfloat16()
        g[999] = float("nan")
        s, n = _sum_sq(gpu_lib, ctx, [z, g])
        assert torch.isnan(s).all() and torch.isnan(n).all()
        gpu_lib.moe_clip_grads(ctx, [g], s, 1.0)
        assert torch.isnan(g).all()
        g = torch.randn(1000, device="cuda")
        s, _ = _sum_sq(gpu_lib, ctx, [g])
        gpu_lib.moe_clip_grads(ctx, [g], s, 0.0)
        assert (g == 0).all()


def test_a_sum_from_elsewhere(gpu_lib):
    """What several ranks add up between the two calls; norm not asked for."""
    g = torch.randn(5000, device="cuda")
    h, s = g.clone(), torch.empty(1, dtype=torch.float64, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_grad_norm(ctx, [g], s)
        s *= 4
        gpu_lib.moe_clip_grads(ctx, [g], s, 1.0)
    factor = np.float32(1.0 / np.sqrt(float(s)))
    assert torch.equal(g, h * float(factor))


def test_refusals(gpu_lib):
    t, s = torch.randn(64, device="cuda"), torch.empty(1, dtype=torch.float64, device="cuda")
    E = gpu_lib.MoEError
    for bad in ([t, t], [t[:40], t[30:]], [t.half()], [t.view(8, 8).t()], [t.cpu()], [t[::2]]):
        with pytest.raises(E):
            gpu_lib.GradList(bad)
    with Context(gpu_lib) as ctx:
        for outs in ([t[:32]], [t, t.clone()], [t.bfloat16()], []):
            with pytest.raises(E):
                gpu_lib.moe_clip_grads(ctx, [t], s, 1.0, outs)
        with pytest.raises(E):
            gpu_lib.moe_clip_grads(ctx, [t[:60]], s, 1.0, [t[4:]])         # shifted onto itself
        for args in ((torch.empty(1, device="cuda"),), (torch.empty(2, dtype=torch.float64, device="cuda"),), (s, torch.empty(2, device="cuda"))):
            with pytest.raises(E):
                gpu_lib.moe_grad_norm(ctx, [t], *args)
        for max_norm in (-1.0, float("nan"), float("inf")):
            with pytest.raises(E):
                gpu_lib.moe_clip_grads(ctx, [t], s, max_norm)
    with Context(gpu_lib, reserve=False) as ctx, pytest.raises(E):
        gpu_lib.moe_grad_norm(ctx, [t], s)
