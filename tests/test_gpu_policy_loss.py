"""moe_policy_loss against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import training as tr
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded, randn

pytestmark = pytest.mark.gpu
PARAMS = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05, entropy_coef=0.01, temperature=0.8)


def _inputs(rows, V, type, seed, masked=False):
    rng = np.random.default_rng(seed)
    z = randn((rows, V), type, seed, 2.5)
    target = rng.integers(0, V, rows).astype(np.int32)
    if masked:
        z[:, torch.from_numpy(rng.random(V) < 0.2)] = float("-inf")
        low = torch.finfo(TYPES[type]).min
        z[rng.random((rows, V)) < 0.1] = low
        z[np.arange(rows), target] = 1.0
    logp = tr.policy_loss(f64(z), target, np.zeros(rows), None, np.zeros(rows), np.zeros(rows), 0, 0, 0, 0, PARAMS["temperature"])[0]
    logp = np.where(np.isfinite(logp), logp, -1.0)
    f = lambda v: v.astype(np.float32)  # noqa: E731
    return dict(z=z, target=target, old=f(logp + rng.normal(size=rows) * 0.2), ref=f(logp + rng.normal(size=rows) * 0.3),
                A=f(rng.normal(size=rows)), w=f(rng.random(rows) * (rng.random(rows) > 0.2)))


def _call(moe, ctx, n, grad=None, ref=True, ld=None, **params):
    """Outputs of a call, everything it writes guarded"""
    rows, V = n["z"].shape
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    outs = [guarded((rows,), torch.float32) for _ in range(3)] + [guarded((1,), torch.float32)]
    g, check_g = guarded((rows, V), TYPES[grad]) if grad else (None, lambda: None)
    z = n["z"].cuda()
    if ld:
        wide = torch.full((rows, ld), 50.0, dtype=z.dtype, device="cuda")
        wide[:, 3:3 + V] = z
        z = wide[:, 3:3 + V]
    clip = params.pop("clip_rows", None)
    moe.moe_policy_loss(ctx, z, dev(n["target"]), dev(n["old"]), dev(n["ref"]) if ref else None, dev(n["A"]), dev(n["w"]),
                        *(o for o, _ in outs), g, clip_rows=None if clip is None else dev(clip), **params)
    torch.cuda.synchronize()
    for _, check in outs:
        check()
    check_g()
    return [o for o, _ in outs] + [g]


def _compare(n, got, type, grad, ref=True, clip_low=0.0, clip_high=0.0, kl_coef=0.0, entropy_coef=0.0, temperature=1.0):
    logp, H, loss, total, g = got
    z = f64(n["z"])
    arg = (z, n["target"], n["old"].astype(np.float64), n["ref"].astype(np.float64) if ref else None, n["A"].astype(np.float64), n["w"].astype(np.float64))
    logp_o, H_o, loss_o, g_o = tr.policy_loss(*arg, clip_low, clip_high, kl_coef, entropy_coef, temperature)
    # z/temperature and its distance from the maximum: a rounding or two each, of the largest |z| that counts; log-sum-exp: sums in fp32
    with np.errstate(invalid="ignore"):
        reach = np.where(np.isfinite(z) & (z > -1e30), np.abs(z), 0).max(axis=1) / temperature
    e_logp = (8 * reach + 4 * np.abs(np.where(np.isfinite(logp_o), logp_o, 0)) + 32) * F32
    assert np.array_equal(np.isfinite(f64(logp)), np.isfinite(logp_o))
    live = np.isfinite(logp_o)
    assert (np.abs(f64(logp)[live] - logp_o[live]) <= e_logp[live]).all()
    # entropy = log s - u/s: each term of u carries the error of e^x, |x| roundings
    e_H = (64 + 16 * reach) * F32 * (1 + np.abs(H_o) + reach)
    assert (np.abs(f64(H) - H_o) <= e_H).all()
    A, w = n["A"].astype(np.float64), n["w"].astype(np.float64)
    lp = np.where(live, logp_o, 0)
    rho = np.exp(lp - n["old"])
    back = np.exp(n["ref"] - lp) if ref else np.ones_like(lp)
    e_rho = rho * (e_logp + (4 + np.abs(lp - n["old"])) * F32)
    e_loss = w * (np.abs(A) * e_rho + kl_coef * (np.abs(back - 1) + 1) * 4 * e_logp * (1 + back) + entropy_coef * e_H + 4 * F32 * (rho * np.abs(A)))
    assert (np.abs(f64(loss) - loss_o) <= e_loss + 4 * F32 * np.abs(loss_o)).all()
    assert abs(float(total[0]) - loss_o.sum()) <= e_loss.sum() + 4 * F32 * np.abs(loss_o).sum()
    if g is None:
        return
    with np.errstate(invalid="ignore"):
        zt = z / temperature
        m = zt.max(axis=1, keepdims=True)
        x = np.where(np.isfinite(zt), zt - m, -np.inf)
        p = np.exp(x)
        p = p / np.where(p.sum(axis=1, keepdims=True) > 0, p.sum(axis=1, keepdims=True), 1)
        p = np.where(np.isnan(p), 0, p)
        x = np.where(p > 0, x, 0)
    slope = w * (np.abs(A) * rho + kl_coef * (1 + back))
    e_slope = w * (np.abs(A) * e_rho + kl_coef * back * 4 * e_logp) + 8 * F32 * slope
    bonus = (w * entropy_coef)[:, None]
    H_ = np.abs(H_o)[:, None]
    rel = (16 + 4 * np.abs(x)) * F32 + e_logp[:, None]
    bound = p * (e_slope[:, None] + slope[:, None] * rel + bonus * (e_H[:, None] + (np.abs(x) + H_ + reach[:, None] + 20) * rel))
    bound[np.arange(len(A)), np.clip(n["target"], 0, z.shape[1] - 1)] += e_slope + 8 * F32 * slope
    # values below the normal range of the type may be lost
    assert (np.abs(f64(g) - g_o) <= bound / temperature + HALF_ULP[grad] * 1.01 * np.abs(g_o) + 2e-38).all()


@pytest.mark.parametrize("type,grad", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32"), ("bf16", None), ("f32", None)])
@pytest.mark.parametrize("shape", [(1, 1), (3, 2), (1, 9), (5, 63), (9, 512), (40, 1000), (7, 4099), (3, 32768), (2, 50001), (2, 131072), (1, 262144),
                                   (300, 130)], ids=str)
def test_loss_and_gradient(gpu_lib, shape, type, grad):
    n = _inputs(*shape, type, 1)
    with Context(gpu_lib) as ctx:
        got = _call(gpu_lib, ctx, n, grad, **PARAMS)
        again = _call(gpu_lib, ctx, n, grad, **PARAMS)
    _compare(n, got, type, grad, **PARAMS)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(6, 300), (4, 5001), (3, 70000), (3, 131072)], ids=str)
def test_masked_logits_and_rows_without_effect(gpu_lib, shape, type):
    rows, V = shape
    n = _inputs(rows, V, type, 2, masked=True)
    n["z"][0] = float("-inf")                                  # nothing left
    n["target"][1] = -100                                      # no target
    n["w"][2] = 0.0                                            # no weight, and values that would spoil a sum
    n["A"][2], n["old"][2], n["ref"][2] = np.inf, -np.inf, np.nan
    with Context(gpu_lib) as ctx:
        got = _call(gpu_lib, ctx, n, type, **PARAMS)
    logp, H, loss, _, g = got
    assert logp[0] == float("-inf") and H[0] == 0 and logp[1] == 0
    for r in (0, 1, 2):
        assert loss[r] == 0 and (g[r] == 0).all()
    assert (g[n["z"].cuda() == float("-inf")] == 0).all()
    n["A"][2], n["old"][2], n["ref"][2] = 0, 0, 0
    _compare(n, got, type, type, **PARAMS)


def test_strided_rows_and_in_place(gpu_lib):
    n = _inputs(37, 1001, "bf16", 3)
    with Context(gpu_lib) as ctx:
        want = _call(gpu_lib, ctx, n, "bf16", **PARAMS)
        strided = _call(gpu_lib, ctx, n, "bf16", ld=1100, **PARAMS)
        _compare(n, strided, "bf16", "bf16", **PARAMS)
        for V in (1001, 16384, 131072):                        # the gradient in the logits' place
            n = _inputs(5, V, "bf16", 4)
            want = _call(gpu_lib, ctx, n, "bf16", **PARAMS)
            z = n["z"].cuda()
            dev = lambda k: torch.from_numpy(n[k]).cuda()  # noqa: E731
            o = [torch.empty(5, device="cuda") for _ in range(3)] + [torch.empty(1, device="cuda")]
            gpu_lib.moe_policy_loss(ctx, z, dev("target"), dev("old"), dev("ref"), dev("A"), dev("w"), *o, z, **PARAMS)
            for a, b in zip(o + [z], want):
                assert torch.equal(a, b)


def test_terms_one_at_a_time_and_bounds_of_rows(gpu_lib):
    n = _inputs(64, 777, "f32", 5)
    rng = np.random.default_rng(6)
    clip = rng.uniform(0.01, 0.4, 64).astype(np.float32)
    with Context(gpu_lib) as ctx:
        _compare(n, _call(gpu_lib, ctx, n, "f32", ref=False, clip_low=0.1, clip_high=0.3), "f32", "f32", ref=False, clip_low=0.1, clip_high=0.3)
        none = dict(clip_low=0.0, clip_high=0.0)
        _compare(n, _call(gpu_lib, ctx, n, "f32", kl_coef=0.5, **none), "f32", "f32", kl_coef=0.5, **none)
        _compare(n, _call(gpu_lib, ctx, n, "f32", ref=False, entropy_coef=0.5, **none), "f32", "f32", ref=False, entropy_coef=0.5, **none)
        c = clip.astype(np.float64)
        _compare(n, _call(gpu_lib, ctx, n, "f32", clip_rows=clip, clip_low=9.0, clip_high=9.0), "f32", "f32", clip_low=c, clip_high=c)


def test_bad_logits_stay_in_their_rows(gpu_lib):
    n = _inputs(6, 2000, "bf16", 7)
    n["w"][:] = 0.5
    n["z"][1, 5], n["z"][4, 70] = float("nan"), float("inf")
    with Context(gpu_lib) as ctx:
        logp, H, loss, total, g = _call(gpu_lib, ctx, n, "bf16", **PARAMS)
    for r in (1, 4):
        assert logp[r].isnan() and loss[r].isnan() and g[r].isnan().all()
    assert total.isnan().all()
    fine = [0, 2, 3, 5]
    m = {k: v[fine] for k, v in n.items()}
    _compare(m, [logp[fine], H[fine], loss[fine], loss[fine].sum()[None], g[fine]], "bf16", "bf16", **PARAMS)


def test_gradient_against_differences_of_the_kernels_own_loss(gpu_lib):
    """Directional differences in fp32: the loss changes by the gradient's product with a step, up to second order and fp32's resolution."""
    n = _inputs(48, 311, "f32", 8)
    logp = tr.policy_loss(f64(n["z"]), n["target"], n["old"], None, n["A"], n["w"], 0, 0, 0, 0, 0.8)[0]
    n["old"] = (logp + np.where(np.arange(48) % 2, 0.05, 0.6)).astype(np.float32)     # far from the clip bounds
    with Context(gpu_lib) as ctx:
        g = f64(_call(gpu_lib, ctx, n, "f32", **PARAMS)[4])
        rng = np.random.default_rng(9)
        for _ in range(3):
            v = rng.normal(size=g.shape)
            h, z = 2.0 ** -9, n["z"]
            step = torch.from_numpy(v).float() * h
            ends = []
            for sign in (1, -1):
                n["z"] = z + sign * step
                ends.append(f64(_call(gpu_lib, ctx, n, None, **PARAMS)[2]).sum())
            n["z"] = z
            slope = (ends[0] - ends[1]) / (2 * h)
            assert abs(slope - (g * v).sum()) <= 1e-3 * np.sqrt((g ** 2).sum()) * np.sqrt(g.size) / 17 + 1e-3, (slope, (g * v).sum())


def test_no_rows_and_refusals(gpu_lib):
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    loss = torch.full((1,), 7.0, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_policy_loss(ctx, f(0, 10), i(0), f(0), None, f(0), f(0), f(0), f(0), f(0), loss)
        assert loss[0] == 0
        base = lambda: [f(4, 10), i(4), f(4), f(4), f(4), f(4), f(4), f(4), f(4), f(1)]  # noqa: E731

        def refused(change=None, **kw):
            args = base()
            for k, v in (change or {}).items():
                args[k] = v
            with pytest.raises(gpu_lib.MoEError):
                gpu_lib.moe_policy_loss(ctx, *args, **kw)
        for kw in (dict(clip_low=-0.1), dict(clip_high=float("nan")), dict(kl_coef=float("inf")), dict(entropy_coef=-1.0), dict(temperature=0.0),
                   dict(temperature=float("nan")), dict(temperature=1e-45), dict(dlogits=f(4, 11)), dict(dlogits=f(4, 10).half()),
                   dict(clip_rows=f(5))):
            refused(**kw)
        for change in ({0: f(4, 10).half()}, {0: f(10, 4).t()}, {1: i(3)}, {1: f(4)}, {2: f(5)}, {4: None}, {5: None}, {6: f(3)}, {9: f(2)}, {0: f(4, 0)}):
            refused(change)
    with Context(gpu_lib, reserve=False) as ctx, pytest.raises(gpu_lib.MoEError):
        gpu_lib.moe_policy_loss(ctx, *base())
