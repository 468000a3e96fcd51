"""moe_policy_loss on logits of any size: large ones, small and large temperatures, finite masks, rows shifted by a constant; in each form of the kernel."""
import numpy as np
import pytest
import torch

from oracle import training as tr
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded

pytestmark = pytest.mark.gpu
# a row in registers; a row read twice; few rows in parts (the gradient in a second launch)
FORMS = {"held": (64, 1000), "held-wide": (40, 30011), "streamed": (136, 70001), "parts": (24, 40003)}
PARAMS = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05, entropy_coef=0.01)


def _rows(rows, V, T, type, seed):
    """Rows of many kinds, and targets that have some probability where the row leaves a choice"""
    rng = np.random.default_rng(seed)
    z = np.empty((rows, V), np.float32)
    target = rng.integers(0, V, rows).astype(np.int32)
    pairs = [(9321, 1), (5321, 1), (30000, 20000), (20.3, 10), (10.3, 1), (1e30, -9e29), (-9e29, -9.9e29)]
    fills = [-1e9, -1e10, -1e29, 1e10, 1e30, 0.0]
    for r in range(rows):
        kind = r % 20
        if kind < len(pairs):                                  # one large logit; the others are lower
            z[r] = pairs[kind][1]
            z[r, target[r]] = pairs[kind][0]
        elif kind < len(pairs) + len(fills):                   # all alike
            z[r] = fills[kind - len(pairs)]
        elif kind == 13:                                       # a finite mask on most of the row
            z[r] = -1e9
            z[r, rng.integers(0, V, 20)] = rng.normal(size=20) * T
            z[r, target[r]] = 2 * T
        elif kind == 14:                                       # nothing but finite masks of two sizes
            z[r] = rng.choice([-1e9, -1e10], V)
            z[r, target[r]] = -1e9
        else:                                                  # ordinary distances, in units of the temperature, around any value
            z[r] = rng.normal(size=V) * 2.5 * T + [0, 100, -7000, 1e5, -1e6][kind - 15] * T
            z[r, target[r]] = z[r].max()
    return torch.from_numpy(z).to(TYPES[type]), target


def _distance(z, T):
    """(p, distance from the row's maximum in nats, 0 where p is), of fp64 logits"""
    x = (z.max(axis=1, keepdims=True) - z) / T
    e = np.exp(-x)
    p = e / e.sum(axis=1, keepdims=True)
    return p, np.where(p > 0, x, 0.0)


def _call(moe, ctx, z, n, grad, **params):
    rows, V = z.shape
    dev = {k: torch.from_numpy(v).cuda() for k, v in n.items()}
    outs = [guarded((rows,), torch.float32) for _ in range(3)] + [guarded((1,), torch.float32)]
    g, check_g = guarded((rows, V), TYPES[grad]) if grad else (None, lambda: None)
    moe.moe_policy_loss(ctx, z.cuda(), dev["target"], dev["old"], dev["ref"], dev["A"], dev["w"], *(o for o, _ in outs), g, **params)
    torch.cuda.synchronize()
    for _, check in outs:
        check()
    check_g()
    return [o for o, _ in outs] + [g]


def _inputs(z, target, T, seed):
    rng = np.random.default_rng(seed)
    rows, zero = len(target), np.zeros(len(target))
    logp = tr.policy_loss(f64(z), target, zero, None, zero, zero, 0, 0, 0, 0, T)[0]
    f = lambda v: v.astype(np.float32)  # noqa: E731
    return dict(target=target, old=f(logp + rng.normal(size=rows) * 0.2), ref=f(logp + rng.normal(size=rows) * 0.3), A=f(rng.normal(size=rows)),
                w=f(0.1 + rng.random(rows)))


def _compare(z, n, got, grad, T):
    logp, H, loss, total, g = got
    z = f64(z)
    arg = [n[k].astype(np.float64) for k in ("old", "ref", "A", "w")]
    logp_o, H_o, loss_o, g_o = tr.policy_loss(z, n["target"], *arg, *PARAMS.values(), T)
    p, x = _distance(z, T)
    at = np.arange(len(z))
    # In fp32: a distance, the factor on it (three roundings) and their product make the exponent, off by five roundings of itself; 2^y two more; the sum
    # of a row a chain of at most 128 additions, a tree over a block, and as many again where a larger maximum turns up on the way
    mean, square = (p * x).sum(axis=1), (p * x * x).sum(axis=1)
    e_log = F32 * (5 * mean + 300)
    e_logp = e_log + F32 * (2 * x[at, n["target"]] + np.abs(logp_o))
    assert (np.abs(f64(logp) - logp_o) <= e_logp).all(), np.abs((f64(logp) - logp_o) / e_logp).max()
    e_H = 2 * e_log + F32 * (300 * mean + 8 * square + 2 * H_o) + mean * e_log
    assert (np.abs(f64(H) - H_o) <= e_H).all(), np.abs((f64(H) - H_o) / e_H).max()
    old, ref, A, w = arg
    rho, back = np.exp(logp_o - old), np.exp(ref - logp_o)
    e_rho = rho * (e_logp + 4 * F32)
    e_loss = w * (np.abs(A) * e_rho + 0.05 * (1 + back) * 2 * e_logp + 0.01 * e_H) + 8 * F32 * w * (np.abs(A) * rho + 1)
    assert (np.abs(f64(loss) - loss_o) <= e_loss).all()
    assert abs(float(total[0]) - loss_o.sum()) <= e_loss.sum() + F32 * np.abs(loss_o).sum()
    if g is None:
        return
    slope = w * (np.abs(A) * rho + 0.05 * (1 + back))
    e_slope = w * (np.abs(A) * e_rho + 0.05 * back * 2 * e_logp) + 8 * F32 * slope
    rel = (5 * x + 16) * F32 + e_log[:, None]
    size = slope[:, None] + (w * 0.01)[:, None] * (x + np.log(z.shape[1]) + H_o[:, None] + 1)
    bound = p * (2 * rel * size + e_slope[:, None] + (w * 0.01 * (e_H + e_log))[:, None])
    bound[at, n["target"]] += e_slope + 4 * F32 * slope
    assert (np.abs(f64(g) - g_o) <= bound / T + HALF_ULP[grad] * 1.01 * np.abs(g_o) + 2e-38).all()


@pytest.mark.parametrize("T", [1e-6, 1e-3, 1.0, 1e6])
@pytest.mark.parametrize("type,grad", [("f32", "f32"), ("bf16", "bf16"), ("f32", None)])
@pytest.mark.parametrize("form", FORMS)
def test_logits_of_any_size(gpu_lib, form, type, grad, T):
    T = float(np.float32(T))
    z, target = _rows(*FORMS[form], T, type, 1)
    n = _inputs(z, target, T, 2)
    with Context(gpu_lib) as ctx:
        got = _call(gpu_lib, ctx, z, n, grad, temperature=T, **PARAMS)
    _compare(z, n, got, grad, T)


@pytest.mark.parametrize("shift", [4096.0, -65536.0])
@pytest.mark.parametrize("form", FORMS)
def test_a_shift_changes_nothing(gpu_lib, form, shift):
    """log-softmax depends on differences alone: the same bits, where the shifted logits are exact"""
    rows, V = FORMS[form]
    rng = np.random.default_rng(3)
    z = torch.from_numpy((rng.integers(-2000, 2000, (rows, V)) / 128).astype(np.float32))
    n = _inputs(z, rng.integers(0, V, rows).astype(np.int32), 0.7, 4)
    with Context(gpu_lib) as ctx:
        want = _call(gpu_lib, ctx, z, n, "f32", temperature=0.7, **PARAMS)
        got = _call(gpu_lib, ctx, z + shift, n, "f32", temperature=0.7, **PARAMS)
    assert torch.equal((z + shift).double() - shift, z.double())
    for name, a, b in zip(("logp", "entropy", "row_loss", "loss", "dlogits"), got, want):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("T", [1e-6, 1.0])
def test_known_values(gpu_lib, T):
    """Rows whose log-probability is known without any sum: 0 next to far lower logits, -log V where all are alike"""
    V = 1000
    z = torch.full((6, V), 1.0)
    z[0, 7], z[1, 7], z[2, 7] = 9321.0, 5321.0, 30000.0
    z[3], z[4], z[5] = -1e9, -1e10, -1e29
    n = _inputs(z, np.full(6, 7, np.int32), T, 5)
    with Context(gpu_lib) as ctx:
        logp, H, _, loss, g = _call(gpu_lib, ctx, z, n, "f32", temperature=T, **PARAMS)
    assert (logp[:3] == 0).all() and (H[:3] == 0).all()
    assert (logp[3:] + np.log(V)).abs().max() <= 1e-5 and (H[3:] - np.log(V)).abs().max() <= 1e-5
    assert loss.isfinite().all() and g.isfinite().all()
