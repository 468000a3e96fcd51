"""moe_token_logp and moe_token_logp_backward against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import step_ends as ends
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded, randn

pytestmark = pytest.mark.gpu
LOW = -1e30                                                    # logits up to it are masked
SHAPES = [(1, 1, 1, 1), (3, 2, 2, 5), (1, 9, 1, 0), (5, 63, 3, 64), (9, 512, 1, 20), (40, 1000, 64, 64), (7, 4099, 2, 7), (3, 32768, 1, 20), (2, 50001, 5, 33),
          (2, 131072, 1, 64), (300, 130, 4, 1), (700, 2500, 1, 8), (1, 262144, 0, 20), (64, 20000, 0, 0)]


def _ids(z, m, seed):
    return np.random.default_rng(seed).integers(0, z.shape[1], (z.shape[0], m)).astype(np.int32)


def _inputs(rows, V, m, type, seed, ties=False):
    z = randn((rows, V), type, seed, 2.5)
    if ties:
        z = torch.round(z * 2) / 2
        z[z == 0] = -0.0
        z[:, ::3] = z[:, ::3] + 0.0                            # zeros of both signs
    return z, _ids(z, m, seed)


def _strided(z, ld, at):
    wide = torch.full((z.shape[0], ld), 50.0, dtype=z.dtype, device="cuda")
    wide[:, at:at + z.shape[1]] = z
    return wide[:, at:at + z.shape[1]]


def _forward(moe, ctx, z, ids, n, temperature=1.0):
    rows, m = ids.shape
    out = [guarded((rows, m), torch.float32), guarded((rows,), torch.float32), guarded((rows, n), torch.int32, -7), guarded((rows, n), torch.float32),
           guarded((rows, 2), torch.float32)]
    t = [o for o, _ in out]
    moe.moe_token_logp(ctx, z.cuda(), torch.from_numpy(ids).cuda() if m else None, t[0] if m else None, t[1], t[2] if n else None, t[3] if n else None, t[4],
                       temperature=temperature)
    torch.cuda.synchronize()
    for _, check in out:
        check()
    return t


def _reach(z, temperature):
    """The largest distance of a logit that counts from its row's largest, in units of the temperature"""
    z = np.where(z > LOW, z, np.nan)
    with np.errstate(all="ignore"):
        m = np.where(np.isnan(z).all(axis=1), 0, np.nanmax(np.where(np.isnan(z), -np.inf, z), axis=1))
        x = (m[:, None] - z) / temperature
    return np.nanmax(np.where(x < 200, x, 0), axis=1, initial=0)   # (terms beyond are zero)


def _check_forward(z, ids, n, temperature, got):
    """Errors of fp32 sums over exponentials whose exponents carry three roundings of their distance from the largest logit.  Up to 1024 positive terms are
    added one after another: independent roundings, 0.29 * 2^-24 each in the mean square, make 9 * 2^-24 of that, seven times which is taken"""
    logp, H, idx, lp, stats = got
    z = f64(z)
    temperature = float(np.float32(temperature))
    logp_o, H_o, idx_o, lp_o, stats_o = ends.token_logp(z, ids, n, temperature)
    e_sum = ((4 * _reach(z, temperature) + 64) * F32)[:, None]

    def near(a, b):
        live = np.isfinite(b)
        assert np.array_equal(np.isfinite(a), live) and (a[~live] == b[~live]).all()
        e = np.broadcast_to(e_sum, b.shape) + 3 * F32 * np.abs(np.where(live, b, 0))
        assert (np.abs(a - b)[live] <= e[live]).all(), (np.abs(a - b)[live] / e[live]).max()
    near(f64(logp), logp_o)
    assert np.array_equal(idx.cpu().numpy(), idx_o)
    near(f64(lp), lp_o)
    assert (np.abs(f64(H) - H_o) <= (64 + 16 * _reach(z, temperature)) * F32 * (1 + np.abs(H_o) + _reach(z, temperature))).all()
    assert np.array_equal(f64(stats)[:, 0], stats_o[:, 0])
    assert (np.abs(f64(stats)[:, 1] - stats_o[:, 1]) <= e_sum[:, 0] * stats_o[:, 1]).all()


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(gpu_lib, shape, type, ties):
    rows, V, m, n = shape
    z, ids = _inputs(rows, V, m, type, 1, ties)
    with Context(gpu_lib) as ctx:
        got = _forward(gpu_lib, ctx, z, ids, n, 0.8)
        again = _forward(gpu_lib, ctx, z, ids, n, 0.8)
        _check_forward(z, ids, n, 0.8, got)
        for a, b in zip(got, again):
            assert torch.equal(a, b)
        for ld, at in ((V + 5, 3), (V + 8, 8)):
            for a, b in zip(got, _forward(gpu_lib, ctx, _strided(z, ld, at), ids, n, 0.8)):
                assert torch.equal(a, b)


def _order(rows, V, how, type):
    step = torch.arange(V).double()
    z = {"rising": step / V * 20, "falling": -step / V * 20, "equal": step * 0 + 3, "saw": (step % 17) + (step // 1000) / 1000,
         "late": torch.where(step > V - 70, step, step * 0), "two": (step == V - 1).double() + (step == 0).double()}[how]
    return z.repeat(rows, 1).to(TYPES[type])


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["rising", "falling", "equal", "saw", "late", "two"])
@pytest.mark.parametrize("rows,V,n", [(1, 70, 64), (2, 5000, 20), (2, 40000, 64), (1, 131072, 7), (600, 9001, 3)])
def test_alternatives_in_every_order(gpu_lib, rows, V, n, how, type):
    z = _order(rows, V, how, type)
    ids = _ids(z, 1, 2)
    with Context(gpu_lib) as ctx:
        _check_forward(z, ids, n, 1.0, _forward(gpu_lib, ctx, z, ids, n))


def _crowded(V, how, type):
    """Rows in which many logits reach what the first ones promise."""
    step, noise = torch.arange(V).double(), randn((V,), "f32", 21).double()
    z = {"rising": step / V * 20, "equal": step * 0 - 2, "rising noise": noise + step / V * 30, "steps": torch.floor(step / 5000), "noise": noise,
         "open behind": torch.where(step < V * 3 // 4, float("-inf"), noise), "one open, then equal": torch.where(step < 20000, float("-inf"), 1.0)}[how]
    if how == "one open, then equal":
        z[5] = 0.5
    z[V - 2] = float("-inf")
    return z.to(TYPES[type])


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["rising", "equal", "rising noise", "steps", "noise", "open behind", "one open, then equal"])
@pytest.mark.parametrize("rows,V", [(3, 270001), (130, 100003), (650, 50005)])
def test_many_alternatives_for_a_place(gpu_lib, rows, V, how, type):
    z = _crowded(V, how, type).reshape(1, V)
    ids = np.array([[7, V - 1]], dtype=np.int32)
    with Context(gpu_lib) as ctx:
        for n in (1, 33, 64):
            got = _forward(gpu_lib, ctx, z.repeat(rows, 1), np.tile(ids, (rows, 1)), n)
            _check_forward(z, ids, n, 1.0, [x[:1] for x in got])
            for x in got:
                assert torch.equal(x, x[:1].expand_as(x))


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 3001, 70000])
def test_masks(gpu_lib, V, type):
    """Masked by -inf and by the type's lowest value; rows with fewer open tokens than alternatives, with one, with none; given tokens that are masked or
    outside the vocabulary."""
    rows, n = 9, 24
    z, ids = _inputs(rows, V, 4, type, 3)
    low = torch.finfo(TYPES[type]).min
    g = torch.Generator().manual_seed(4)
    z[torch.rand((rows, V), generator=g) < 0.3] = -float("inf")
    z[torch.rand((rows, V), generator=g) < 0.1] = low
    z[0], z[1], z[2] = -float("inf"), low, -float("inf")
    z[2, V - 1] = -4.0
    z[3] = low
    z[3, ::V // 7] = torch.randn(len(range(0, V, V // 7)), generator=g).to(TYPES[type])
    z[4] = -1e29                                               # low, but open
    ids[5] = [-1, V, -2 ** 31, 2 ** 31 - 1]
    ids[6, 0], z[6, ids[6, 0]] = 5, low
    with Context(gpu_lib) as ctx:
        got = _forward(gpu_lib, ctx, z, ids, n, 0.9)
        _check_forward(z, ids, n, 0.9, got)
        dlogp, dH = randn((rows, 4), "f32", 5), randn((rows,), "f32", 6)
        dlogp[5], dlogp[6, 0] = float("nan"), float("inf")     # of tokens without effect
        grad = _backward(gpu_lib, ctx, z, ids, dlogp, dH, got, type, 0.9)
    clean = torch.nan_to_num(dlogp, nan=0.0, posinf=0.0)
    _check_backward(z, ids, clean, dH, 0.9, type, grad)
    assert (grad[z.cuda() <= LOW] == 0).all() and (grad[:2] == 0).all()


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 9000, 100000])
def test_nan_and_infinity(gpu_lib, V, type):
    """They spoil their own row, alternatives are the largest of the other logits."""
    z, ids = _inputs(6, V, 2, type, 7)
    clean = z.clone()
    z[1, 3], z[2, V - 1], z[4, V // 2] = float("nan"), float("inf"), float("nan")
    z[5] = float("nan")
    ids[1, 1] = -1
    with Context(gpu_lib) as ctx:
        logp, H, idx, lp, _ = _forward(gpu_lib, ctx, z, ids, 20)
        want = _forward(gpu_lib, ctx, clean, ids, 20)
    for r in (0, 3):
        for a, b in zip((logp, H, idx, lp), want):
            assert torch.equal(a[r], b[r])
    assert torch.isnan(logp[[1, 2, 4, 5], 0]).all() and torch.isnan(H[[1, 2, 4, 5]]).all() and logp[1, 1] == 0
    assert idx[2, 0] == V - 1 and (idx[5] == -1).all() and (lp[5] == -float("inf")).all() and torch.isnan(lp[[1, 2, 4]]).all()
    for r in (1, 4):
        rest = torch.where(torch.isnan(z[r]), torch.full_like(z[r], -float("inf")), z[r])
        assert torch.equal(idx[r].cpu().long(), torch.sort(rest, descending=True, stable=True).indices[:20])


def test_large_logits_and_temperatures(gpu_lib):
    """Errors go by a logit's distance from the largest: logits that a constant shifts exactly give the same bits."""
    z, ids = _inputs(6, 3000, 3, "f32", 8)
    z = torch.round(z * 64) / 64
    with Context(gpu_lib) as ctx:
        for temperature in (1e-6, 0.01, 1.0, 100.0, 1e6):
            a = _forward(gpu_lib, ctx, z, ids, 10, temperature)
            b = _forward(gpu_lib, ctx, z + 32768.0, ids, 10, temperature)
            _check_forward(z, ids, 10, temperature, a)
            for x, y in zip(a[:4], b[:4]):
                assert torch.equal(x, y)


def _backward(moe, ctx, z, ids, dlogp, dH, forward, out, temperature, in_place=False):
    rows, V = z.shape
    z = z.cuda().clone() if in_place else z.cuda()
    g, check = (z, lambda: None) if in_place else guarded((rows, V), TYPES[out])
    moe.moe_token_logp_backward(ctx, z, torch.from_numpy(ids).cuda() if ids.shape[1] else None, dlogp.cuda() if ids.shape[1] else None,
                                None if dH is None else dH.cuda(), forward[4], forward[1], g, temperature=temperature)
    torch.cuda.synchronize()
    check()
    return g


def _check_backward(z, ids, dlogp, dH, temperature, out, got):
    z, d = f64(z), f64(dlogp)
    temperature = float(np.float32(temperature))
    h = np.zeros(len(z)) if dH is None else f64(dH)
    want = ends.token_logp_backward(z, ids, d, h, temperature)
    rows, V = z.shape
    reach = _reach(z, temperature)
    with np.errstate(all="ignore"):
        m = z.max(axis=1, keepdims=True)
        x = np.where(z > LOW, (z - m) / temperature, -np.inf)
        p = np.exp(x) / np.maximum(np.exp(x).sum(axis=1, keepdims=True), 1e-300)
    p = np.where(np.isfinite(p), p, 0)
    x = np.where(p > 0, x, 0)
    H = np.log(V) + 1
    # p: the exponent's roundings and those of the sum; H: as the forward call gives it; the factors of p: roundings of their parts
    rel = (4 * np.abs(x) + 4 * reach[:, None] + 80) * F32
    size = np.abs(d).sum(axis=1)[:, None] + np.abs(h)[:, None] * (np.abs(x) + 2 * H + reach[:, None])
    bound = p * (size * rel + np.abs(h)[:, None] * (64 + 16 * reach[:, None]) * F32 * (1 + H + reach[:, None]))
    for j in range(ids.shape[1]):
        known = (ids[:, j] >= 0) & (ids[:, j] < V)
        bound[np.arange(rows)[known], ids[known, j]] += (ids.shape[1] + 4) * F32 * np.abs(d).sum(axis=1)[known]
    bound = bound / temperature + HALF_ULP[out] * 1.01 * np.abs(want) + 2e-38
    assert (np.abs(f64(got) - want) <= bound).all(), (np.abs(f64(got) - want) / bound).max()


@pytest.mark.parametrize("type,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(gpu_lib, shape, type, out):
    rows, V, m, _ = shape
    z, ids = _inputs(rows, V, m, type, 9)
    if m > 2:
        ids[:, 2] = ids[:, 0]                                  # given twice
    dlogp, dH = randn((rows, m), "f32", 10), randn((rows,), "f32", 11, 0.3)
    if rows > 4:
        dlogp[3], dH[3], dH[4] = 0, 0, 0                       # without effect, with one of them
    with Context(gpu_lib) as ctx:
        fwd = _forward(gpu_lib, ctx, z, ids, 0, 0.8)
        for h in (dH, None):
            g = _backward(gpu_lib, ctx, z, ids, dlogp, h, fwd, out, 0.8)
            assert torch.equal(g, _backward(gpu_lib, ctx, z, ids, dlogp, h, fwd, out, 0.8))
            _check_backward(z, ids, dlogp, h, 0.8, out, g)
            if rows > 4:
                assert (g[3] == 0).all()
            if type == out:
                assert torch.equal(g, _backward(gpu_lib, ctx, z, ids, dlogp, h, fwd, out, 0.8, in_place=True))


@pytest.mark.parametrize("type,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("V,m", [(1, 1), (70, 3), (1023, 2), (2048, 1)])
def test_backward_of_many_short_rows(gpu_lib, V, m, type, out):
    rows = 2050
    z, ids = _inputs(rows, V, m, type, 22)
    ids[::7] = -1
    dlogp, dH = randn((rows, m), "f32", 23), randn((rows,), "f32", 24)
    with Context(gpu_lib) as ctx:
        got = _forward(gpu_lib, ctx, z, ids, 0, 1.3)
        grad = _backward(gpu_lib, ctx, z, ids, dlogp, dH, got, out, 1.3)
        _check_backward(z, ids, dlogp, dH, 1.3, out, grad)


def test_rows_without_effect_are_zeros_whatever_they_hold(gpu_lib):
    z, ids = _inputs(4, 500, 2, "f32", 12)
    z[1] = float("nan")
    dlogp = randn((4, 2), "f32", 13)
    dlogp[1] = 0
    with Context(gpu_lib) as ctx:
        fwd = _forward(gpu_lib, ctx, z, ids, 0)
        g = _backward(gpu_lib, ctx, z, ids, dlogp, torch.zeros(4), fwd, "f32", 1.0)
    assert (g[1] == 0).all() and (g[[0, 2, 3]].abs().sum(dim=1) > 0).all()


def test_strided_gradients(gpu_lib):
    z, ids = _inputs(37, 1001, 3, "bf16", 14)
    dlogp, dH = randn((37, 3), "f32", 15), randn((37,), "f32", 16)
    with Context(gpu_lib) as ctx:
        fwd = _forward(gpu_lib, ctx, z, ids, 0)
        want = _backward(gpu_lib, ctx, z, ids, dlogp, dH, fwd, "bf16", 1.0)
        for ld, at in ((1006, 3), (1009, 8)):
            wide = torch.full((37, ld), 5.0, dtype=torch.bfloat16, device="cuda")
            gpu_lib.moe_token_logp_backward(ctx, _strided(z, 1010, 2), torch.from_numpy(ids).cuda(), dlogp.cuda(), dH.cuda(), fwd[4], fwd[1],
                                            wide[:, at:at + 1001])
            assert torch.equal(wide[:, at:at + 1001], want) and (wide[:, :at] == 5).all() and (wide[:, at + 1001:] == 5).all()
            wide[:, at:at + 1001] = z.cuda()                   # and in place
            gpu_lib.moe_token_logp_backward(ctx, wide[:, at:at + 1001], torch.from_numpy(ids).cuda(), dlogp.cuda(), dH.cuda(), fwd[4], fwd[1],
                                            wide[:, at:at + 1001])
            assert torch.equal(wide[:, at:at + 1001], want) and (wide[:, :at] == 5).all() and (wide[:, at + 1001:] == 5).all()


def test_gradient_against_differences_of_the_forward_call(gpu_lib):
    """Directional differences: the outputs' change in fp32, up to second order (h^2 |v|^3, a few 1e-5) and fp32's resolution over h."""
    rows, V, m = 24, 311, 4
    z, ids = _inputs(rows, V, m, "f32", 17)
    dlogp, dH = randn((rows, m), "f32", 18), randn((rows,), "f32", 19)
    with Context(gpu_lib) as ctx:
        fwd = _forward(gpu_lib, ctx, z, ids, 0, 0.8)
        g = f64(_backward(gpu_lib, ctx, z, ids, dlogp, dH, fwd, "f32", 0.8))
        for seed in range(3):
            v = torch.from_numpy(np.random.default_rng(seed).normal(size=g.shape)).float()
            h, ends_ = 2.0 ** -9, []
            for sign in (1, -1):
                logp, H = _forward(gpu_lib, ctx, z + sign * h * v, ids, 0, 0.8)[:2]
                ends_.append((f64(logp) * f64(dlogp)).sum() + (f64(H) * f64(dH)).sum())
            slope = (ends_[0] - ends_[1]) / (2 * h)
            size = np.abs(f64(dlogp)).sum() + 6 * np.abs(f64(dH)).sum()
            assert abs(slope - (g * f64(v)).sum()) <= size * (40 * F32 * 20 / h + 50 * h * h), (slope, (g * f64(v)).sum())
