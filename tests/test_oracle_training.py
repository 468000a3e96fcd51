"""The oracle's gradients of the training side against central differences of its own forward definitions, in fp64."""
import numpy as np
import pytest

from oracle import fp_formats as ff
from oracle import training as tr

STEP = 1e-6


def _difference(f, x):
    """df/dx of a scalar f by central differences (error about STEP^2 and 1e-16/STEP, times the function's size)"""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        was = x[i]
        x[i] = was + STEP
        up = f()
        x[i] = was - STEP
        g[i] = (up - f()) / (2 * STEP)
        x[i] = was
    return g


def _close(a, b):
    assert np.abs(a - b).max() <= 1e-7 * (1 + np.abs(b).max()), np.abs(a - b).max()


def test_norm_gradient():
    rng = np.random.default_rng(1)
    x, gain, dy, dh = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))

    def value():
        h, y, _ = tr.add_rmsnorm(x, None, gain, 1e-6, None)
        return (y * dy).sum() + (h * dh).sum()
    _, _, r = tr.add_rmsnorm(x, None, gain, 1e-6, None)
    dx, dgain = tr.add_rmsnorm_backward(dy, x, r, gain, dh)
    _close(dx, _difference(value, x))
    _close(dgain, _difference(value, gain))


@pytest.mark.parametrize("case", ["plain", "masked", "per_row_clip", "no_reference", "temperature"])
def test_policy_loss_gradient(case):
    rng = np.random.default_rng(2)
    rows, V = 12, 9
    z = rng.normal(size=(rows, V)) * 2
    target = rng.integers(0, V, rows)
    if case == "masked":
        for t in range(rows):
            z[t, (target[t] + 1 + t % (V - 1)) % V] = -np.inf
        target[3] = -100
    temp = 0.7 if case == "temperature" else 1.0
    logp = tr.policy_loss(z, target, np.zeros(rows), None, np.zeros(rows), np.zeros(rows), 0, 0, 0, 0, temp)[0]
    old = logp + rng.choice([-0.5, -0.1, 0.1, 0.5], rows)      # both sides of the clip bounds, and not at them
    ref = None if case == "no_reference" else logp + rng.normal(size=rows) * 0.3
    A, w = rng.choice([-1.0, 1.0, 0.5], rows), rng.choice([0.0, 0.1, 1.0], rows)
    low, high = (rng.uniform(0.15, 0.25, rows),) * 2 if case == "per_row_clip" else (0.2, 0.28)

    def value():
        return tr.policy_loss(z, target, old, ref, A, w, low, high, 0.05, 0.01, temp)[2].sum()
    g = tr.policy_loss(z, target, old, ref, A, w, low, high, 0.05, 0.01, temp)[3]
    live = np.isfinite(z)
    with np.errstate(invalid="ignore"):
        d = _difference(value, z)
    _close(g[live], d[live])
    assert (g[~live] == 0).all()
    assert np.abs(g.sum(axis=1)).max() < 1e-12                 # a shift of a row's logits changes nothing


def test_combine_and_router_gradient():
    rng = np.random.default_rng(3)
    T, k, E, d = 5, 3, 6, 4
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    inv = np.argsort(np.argsort(idx.reshape(-1), kind="stable"), kind="stable")
    y_perm, dy, logits = rng.normal(size=(T * k, d)), rng.normal(size=(T, d)), rng.normal(size=(T, E))

    def weights():
        chosen = np.exp(np.take_along_axis(logits, idx, axis=1))
        return chosen / chosen.sum(axis=1, keepdims=True)

    def value():
        return ((weights()[:, :, None] * y_perm[inv].reshape(T, k, d)).sum(axis=1) * dy).sum()
    dy_perm, dw, dlogits = tr.combine_backward(dy, y_perm, inv, weights(), idx, E, 0.0)
    _close(dy_perm, _difference(value, y_perm))
    _close(dlogits, _difference(value, logits))


def test_token_order_gradient():
    rng = np.random.default_rng(4)
    T, k, d = 4, 3, 5
    inv = rng.permutation(T * k)
    inv[5] = -1
    x, g = rng.normal(size=(T, d)), rng.normal(size=(T * k, d))
    missing = np.setdiff1d(np.arange(T * k), inv)
    g[missing] = 0
    _close(tr.dispatch_backward(g, inv, k, None), _difference(lambda: (tr.dispatch(x, inv, k, 0.0) * g).sum(), x))


def test_linear_gradient():
    rng = np.random.default_rng(5)
    rows, NOUT, K = 3, 128, 128
    Wq, xq = rng.integers(0, 127, (1, NOUT, K)).astype(np.uint8), rng.integers(0, 127, (rows, K)).astype(np.uint8)
    ws, xs = rng.uniform(0.5, 2, (1, 1, 1)) * 1e-3, rng.uniform(0.5, 2, (1, rows)) * 1e-3
    dy = rng.normal(size=(rows, NOUT))
    dx, dW = tr.linear_backward(dy, Wq, ws, xq, xs, [0, rows])
    x, W = tr.activations(xq, xs), tr.block_weights(Wq[0], ws[0])
    some = np.s_[:2, :3]
    xsome, Wsome = x[some].copy(), W[some].copy()

    def value_x():
        v = x.copy()
        v[some] = xsome
        return ((v @ W.T) * dy).sum()

    def value_W():
        v = W.copy()
        v[some] = Wsome
        return ((x @ v.T) * dy).sum()
    _close(dx[some], _difference(value_x, xsome))
    _close(dW[0][some], _difference(value_W, Wsome))
    assert np.isfinite(ff.e4m3_decode(Wq)).all()
