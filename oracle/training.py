"""What stands around a replayed layer in training, in fp64: norm with residual and e4m3 output, token order, combine's gradient, policy
loss, and the gradients of the block-scaled linear.  Plain numpy from the definitions; shares no code with the HIP path.

Arrays are float64 unless said otherwise; e4m3 operands come as codes (uint8) with their scales.
"""
from __future__ import annotations

import numpy as np

from . import fp_formats as ff

BLOCK = 128
MASKED = -1e30                                                  # logits up to it are masked


def add_rmsnorm(x, residual, gain, eps, keep):
    """(h, y, r); keep(v): v as the sum's type holds it."""
    h = x if residual is None else keep(x + residual)
    r = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h, h * r[:, None] * gain, r


def group_scales(y):
    """[cols/128, rows]: amax/448 of each row's groups of 128 columns, 1 for a group of zeros."""
    amax = np.abs(y.reshape(y.shape[0], -1, BLOCK)).max(axis=2)
    return np.where(amax == 0, 1.0, amax / 448.0).T


def add_rmsnorm_backward(dy, h, r, gain, dh):
    """(dx, dgain)"""
    u = dy * gain
    dx = r[:, None] * u - h * (r ** 3 * (u * h).sum(axis=1) / h.shape[1])[:, None]
    return (dx if dh is None else dx + dh), (dy * h * r[:, None]).sum(axis=0)


def dispatch(x, inv_perm, k, fill):
    out = np.full((x.shape[0] * k, x.shape[1]), fill, np.float64)
    for i, p in enumerate(inv_perm):
        if p >= 0:
            out[p] = x[i // k]
    return out


def dispatch_backward(dx_perm, inv_perm, k, dx_add):
    T = len(inv_perm) // k
    dx = np.zeros((T, dx_perm.shape[1])) if dx_add is None else dx_add.copy()
    for i, p in enumerate(inv_perm):
        if p >= 0:
            dx[i // k] += dx_perm[p]
    return dx


def combine_backward(dy, y_perm, inv_perm, topk_w, topk_idx, E, fill):
    """(dy_perm, dw, dlogits); rows that no slot names hold `fill`."""
    T, k = topk_w.shape
    dy_perm, dw, dlogits = np.full(y_perm.shape, fill, np.float64), np.zeros((T, k)), np.zeros((T, E))
    for i, p in enumerate(inv_perm):
        if p >= 0:
            t, j = divmod(i, k)
            dy_perm[p] = topk_w[t, j] * dy[t]
            dw[t, j] = dy[t] @ y_perm[p]
    dl = topk_w * (dw - (topk_w * dw).sum(axis=1, keepdims=True))
    for t in range(T):
        for j in range(k):
            if 0 <= topk_idx[t, j] < E:
                dlogits[t, topk_idx[t, j]] += dl[t, j]
    return dy_perm, dw, dlogits


def policy_loss(logits, target, old_logp, ref_logp, advantage, weight, low, high, kl_coef, entropy_coef, temperature):
    """(logp, entropy, row_loss, dlogits); low, high: a number or one for each row."""
    rows, V = logits.shape
    low, high = np.broadcast_to(low, rows), np.broadcast_to(high, rows)
    logp, entropy, row_loss, grad = np.zeros(rows), np.zeros(rows), np.zeros(rows), np.zeros((rows, V))
    for t in range(rows):
        known, m = 0 <= target[t] < V, logits[t].max()
        if m <= MASKED:
            logp[t] = -np.inf if known else 0.0
            continue
        z = np.where(logits[t] > MASKED, (logits[t] - m) / temperature, -np.inf)               # (the maximum first: large logits differ by little)
        ls = z - np.log(np.exp(z).sum())
        p = np.exp(ls)
        plogp = np.zeros(V)
        plogp[p > 0] = p[p > 0] * ls[p > 0]
        H = entropy[t] = -plogp.sum()
        if not known:
            continue
        lp = logp[t] = ls[target[t]]
        if weight[t] == 0 or lp == -np.inf:                    # (a masked target has no effect)
            continue
        A, loss, slope = advantage[t], 0.0, 0.0
        if A != 0:
            rho = np.exp(lp - old_logp[t])
            free, held = rho * A, min(max(rho, 1 - low[t]), 1 + high[t]) * A
            loss, slope = -min(free, held), (-free if free <= held else 0.0)
        if ref_logp is not None:
            x = ref_logp[t] - lp
            loss += kl_coef * (np.expm1(x) - x)
            slope += kl_coef * (1 - np.exp(x))
        row_loss[t] = weight[t] * (loss - entropy_coef * H)
        g = -p * slope + entropy_coef * (plogp + p * H)
        g[target[t]] += slope
        grad[t] = weight[t] * g / temperature
    return logp, entropy, row_loss, grad


def block_weights(Wq, ws):
    """[NOUT, K] of e4m3 codes and the scales of 128 x 128 blocks"""
    return ff.e4m3_decode(Wq) * np.kron(ws.astype(np.float64), np.ones((BLOCK, BLOCK)))


def activations(xq, xs):
    """[rows, K] of e4m3 codes and group-major scales"""
    return ff.e4m3_decode(xq) * np.repeat(xs.astype(np.float64), BLOCK, axis=0).T


def linear_backward(dy, Wq, ws, xq, xs, offsets):
    """(dx, dW): one matrix per expert; Wq [E,NOUT,K]"""
    x = activations(xq, xs)
    dx, dW = np.zeros(x.shape), np.zeros(Wq.shape)
    for e in range(Wq.shape[0]):
        at = slice(offsets[e], offsets[e + 1])
        dx[at] = dy[at] @ block_weights(Wq[e], ws[e])
        dW[e] = dy[at].T @ x[at]
    return dx, dW
