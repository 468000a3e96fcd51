"""The two ends of a policy step around the layer, in fp64: embedding and its gradient, token log-probabilities with the most likely tokens and their
gradient, gradient norm and clipping.  Plain numpy from the definitions; shares no code with the HIP path.
"""
from __future__ import annotations

import numpy as np

from .training import MASKED


def embed(ids, table, scale):
    y = np.zeros((len(ids), table.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < len(table):
            y[t] = scale * table[v]
    return y


def embed_backward(dy, ids, scale, dtable, accumulate):
    """dtable [V, d] before the call: added to, or taken for its shape."""
    out = dtable.copy() if accumulate else np.zeros(dtable.shape)
    for t, v in enumerate(ids):
        if 0 <= v < len(out):
            out[v] += scale * dy[t]
    return out


def _log_softmax(z, temperature):
    """(log p, max, sum of exponentials) of one row; masked logits have log p = -inf.  None: all are masked"""
    m = z.max()
    if m <= MASKED:
        return None
    x = np.where(z > MASKED, (z - m) / temperature, -np.inf)
    s = np.exp(x).sum()
    return x - np.log(s), m, s


def token_logp(logits, ids, n, temperature):
    """(logp [rows, m], entropy [rows], top_idx [rows, n], top_logp [rows, n], stats [rows, 2])"""
    rows, V = logits.shape
    logp, entropy = np.zeros(ids.shape), np.zeros(rows)
    top_idx, top_logp = np.full((rows, n), -1), np.full((rows, n), -np.inf)
    stats = np.tile([-np.inf, 0.0], (rows, 1))
    for t in range(rows):
        got = _log_softmax(logits[t], temperature)
        known = (ids[t] >= 0) & (ids[t] < V)
        if got is None:
            logp[t][known] = -np.inf
            continue
        lp, *stats[t] = got
        logp[t][known] = lp[ids[t][known]]
        p = np.exp(lp)
        entropy[t] = -(p[p > 0] * lp[p > 0]).sum()
        best = np.lexsort((np.arange(V), -logits[t]))          # by descending logit, then by index
        best = best[logits[t][best] > MASKED][:n]
        top_idx[t, :len(best)], top_logp[t, :len(best)] = best, lp[best]
    return logp, entropy, top_idx, top_logp, stats


def token_logp_backward(logits, ids, dlogp, dentropy, temperature):
    rows, V = logits.shape
    grad = np.zeros((rows, V))
    for t in range(rows):
        got = _log_softmax(logits[t], temperature)
        if got is None:
            continue
        lp = got[0]
        p = np.exp(lp)
        for j, v in enumerate(ids[t]):
            if dlogp is not None and 0 <= v < V and lp[v] != -np.inf:      # (a masked token has no effect)
                grad[t] -= dlogp[t, j] * p
                grad[t, v] += dlogp[t, j]
        if dentropy is not None:
            plogp = np.zeros(V)
            plogp[p > 0] = p[p > 0] * lp[p > 0]
            grad[t] -= dentropy[t] * (plogp - p * plogp.sum())
    return grad / temperature


def clip(grads, max_norm):
    """(sum of squares, scaled gradients)"""
    sum_sq = sum(float((g * g).sum()) for g in grads)
    factor = 1.0 if sum_sq == 0 else min(1.0, max_norm / np.sqrt(sum_sq))
    return sum_sq, [g * factor for g in grads]
