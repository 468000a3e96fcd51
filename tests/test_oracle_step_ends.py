"""The oracle of the two ends of a policy step: gradients against central differences of its own forward definitions, in fp64, and small cases by hand."""
import numpy as np
import pytest

from oracle import step_ends as ends
from oracle import training as tr
from test_oracle_training import _close, _difference


def test_embedding_gradient():
    rng = np.random.default_rng(1)
    table, ids = rng.normal(size=(5, 3)), np.array([1, 4, 1, -1, 0, 5, 1])
    dy = rng.normal(size=(7, 3))

    def value():
        return (ends.embed(ids, table, 1.5) * dy).sum()
    _close(ends.embed_backward(dy, ids, 1.5, table, False), _difference(value, table))
    _close(ends.embed_backward(dy, ids, 1.5, table, True) - table, _difference(value, table))
    assert (ends.embed(ids, table, 2.0)[[3, 5]] == 0).all() and (ends.embed(ids, table, 2.0)[1] == 2 * table[4]).all()


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_token_logp_gradient(temperature):
    rng = np.random.default_rng(2)
    rows, V, m = 6, 9, 4
    z, ids = rng.normal(size=(rows, V)) * 2, rng.integers(0, V, (rows, m))
    ids[:, 3] = ids[:, 0]                                      # a token given twice
    ids[2, 1], ids[3, 0], ids[3, 3] = -5, V, V
    z[1, (ids[1].max() + 1) % V] = -np.inf
    z[4, ids[4, 2]] = -np.inf
    z[5] = -np.inf
    dlogp, dH = rng.normal(size=(rows, m)), rng.normal(size=rows)

    def value():
        logp, H = ends.token_logp(z, ids, 0, temperature)[:2]
        return np.where(np.isfinite(logp), logp * dlogp, 0).sum() + (H * dH).sum()
    with np.errstate(invalid="ignore"):
        _close(ends.token_logp_backward(z, ids, dlogp, dH, temperature), _difference(value, z))


def test_token_logp_is_the_policy_loss_own():
    rng = np.random.default_rng(3)
    z, ids = rng.normal(size=(5, 11)) * 3, rng.integers(0, 11, 5)
    z[2, :4] = -np.inf
    zeros = np.zeros(5)
    want = tr.policy_loss(z, ids, zeros, None, zeros, zeros, 0, 0, 0, 0, 0.8)[:2]
    got = ends.token_logp(z, ids[:, None], 3, 0.8)
    _close(np.where(np.isfinite(got[0][:, 0]), got[0][:, 0], -99), np.where(np.isfinite(want[0]), want[0], -99))
    _close(got[1], want[1])


def test_most_likely_tokens():
    z = np.array([[1.0, 3.0, -np.inf, 3.0, 2.0], [-np.inf] * 5])
    _, H, idx, lp, stats = ends.token_logp(z, np.zeros((2, 0), int), 6, 1.0)
    assert idx.tolist() == [[1, 3, 4, 0, -1, -1], [-1] * 6] and H[1] == 0 and stats[1].tolist() == [-np.inf, 0]
    assert np.isclose(np.exp(lp[0]).sum(), 1) and (lp[1] == -np.inf).all() and stats[0, 0] == 3


def test_clipping():
    g = [np.array([3.0]), np.array([]), np.array([0.0, 4.0])]
    assert ends.clip(g, 10.0)[0] == 25 and all((a == b).all() for a, b in zip(ends.clip(g, 10.0)[1], g))
    assert np.isclose(np.concatenate(ends.clip(g, 2.5)[1]), [1.5, 0, 2]).all()
    assert ends.clip([np.zeros(3)], 0.0)[1][0].tolist() == [0, 0, 0]
