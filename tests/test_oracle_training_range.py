"""The policy loss's oracle on large logits: it goes by differences from the row's maximum."""
import numpy as np

from oracle import training as tr


def test_shifted_and_large_rows():
    rng = np.random.default_rng(1)
    z = rng.integers(-2000, 2000, (5, 40)) / 128
    arg = (np.arange(5), rng.normal(size=5) - 4, rng.normal(size=5) - 4, rng.normal(size=5), np.ones(5), 0.2, 0.2, 0.1, 0.01, 0.5)
    want = tr.policy_loss(z, *arg)
    for shift in (4096.0, -2.0 ** 30):
        for a, b in zip(tr.policy_loss(z + shift, *arg), want):
            assert np.array_equal(a, b)
    for fill in (-1e9, -1e29, 1e30):
        logp, H, _, _ = tr.policy_loss(np.full((5, 40), fill), *arg)
        assert np.allclose(logp, -np.log(40)) and np.allclose(H, np.log(40))
    logp, H, loss, g = tr.policy_loss(np.full((5, 40), -3e38), *arg)                           # a mask, not a size
    assert (logp == -np.inf).all() and (H == 0).all() and (loss == 0).all() and (g == 0).all()


def test_masked_target_has_no_effect():
    rng = np.random.default_rng(2)
    z = rng.normal(size=(4, 30))
    z[0, 3], z[1, 3] = -np.inf, -3e38
    old, ref, A = (rng.normal(size=4) - 3 for _ in range(3))
    logp, H, loss, g = tr.policy_loss(z, np.full(4, 3), old, ref, A, np.ones(4), 0.2, 0.2, 0.1, 0.01, 0.5)
    assert (logp[:2] == -np.inf).all() and (loss[:2] == 0).all() and (g[:2] == 0).all() and (H > 0).all()
    assert np.isfinite(logp[2:]).all() and (loss[2:] != 0).all() and np.isfinite(g).all()
