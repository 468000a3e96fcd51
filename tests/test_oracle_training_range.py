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
