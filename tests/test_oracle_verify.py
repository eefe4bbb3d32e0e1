"""The verification oracle: the tokens it yields are distributed as the target's own samples (CPU)."""
import numpy as np
import pytest

from oracle import verify


@pytest.mark.parametrize("copied", [False, True])
def test_first_token_is_a_sample_of_the_target(copied):
    rng = np.random.default_rng(0)
    V, B = 6, 40000
    t, d = rng.normal(0, 1, V), rng.normal(0, 1, V)
    p, q = np.exp(t) / np.exp(t).sum(), np.exp(d) / np.exp(d).sum()
    drafts = np.full(B, 2) if copied else rng.choice(V, size=B, p=q)
    o = verify.verify_drafts(np.tile(t, (2 * B, 1)), None if copied else np.tile(d, (B, 1)), drafts, np.arange(B + 1), rng.random(B),
                             rng.exponential(size=(B, V)), 1.0, 1.0)
    first = o["tokens"][0::2]
    got = np.bincount(first, minlength=V) / B
    assert np.abs(got - p).max() < 5 * np.sqrt(0.25 / B)             # five standard deviations
    rate = np.minimum(p, q).sum() if not copied else p[2]
    assert abs(o["n_accepted"].mean() - rate) < 5 * np.sqrt(0.25 / B)


def test_same_policies_accept_everything():
    rng = np.random.default_rng(1)
    V, n = 9, 5
    z = rng.normal(0, 1, (n + 1, V))
    drafts = rng.integers(0, V, n)
    o = verify.verify_drafts(z, z[:n], drafts, np.array([0, n]), rng.random(n), rng.exponential(size=(1, V)), 0.7, 0.7)
    assert o["n_accepted"][0] == n and list(o["tokens"][:n]) == list(drafts)
    lp = z / 0.7 - np.log(np.exp(z / 0.7).sum(1, keepdims=True))
    assert np.allclose(o["logp"][:n], lp[np.arange(n), drafts])
