"""The distillation oracle against what its definitions imply (CPU)."""
import numpy as np
import pytest

from oracle import distill


def make(T, V, K, seed):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 2, (T, V))
    t = z + rng.normal(0, 1, (T, V))
    lt = t - np.log(np.exp(t).sum(1, keepdims=True))
    ids = np.argsort(-lt, axis=1)[:, :K]
    return z, ids, np.take_along_axis(lt, ids, 1), lt


@pytest.mark.parametrize("mode", [distill.GIVEN, distill.NORMALIZED, distill.REST])
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_gradient_against_differences(mode, tau):
    z, ids, lp, _ = make(3, 9, 4, 5)
    ids[1, 2] = ids[1, 0]                                            # a token listed twice
    ids[2, 3] = -1
    g = distill.distill_topk(z, ids, lp, mode, tau)["dz"]
    h = 1e-5
    for v in range(z.shape[1]):
        d = np.zeros_like(z)
        d[:, v] = h
        up, dn = (distill.distill_topk(z + s * d, ids, lp, mode, tau)["loss"] for s in (1, -1))
        # central differences: h^2 / 6 times a third derivative of order 1 / tau^3, and 1e-16 / h of rounding
        assert np.abs((up - dn) / (2 * h) - g[:, v]).max() < 1e-9


def test_all_listed_is_the_whole_divergence():
    z, ids, lp, lt = make(4, 7, 7, 1)
    o = distill.distill_topk(z, ids, lp, distill.REST, 1.0)
    ls = z - np.log(np.exp(z).sum(1, keepdims=True))
    assert np.allclose(o["loss"], (np.exp(lt) * (lt - ls)).sum(1), atol=1e-12) and (o["r"] == 0).all()
    assert np.allclose(o["dz"], np.exp(ls) - np.exp(lt), atol=1e-12)


def test_equal_distributions_have_no_loss():
    z, _, _, _ = make(4, 30, 5, 2)
    lz = z - np.log(np.exp(z).sum(1, keepdims=True))
    ids = np.argsort(-lz, axis=1)[:, :5]
    for mode in (distill.REST, ):
        o = distill.distill_topk(z, ids, np.take_along_axis(lz, ids, 1), mode, 1.0)
        assert np.abs(o["loss"]).max() < 1e-12 and np.abs(o["dz"]).max() < 1e-12


def test_rows_with_nothing():
    z, ids, lp, _ = make(4, 6, 2, 3)
    ids[0] = -1
    z[1] = -np.inf
    z[2, 0] = np.nan
    for mode in range(3):
        o = distill.distill_topk(z, ids, lp, mode, 1.0)
        assert o["loss"][0] == 0 and (o["dz"][0] == 0).all()
        assert o["loss"][1] == np.inf and o["lse"][1] == -np.inf and (o["dz"][1] == 0).all()
        assert np.isnan(o["loss"][2]) and np.isnan(o["dz"][2]).all()
