"""The oracle of the scoring operators against closed forms and finite differences (CPU)."""
import numpy as np
import pytest

from oracle import scoring


def test_uniform_and_peaked_rows():
    z = np.zeros((1, 7))
    r = scoring.token_logprobs(z, [3], 3, 0.5)
    assert np.allclose([r["logp"][0], r["entropy"][0], r["lse"][0]], [-np.log(7), np.log(7), np.log(7)])
    assert list(r["top_ids"][0]) == [0, 1, 2]                        # ties go to the lower index
    z = np.array([[1000.0, 0.0, -1000.0, -np.inf]])
    r = scoring.token_logprobs(z, [0], 4, 1.0)
    assert r["logp"][0] == 0.0 and abs(r["entropy"][0]) < 1e-300 and list(r["top_ids"][0]) == [0, 1, 2, -1]


def test_empty_and_invalid_rows():
    z = np.array([[-np.inf, -np.inf], [np.nan, 0.0], [np.inf, 0.0]])
    r = scoring.token_logprobs(z, [0, 0, 0], 1, 1.0)
    assert r["logp"][0] == -np.inf and r["lse"][0] == -np.inf and r["entropy"][0] == 0
    assert np.isnan(r["logp"][1:]).all() and (r["top_ids"] == -1).all() and np.isnan(r["top_logp"][1:]).all()


@pytest.mark.parametrize("tau", [0.5, 1.0, 1.7])
def test_gradient_against_differences(tau):
    rng = np.random.default_rng(0)
    z = rng.normal(size=(3, 9))
    y, a, b = np.array([0, 4, 8]), rng.normal(size=3), rng.normal(size=3)

    def f(z):
        r = scoring.token_logprobs(z, y, 0, tau)
        return (a * r["logp"] + b * r["entropy"]).sum()

    g = scoring.token_logprobs_backward(z, y, a, b, tau)
    h = 1e-6
    for t in range(3):
        for v in range(9):
            zp, zm = z.copy(), z.copy()
            zp[t, v] += h
            zm[t, v] -= h
            assert abs((f(zp) - f(zm)) / (2 * h) - g[t, v]) < 1e-7


def test_quantisation():
    x = np.array([[0.0, 0.0], [-254.0, 127.0], [1.0, np.inf], [0.5, 127.0], [1.5, 127.0]], dtype=np.float32)
    q, s = scoring.quantize_rows_i8(x)
    assert q.tolist() == [[0, 0], [-127, 64], [0, 0], [0, 127], [2, 127]]   # 63.5, 0.5, 1.5: ties to even
    assert s[0] == 0 and s[1] == 2 and np.isnan(s[2])
    y = scoring.linear_i8(q[1:2], s[1:2], np.array([[1, -1]], dtype=np.int8), np.array([0.25], dtype=np.float32))
    assert y.tolist() == [[-191 * 0.5]]
