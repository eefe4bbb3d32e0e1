"""Verification of drafts with noise of any positive size, uniforms of zero, and single sequences, on the GPU against the float64 oracle.

The bounds are those of test_gpu_verify.py; here every sequence has a margin (asserted), so that nothing is left out of the comparison.
"""
import math

import pytest
import torch

from test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


def check_all(c, out, least=1e-4):
    got, w = c.check(out)
    assert (w["margin"] >= least).all(), w["margin"].min()
    return got, w


def least_likely(c, row, among):
    """The token of the given ones that the target's row holds least likely, masked ones aside."""
    z = c.target[row, among].float()
    return int(among[int(torch.where(z > -math.inf, z, torch.full_like(z, math.inf)).argmin())])


# V: a row in one CTA's first vectors; rows of which most entries lie behind them
@pytest.mark.parametrize("V,dtype", [(7, "f32"), (1000, "f32"), (1000, "bf16"), (40000, "bf16"), (70001, "f32")])
@pytest.mark.parametrize("lens", [[0], [3]])
@pytest.mark.parametrize("tiny", [1e-20, 2.0 ** -127, 1e-39, 1e-42, 2.0 ** -149])
def test_tiny_noise(B, V, dtype, lens, tiny):
    c = Case(lens, V, dtype, False, 1.0, 1.0, V)
    c.u.fill_(0.0)                                                   # all drafts stand: the race is over the target's last row
    if lens[0]:
        c.u[1] = 0.999999                                            # ... or most likely over what is left of an earlier one
    last = sum(lens)
    for at in sorted({0, V // 2, V - 1, least_likely(c, last, torch.arange(V, device="cuda"))}):
        keep = float(c.noise[0, at])
        c.noise[0, at] = tiny
        got, w = check_all(c, c.run(B))
        if not lens[0]:
            assert int(got["tokens"][0]) == at
        c.noise[0, at] = keep


@pytest.mark.parametrize("V,dtype", [(1000, "f32"), (40000, "bf16")])
@pytest.mark.parametrize("size", [1e-44, 1e-38, 1e-30, 1e30, 1e38])
def test_all_of_the_noise_tiny_or_huge(B, V, dtype, size):
    c = Case([2, 0, 4], V, dtype, False, 1.0, 1.0, V + 1)
    if size > 1e-44:
        c.noise.clamp_(0.1, 3.0).mul_(size)
        check_all(c, c.run(B))
    else:                                                            # multiples of the smallest number: the same ratios for many entries
        c.noise.fill_(2.0 ** -149 * 9)
        c.noise[:, V // 3] = 2.0 ** -149
        c.target[:, V // 3] = c.target[:, :V].nan_to_num(nan=0.0).float().amax(1).to(c.target.dtype)
        c.u.fill_(0.0)
        got, _ = check_all(c, c.run(B))
        assert [int(got["tokens"][i]) for i in (2, 3, 8)] == [V // 3] * 3


def test_unlikely_token_with_noise_to_match(B):
    """p = e^-95 is below the normal f32 numbers; with noise below them too the token is ahead of the likely ones, or behind."""
    c = Case([0, 0], 5000, "f32", False, 1.0, 1.0, 11)
    c.target[:2, :5000] = 0.0
    c.target[:2, 4000] = -95.0
    c.noise[:2].clamp_(0.5, 2.0)
    c.noise[0, 4000], c.noise[1, 4000] = 2.0 ** -149, 2.0 ** -126
    got, w = c.check(c.run(B))
    assert w["margin"][0] > 0.1 and int(got["tokens"][0]) == 4000
    # the second sequence is a tie: the other tokens are alike, and the clamp has left many of them the same noise
    assert int(got["tokens"][1]) == w["tokens"][1] == int((c.noise[1, :5000] == 0.5).nonzero()[0])


@pytest.mark.parametrize("z", [-100.0, -690.0, -720.0, -900.0])
def test_a_uniform_of_zero_accepts_whatever_is_possible(B, z):
    """u q < p at u = 0 is 0 < p: true of every token that is not masked, also where p is below the f64 numbers."""
    V = 300
    c = Case([2], V, "f32", True, 1.0, 1.0, 12)
    c.target[:3, :V] = -math.inf
    c.target[:3, 5] = 0.0
    c.target[:3, 9] = z
    c.drafts[:2] = 9
    c.u[:2] = 0.0
    out = c.run(B)
    torch.cuda.synchronize()
    assert int(out["n"][0]) == 2 and out["tokens"][:3].tolist() == [9, 9, 5]
    assert out["logp"][:3].tolist() == [z, z, 0.0]
    c.target[1, 9] = -math.inf
    out = c.run(B)
    torch.cuda.synchronize()
    assert int(out["n"][0]) == 1 and out["tokens"][:3].tolist() == [9, 5, -1]


@pytest.mark.parametrize("lens,V,dtype,copied", [([4], 151936, "bf16", False), ([1], 33001, "bf16", False), ([0], 7, "f32", False), ([12], 50304, "f32", False),
                                                  ([40], 777, "bf16", True), ([2, 9], 5003, "f32", False)])
@pytest.mark.parametrize("seed", [21, 22, 23])
def test_single_sequences(B, lens, V, dtype, copied, seed):
    """Nothing is close here: the margins are asserted, and every count, token and log-prob is compared."""
    c = Case(lens, V, dtype, copied, 1.0, 1.0, seed * 1000 + V)
    check_all(c, c.run(B))
