"""The largest logit that the scoring call keeps for its gradient is an entry of the row, bit for bit: every kernel, with and without
alternatives, rows far from zero and mostly masked."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


@pytest.mark.parametrize("V", [1, 7, 40, 250, 500, 1000, 2000, 4000, 5000, 9001, 30001, 100003])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0.0, -500.0, 3e5])
def test_largest_logit(B, V, dtype, shift):
    per = 16 // dtype.itemsize
    ld = (V + per - 1) // per * per
    for T in (3, 64, 700):
        g = torch.Generator(device="cuda").manual_seed(V + T)
        z = (torch.empty(T, ld, device="cuda").normal_(0.0, 3.0, generator=g) + shift).to(dtype)
        z[T // 2, :V - 1] = -math.inf
        y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=g)
        most = z[:, :V].float().amax(1)
        f = lambda *n: torch.full(n, -7.5, device="cuda")
        for k in (0, 1, 5, 20):
            if k > V:
                continue
            ids = torch.zeros(T, max(k, 1), dtype=torch.int32, device="cuda")
            for entropy in (None, f(T)):
                for target in (y, None):
                    stats = f(T, 4)
                    B.token_logprobs(B.LogprobParams(T, V, B.BF16 if dtype is torch.bfloat16 else B.F32, ld, k, 0, 1.0), z, target, None,
                                     f(T) if target is not None else None, entropy, f(T), ids if k else None, f(T, k) if k else None, stats)
                    assert torch.equal(stats[:, 0], most), (T, k, entropy is None, target is None)
