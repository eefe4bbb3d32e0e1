"""Refusals and host-side layout of the scoring operators: everything here returns before a launch (CPU)."""
import ctypes

import pytest
import torch

from paper_2603_04135_b200 import binding as B


def code(f, *a, **k):
    with pytest.raises(B.DppoError) as e:
        f(*a, **k)
    return e.value.code


def test_struct_layouts_match_header():
    assert ctypes.sizeof(B.LogprobParams) == 40 and B.LogprobParams.temperature.offset == 32 and B.LogprobParams.row_stride.offset == 16
    assert ctypes.sizeof(B.QuantizeParams) == 32 and B.QuantizeParams.q_stride.offset == 24
    assert ctypes.sizeof(B.LinearI8Params) == 48 and B.LinearI8Params.out_stride.offset == 32


P = 1 << 20      # an aligned address that is only looked at


@pytest.mark.parametrize("prm, want", [
    ((-1, 8, 1, 8, 0, 0, 1.0), B.ERR_INVALID_ARG), ((4, 0, 1, 8, 0, 0, 1.0), B.ERR_INVALID_ARG),
    ((4, 8, 2, 8, 0, 0, 1.0), B.ERR_UNSUPPORTED), ((4, 9, 1, 8, 0, 0, 1.0), B.ERR_BAD_SHAPE),
    ((4, 8, 1, 12, 0, 0, 1.0), B.ERR_MISALIGNED), ((4, 8, 1, 8, 33, 0, 1.0), B.ERR_INVALID_ARG),
    ((4, 8, 1, 8, -1, 0, 1.0), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 0, 0, 0.0), B.ERR_INVALID_ARG),
    ((4, 8, 1, 8, 0, 0, float("nan")), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 0, 0, float("inf")), B.ERR_INVALID_ARG),
    ((4, 8, 1, 8, 0, 0, 1e-7), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 0, 0, 1e7), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 0, 0, -1.0), B.ERR_INVALID_ARG),
    ((4, (1 << 30) + 8, 1, (1 << 30) + 8, 0, 0, 1.0), B.ERR_BAD_SHAPE), ((4, 8, 1, 8, 0, -1, 1.0), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 0, 30256, 1.0), B.ERR_UNSUPPORTED),
    ((4, 8, 1, 8, 0, 7, 1.0), B.ERR_UNSUPPORTED), ((1 << 31, 8, 1, 8, 0, 0, 1.0), B.ERR_BAD_SHAPE)])
def test_logprobs_params(prm, want):
    assert code(B.token_logprobs, B.LogprobParams(*prm), P, P, None, P, P, P, None, None, P) == want


def test_logprobs_arrays():
    prm = B.LogprobParams(4, 8, 1, 8, 2, 0, 1.0)
    assert code(B.token_logprobs, prm, None, P, None, P, P, P, P, P, P) == B.ERR_INVALID_ARG
    assert code(B.token_logprobs, prm, P + 8, P, None, P, P, P, P, P, P) == B.ERR_MISALIGNED
    assert code(B.token_logprobs, prm, P, P, None, P, P, P, P, P, P + 4) == B.ERR_MISALIGNED
    assert code(B.token_logprobs, prm, P, P, None, P, P, P, None, P, P) == B.ERR_INVALID_ARG    # top_k without ids
    assert code(B.token_logprobs, prm, P, None, None, P, P, P, P, P, P) == B.ERR_INVALID_ARG    # logp without tokens
    prm0 = B.LogprobParams(4, 8, 1, 8, 0, 0, 1.0)
    assert code(B.token_logprobs, prm0, P, P, None, P, P, P, P, P, P) == B.ERR_INVALID_ARG      # ids without top_k
    B.token_logprobs(B.LogprobParams(0, 8, 1, 8, 0, 0, 1.0), None, None, None, None, None, None, None, None, None)   # no rows


def test_backward_arrays():
    prm = B.LogprobParams(4, 8, 1, 8, 0, 0, 1.0)
    assert code(B.token_logprobs_backward, prm, P, P, None, None, P, P, P) == B.ERR_INVALID_ARG
    assert code(B.token_logprobs_backward, prm, P, P, None, P, P, P, None) == B.ERR_INVALID_ARG
    assert code(B.token_logprobs_backward, prm, P, None, None, P, P, None, P) == B.ERR_INVALID_ARG
    assert code(B.token_logprobs_backward, prm, P, P, None, P, P, P, P + 2) == B.ERR_MISALIGNED
    assert code(B.token_logprobs_backward, prm, P, P, None, P + 4, P, P, P) == B.ERR_MISALIGNED
    B.token_logprobs_backward(B.LogprobParams(0, 8, 1, 8, 0, 0, 1.0), None, None, None, None, None, None, None)


def test_quantize_params():
    q = B.quantize_rows_i8
    assert code(q, B.QuantizeParams(-1, 8, 1, 8, 16), P, P, P) == B.ERR_INVALID_ARG
    assert code(q, B.QuantizeParams(4, 0, 1, 8, 16), P, P, P) == B.ERR_INVALID_ARG
    assert code(q, B.QuantizeParams(4, 8, 5, 8, 16), P, P, P) == B.ERR_UNSUPPORTED
    assert code(q, B.QuantizeParams(4, 8, 1, 7, 16), P, P, P) == B.ERR_BAD_SHAPE
    assert code(q, B.QuantizeParams(4, 8, 1, 9, 16), P, P, P) == B.ERR_MISALIGNED
    assert code(q, B.QuantizeParams(4, 8, 1, 8, 8), P, P, P) == B.ERR_MISALIGNED
    assert code(q, B.QuantizeParams(4, 8, 1, 8, 16), P, P + 1, P) == B.ERR_MISALIGNED
    assert code(q, B.QuantizeParams(4, 8, 1, 8, 16), None, P, P) == B.ERR_INVALID_ARG
    assert code(q, B.QuantizeParams(1 << 31, 8, 1, 8, 16), P, P, P) == B.ERR_BAD_SHAPE
    assert code(q, B.QuantizeParams(4, (1 << 30) + 8, 1, (1 << 30) + 8, (1 << 30) + 16), P, P, P) == B.ERR_BAD_SHAPE    # column indices pass 31 bits
    q(B.QuantizeParams(0, 8, 1, 8, 16), None, None, None)


def test_linear_params():
    def lin(*prm, x=P, w=P, out=P, xs=P):
        return code(B.linear_i8, B.LinearI8Params(*prm), x, xs, w, P, out)
    assert lin(-1, 8, 16, 16, 16, 8, 0) == B.ERR_INVALID_ARG
    assert lin(4, 0, 16, 16, 16, 8, 0) == B.ERR_INVALID_ARG
    assert lin(4, 8, 0, 16, 16, 8, 0) == B.ERR_INVALID_ARG
    assert lin(4, 8, 16, 16, 16, 8, 7) == B.ERR_UNSUPPORTED
    assert lin(4, 8, 131072, 131072, 131072, 8, 0) == B.ERR_BAD_SHAPE      # int32 sums could overflow
    assert lin(4, 8, 17, 16, 32, 8, 0) == B.ERR_BAD_SHAPE
    assert lin(4, 8, 16, 16, 16, 7, 0) == B.ERR_BAD_SHAPE
    assert lin(4, 8, 16, 24, 16, 8, 0) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 0, x=P + 4) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 0, w=P + 4) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 0, out=None) == B.ERR_INVALID_ARG
    assert lin(4, 8, 16, 16, 16, 8, 0, xs=None) == B.ERR_INVALID_ARG
    for v in (-1, 3, 100, 103):
        assert lin(4, 8, 16, 16, 16, 8, 0, v) == B.ERR_INVALID_ARG
    B.linear_i8(B.LinearI8Params(0, 8, 16, 16, 16, 8, 0), None, None, None, None, None)


def test_binding_checks_tensors():
    prm = B.LogprobParams(4, 8, B.BF16, 8, 0, 0, 1.0)
    z = torch.zeros(4, 8, dtype=torch.bfloat16)
    assert code(B.token_logprobs, prm, z.float(), P, None, P, P, P, None, None, P) == B.ERR_INVALID_ARG      # type
    assert code(B.token_logprobs, prm, P, torch.zeros(4, dtype=torch.int64), None, P, P, P, None, None, P) == B.ERR_INVALID_ARG
    if torch.cuda.is_available():
        assert code(B.token_logprobs, prm, z, P, None, P, P, P, None, None, P) == B.ERR_INVALID_ARG          # device
        return
    assert code(B.token_logprobs, prm, z[:3].clone(), P, None, P, P, P, None, None, P) == B.ERR_BAD_SHAPE    # too few rows
    assert code(B.token_logprobs, prm, torch.zeros(8, 4, dtype=torch.bfloat16).t(), P, None, P, P, P, None, None, P) == B.ERR_BAD_SHAPE
    assert code(B.token_logprobs, prm, z, torch.zeros(3, dtype=torch.int32), None, P, P, P, None, None, P) == B.ERR_BAD_SHAPE
    assert code(B.token_logprobs, prm, z, torch.zeros(8, dtype=torch.int32)[::2], None, P, P, P, None, None, P) == B.ERR_BAD_SHAPE
