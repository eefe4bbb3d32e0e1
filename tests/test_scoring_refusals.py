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


cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="looks at CPU tensors, which are on no current device there")
BF = torch.bfloat16


def not_held():
    """(tensor, rows, cols, stride): the tensor itself does not hold the rows, though its storage may."""
    buf = torch.zeros(8, 16, dtype=BF)
    seqs = torch.zeros(2, 5, 16, dtype=BF)
    return [
        (seqs[:, :-1], 8, 16, 16),                               # shifted by one: the second sequence's rows are elsewhere
        (seqs[:, 1:], 8, 16, 16),
        (seqs.transpose(0, 1), 10, 16, 16), (seqs.permute(2, 0, 1), 10, 16, 16),
        (torch.zeros(256, dtype=BF)[::2], 8, 16, 16),
        (buf[:5], 8, 16, 16), (buf[:5, :12], 8, 12, 16), (buf[3:, :12], 6, 12, 16),      # rows that were not passed
        (buf[:, :10], 8, 12, 16),                                # columns that were not passed
        (buf[:1], 2, 16, 16), (buf[0], 2, 16, 16), (buf.view(-1)[:100], 8, 16, 16),
        (buf.view(2, 4, 16)[:1], 8, 16, 16), (seqs[:, :, :12], 11, 12, 16),
        (buf.view(4, 32), 8, 16, 16), (buf.view(16, 8), 8, 16, 16),
        (buf[:1].expand(8, 16), 8, 16, 16), (buf.t(), 8, 8, 8), (buf[:, ::2], 8, 8, 16), (buf[::2], 4, 16, 16),
        (torch.zeros(40, dtype=BF).as_strided((2, 32), (8, 1)), 8, 8, 8),                # windows that overlap: 40 elements, 64 asked for
        (torch.zeros(0, 16, dtype=BF), 1, 16, 16), (torch.zeros(8, 0, dtype=BF), 8, 16, 16)]


def held():
    buf, seqs = torch.zeros(8, 16, dtype=BF), torch.zeros(2, 5, 16, dtype=BF)
    return [
        (buf, 8, 16, 16), (buf, 5, 12, 16), (buf[:5], 5, 16, 16), (buf[:, :12], 8, 12, 16), (buf[3:, :12], 5, 12, 16), (buf[::2], 4, 16, 32),
        (buf[2:3, :12], 1, 12, 16), (buf[2:3], 1, 12, 12), (buf[0], 1, 16, 16), (buf.view(-1), 8, 16, 16), (buf.view(-1)[:124], 8, 12, 16),
        (buf.view(1, -1), 8, 16, 16), (seqs, 10, 16, 16), (seqs[:, :, :12], 10, 12, 16), (seqs[:1, :4], 4, 16, 16), (seqs[0, 1:], 4, 16, 16),
        (buf.view(8, 1, 16), 8, 16, 16), (buf.view(8, 4, 4), 8, 16, 16), (buf.view(8, 4, 4)[:, :3], 8, 12, 16), (buf[:, :1], 8, 1, 16),
        (buf[:5], 0, 16, 16)]


@cpu_only
@pytest.mark.parametrize("case", range(len(not_held())))
def test_binding_refuses_tensors_that_do_not_hold_the_rows(case):
    x, rows, cols, stride = not_held()[case]
    assert code(B._mat, x, "x", -1, BF, rows, cols, stride) == B.ERR_BAD_SHAPE


@cpu_only
@pytest.mark.parametrize("case", range(len(held())))
def test_binding_takes_tensors_that_hold_the_rows(case):
    x, rows, cols, stride = held()[case]
    assert B._mat(x, "x", -1, BF, rows, cols, stride) == x.data_ptr()


@cpu_only
def test_every_matrix_argument_is_checked():
    """As input and as output, of each call: rows behind the tensor that is passed are not touched."""
    buf = torch.zeros(8, 16, dtype=BF)
    codes = torch.zeros(8, 16, dtype=torch.int8)
    prm = B.LogprobParams(8, 16, B.BF16, 16, 0, 0, 1.0)
    assert code(B.token_logprobs, prm, buf[:5], P, None, P, P, P, None, None, P) == B.ERR_BAD_SHAPE
    assert code(B.token_logprobs_backward, prm, buf[:5], P, None, P, P, P, buf) == B.ERR_BAD_SHAPE
    assert code(B.token_logprobs_backward, prm, buf, P, None, P, P, P, buf[:5]) == B.ERR_BAD_SHAPE
    q = B.QuantizeParams(8, 16, B.BF16, 16, 16)
    assert code(B.quantize_rows_i8, q, buf[:5], codes, P) == B.ERR_BAD_SHAPE
    assert code(B.quantize_rows_i8, q, buf, codes[:5], P) == B.ERR_BAD_SHAPE
    lin = B.LinearI8Params(8, 8, 16, 16, 16, 16, B.BF16)
    assert code(B.linear_i8, lin, codes[:5], P, codes, P, buf) == B.ERR_BAD_SHAPE
    assert code(B.linear_i8, lin, codes, P, codes[:5], P, buf) == B.ERR_BAD_SHAPE
    assert code(B.linear_i8, lin, codes, P, codes, P, buf[:5]) == B.ERR_BAD_SHAPE
