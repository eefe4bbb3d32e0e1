"""Refusals and host-side layout of the distillation, verification and block-scaled product calls: everything here returns before a launch (CPU)."""
import ctypes

import pytest
import torch

from paper_2603_04135_b200 import binding as B

P = 1 << 20      # an aligned address that is only looked at


def code(f, *a, **k):
    with pytest.raises(B.DppoError) as e:
        f(*a, **k)
    return e.value.code


def test_struct_layouts_match_header():
    assert ctypes.sizeof(B.DistillParams) == 40 and B.DistillParams.temperature.offset == 32 and B.DistillParams.top_k.offset == 24
    assert ctypes.sizeof(B.VerifyParams) == 64 and B.VerifyParams.target_stride.offset == 24 and B.VerifyParams.temperature.offset == 48
    assert ctypes.sizeof(B.QuantizeF8Params) == 48 and B.QuantizeF8Params.block_rows.offset == 40
    assert ctypes.sizeof(B.LinearF8Params) == 64 and B.LinearF8Params.x_scale_stride.offset == 40 and B.LinearF8Params.variant.offset == 60


@pytest.mark.parametrize("prm, want", [
    ((-1, 8, 1, 8, 4, 0, 1.0), B.ERR_INVALID_ARG), ((4, 0, 1, 8, 4, 0, 1.0), B.ERR_INVALID_ARG), ((4, 8, 2, 8, 4, 0, 1.0), B.ERR_UNSUPPORTED),
    ((4, 9, 1, 8, 4, 0, 1.0), B.ERR_BAD_SHAPE), ((4, 8, 1, 12, 4, 0, 1.0), B.ERR_MISALIGNED), ((4, 8, 1, 8, 0, 0, 1.0), B.ERR_INVALID_ARG),
    ((4, 8, 1, 8, 129, 0, 1.0), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 4, 3, 1.0), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 4, -1, 1.0), B.ERR_INVALID_ARG),
    ((4, 8, 1, 8, 4, 0, 0.0), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 4, 0, float("nan")), B.ERR_INVALID_ARG), ((4, 8, 1, 8, 4, 0, 1e7), B.ERR_INVALID_ARG),
    ((4, (1 << 20) + 8, 1, (1 << 20) + 8, 4, 0, 1.0), B.ERR_BAD_SHAPE), ((1 << 31, 8, 1, 8, 4, 0, 1.0), B.ERR_BAD_SHAPE)])
def test_distill_params(prm, want):
    assert code(B.distill_topk, B.DistillParams(*prm), P, P, P, None, None, P, P, P, None) == want
    assert code(B.distill_topk_backward, B.DistillParams(*prm), P, P, P, None, P, P, P) == want


def test_distill_arrays():
    prm, f, b = B.DistillParams(4, 8, 1, 8, 2, 2, 1.0), B.distill_topk, B.distill_topk_backward
    assert code(f, prm, None, P, P, None, None, P, P, P, None) == B.ERR_INVALID_ARG
    assert code(f, prm, P, None, P, None, None, P, P, P, None) == B.ERR_INVALID_ARG
    assert code(f, prm, P, P, None, None, None, P, P, P, None) == B.ERR_INVALID_ARG
    assert code(f, prm, P + 8, P, P, None, None, P, P, P, None) == B.ERR_MISALIGNED
    assert code(f, prm, P, P, P, None, None, P, P, P + 4, None) == B.ERR_MISALIGNED
    assert code(f, prm, P, P, P, None, None, P, P, P, P + 2) == B.ERR_MISALIGNED
    assert code(f, prm, P, P, P, None, None, P, P, None, P) == B.ERR_INVALID_ARG        # a gradient without stats
    assert code(f, prm, P, P, P, None, P, P, P, P, None) == B.ERR_INVALID_ARG           # weights without a gradient
    assert code(b, prm, P, P, P, None, None, P, P) == B.ERR_INVALID_ARG
    assert code(b, prm, P, P, P, None, P, P, None) == B.ERR_INVALID_ARG
    none = B.DistillParams(0, 8, 1, 8, 2, 2, 1.0)
    f(none, None, None, None, None, None, None, None, None, None)
    b(none, None, None, None, None, None, None, None)


@pytest.mark.parametrize("prm, want", [
    ((-1, 2, 8, 1, 8, 8, 8, 1.0, 1.0), B.ERR_INVALID_ARG), ((4, -1, 8, 1, 8, 8, 8, 1.0, 1.0), B.ERR_INVALID_ARG),
    ((4, 2, 0, 1, 8, 8, 8, 1.0, 1.0), B.ERR_INVALID_ARG), ((4, 2, 8, 3, 8, 8, 8, 1.0, 1.0), B.ERR_UNSUPPORTED),
    ((4, 2, 8, 1, 7, 8, 8, 1.0, 1.0), B.ERR_BAD_SHAPE), ((4, 2, 8, 1, 8, 7, 8, 1.0, 1.0), B.ERR_BAD_SHAPE), ((4, 2, 8, 1, 8, 8, 7, 1.0, 1.0), B.ERR_BAD_SHAPE),
    ((4, 2, 8, 1, 12, 8, 8, 1.0, 1.0), B.ERR_MISALIGNED), ((4, 2, 8, 1, 8, 12, 8, 1.0, 1.0), B.ERR_MISALIGNED), ((4, 2, 8, 1, 8, 8, 9, 1.0, 1.0), B.ERR_MISALIGNED),
    ((4, 2, 8, 1, 8, 8, 8, 0.0, 1.0), B.ERR_INVALID_ARG), ((4, 2, 8, 1, 8, 8, 8, 1.0, float("inf")), B.ERR_INVALID_ARG),
    ((1 << 30, 2, 8, 1, 8, 8, 8, 1.0, 1.0), B.ERR_BAD_SHAPE), ((4, 2, (1 << 30) + 8, 1, 1 << 31, 1 << 31, 1 << 31, 1.0, 1.0), B.ERR_BAD_SHAPE)])
def test_verify_params(prm, want):
    assert code(B.verify_drafts, B.VerifyParams(*prm), P, P, P, P, P, P, P, P, P, P, 1 << 20) == want


def test_verify_arrays():
    prm = B.VerifyParams(4, 2, 8, 1, 8, 8, 8, 1.0, 1.0)
    assert B.verify_drafts_workspace_bytes(prm) == 10 * 8 and B.verify_drafts_workspace_bytes(B.VerifyParams(-1, 2, 8, 1, 8, 8, 8, 1.0, 1.0)) == 0
    args = [P] * 10
    for i in (0, 2, 3, 4, 5, 6, 7, 8):
        assert code(B.verify_drafts, prm, *[None if j == i else x for j, x in enumerate(args)], 80) == B.ERR_INVALID_ARG, i
    for i in (0, 1, 5, 9):
        assert code(B.verify_drafts, prm, *[x + 8 if j == i else x for j, x in enumerate(args)], 80) == B.ERR_MISALIGNED, i
    assert code(B.verify_drafts, prm, *args, 79) == B.ERR_WORKSPACE_TOO_SMALL
    assert code(B.verify_drafts, prm, *args[:9], None, 80) == B.ERR_WORKSPACE_TOO_SMALL
    copied = B.VerifyParams(4, 2, 8, 1, 8, 0, 8, 1.0, 0.0)              # without draft logits their stride and temperature are not looked at
    assert code(B.verify_drafts, copied, P, None, *args[2:], 79) == B.ERR_WORKSPACE_TOO_SMALL
    B.verify_drafts(B.VerifyParams(0, 0, 8, 1, 8, 8, 8, 1.0, 1.0), *([None] * 10), 0)


def test_quantize_f8_params():
    q = B.quantize_f8
    assert code(q, B.QuantizeF8Params(-1, 8, 1, 8, 16, 4, 1), P, P, P) == B.ERR_INVALID_ARG
    assert code(q, B.QuantizeF8Params(4, 0, 1, 8, 16, 4, 1), P, P, P) == B.ERR_INVALID_ARG
    assert code(q, B.QuantizeF8Params(4, 8, 5, 8, 16, 4, 1), P, P, P) == B.ERR_UNSUPPORTED
    assert code(q, B.QuantizeF8Params(4, 8, 1, 8, 16, 4, 64), P, P, P) == B.ERR_UNSUPPORTED
    assert code(q, B.QuantizeF8Params(4, 8, 1, 7, 16, 4, 1), P, P, P) == B.ERR_BAD_SHAPE
    assert code(q, B.QuantizeF8Params(4, 8, 1, 8, 16, 3, 1), P, P, P) == B.ERR_BAD_SHAPE      # fewer scales than rows
    assert code(q, B.QuantizeF8Params(4, 300, 1, 304, 304, 2, 128), P, P, P) == B.ERR_BAD_SHAPE
    assert code(q, B.QuantizeF8Params(4, 8, 1, 9, 16, 4, 1), P, P, P) == B.ERR_MISALIGNED
    assert code(q, B.QuantizeF8Params(4, 8, 1, 8, 8, 4, 1), P, P, P) == B.ERR_MISALIGNED
    assert code(q, B.QuantizeF8Params(4, 8, 1, 8, 16, 4, 1), P, P + 1, P) == B.ERR_MISALIGNED
    assert code(q, B.QuantizeF8Params(4, 8, 1, 8, 16, 4, 1), None, P, P) == B.ERR_INVALID_ARG
    assert code(q, B.QuantizeF8Params(1 << 31, 8, 1, 8, 16, 1 << 31, 1), P, P, P) == B.ERR_BAD_SHAPE
    q(B.QuantizeF8Params(0, 8, 1, 8, 16, 4, 1), None, None, None)


def test_linear_f8_params():
    def lin(*prm, x=P, w=P, out=P, xs=P):
        return code(B.linear_f8, B.LinearF8Params(*prm), x, xs, w, P, out)
    assert lin(-1, 8, 16, 16, 16, 8, 4, 1, 0) == B.ERR_INVALID_ARG
    assert lin(4, 0, 16, 16, 16, 8, 4, 1, 0) == B.ERR_INVALID_ARG
    assert lin(4, 8, 0, 16, 16, 8, 4, 1, 0) == B.ERR_INVALID_ARG
    assert lin(4, 8, 16, 16, 16, 8, 4, 1, 2) == B.ERR_UNSUPPORTED
    assert lin(4, 8, 17, 16, 32, 8, 4, 1, 0) == B.ERR_BAD_SHAPE
    assert lin(4, 8, 16, 16, 16, 7, 4, 1, 0) == B.ERR_BAD_SHAPE
    assert lin(5, 8, 16, 16, 16, 8, 4, 1, 0) == B.ERR_BAD_SHAPE                               # fewer scales than tokens
    assert lin(4, 8, 129, 144, 144, 8, 4, 1, 0) == B.ERR_BAD_SHAPE                            # fewer scales than blocks
    assert lin(4, 8, 16, 24, 16, 8, 4, 1, 0) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 5, 1, 0) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 4, 1, 0, xs=P + 4) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 4, 1, 0, x=P + 8) == B.ERR_MISALIGNED
    assert lin(4, 8, 16, 16, 16, 8, 4, 1, 0, w=None) == B.ERR_INVALID_ARG
    assert lin(4, 8, 16, 16, 16, 8, 4, 1, 0, 3) == B.ERR_INVALID_ARG and lin(4, 8, 16, 16, 16, 8, 4, 1, 0, 100) == B.ERR_INVALID_ARG
    assert lin((1 << 31) - 1, 8, 16, 16, 16, 8, 1 << 31, 1, 0) == B.ERR_BAD_SHAPE
    B.linear_f8(B.LinearF8Params(0, 8, 16, 16, 16, 8, 4, 1, 0), None, None, None, None, None)


def test_tensors_are_checked():
    """Type, device and size of every tensor; a CPU tensor is never on the current device."""
    z = torch.zeros(4, 8)
    prm = B.DistillParams(4, 8, 0, 8, 2, 2, 1.0)
    ids, lp, st = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(4, 4)
    assert code(B.distill_topk, prm, z.bfloat16(), ids, lp, None, None, None, None, st, None) == B.ERR_INVALID_ARG
    assert code(B.distill_topk, prm, P, ids.long(), lp, None, None, None, None, st, None) == B.ERR_INVALID_ARG
    q = torch.zeros(4, 16, dtype=torch.int8)
    assert code(B.quantize_f8, B.QuantizeF8Params(4, 8, 0, 8, 16, 4, 1), P, q, P) == B.ERR_INVALID_ARG
    if not torch.cuda.is_available():                                   # device -1 here: sizes are looked at
        assert code(B.distill_topk, prm, z[:3], ids, lp, None, None, None, None, st, None) == B.ERR_BAD_SHAPE
        assert code(B.distill_topk, prm, z, ids[:, :1], lp, None, None, None, None, st, None) == B.ERR_BAD_SHAPE
        assert code(B.distill_topk, prm, z, ids, lp, None, None, None, None, st[:3], None) == B.ERR_BAD_SHAPE
        v = B.VerifyParams(4, 2, 8, 0, 8, 8, 8, 1.0, 1.0)
        assert code(B.verify_drafts, v, torch.zeros(5, 8), None, P, P, P, P, P, P, P, P, 80) == B.ERR_BAD_SHAPE
        assert code(B.verify_drafts, v, P, None, P, P, P, torch.zeros(2, 7), P, P, P, P, 80) == B.ERR_BAD_SHAPE
        assert code(B.verify_drafts, v, P, None, P, P, P, P, P, P, P, torch.zeros(79, dtype=torch.uint8), 80) == B.ERR_BAD_SHAPE
