"""ctypes binding of libdppo.so: same names as include/dppo.h, argument marshalling only.

Array arguments are torch tensors (their device pointer is passed), raw integer addresses, or None
for the nullable ones.  Every function raises DppoError on a non-zero return code.  There is no
fallback: if the library has not been built, importing this module raises.

The scoring calls (token_logprobs, token_logprobs_backward, quantize_rows_i8, linear_i8), the distillation and verification
calls (distill_topk, distill_topk_backward, verify_drafts) and the block-scaled product (quantize_f8, linear_f8) also check the
tensors they are given: element type, on the current device, and large enough for the sizes in the params.  Their plain case (torch
tensors in the exact layout, the current stream) is checked and marshalled in native code (_marshal.so); anything else, and a
tree where that module has not been built, takes the same checks here.
"""
import ctypes
import os

import torch

from . import build

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdppo.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError("libdppo.so is not built: run `python -m paper_2603_04135_b200.build` "
                      "(the CUDA library is the only implementation; there is no CPU path)")
lib = ctypes.CDLL(_LIB_PATH)

F32, BF16 = 0, 1
STATUS_OK, STATUS_BAD_LENGTH, STATUS_BAD_TARGET, STATUS_TIMEOUT, STATUS_BAD_SEGMENTS, STATUS_BAD_INDEX, STATUS_RANGE = \
    0, 1, 2, 3, 4, 5, 6
ERR_INVALID_ARG, ERR_BAD_SHAPE, ERR_MISALIGNED, ERR_WORKSPACE_TOO_SMALL, ERR_UNSUPPORTED, ERR_CUDA = \
    -1, -2, -3, -4, -5, -6


class DppoError(RuntimeError):
    def __init__(self, code, message):
        super().__init__("libdppo error %d: %s" % (code, message))
        self.code = code


class PruneParams(ctypes.Structure):
    _fields_ = [("P", ctypes.c_int32), ("G", ctypes.c_int32), ("r_q", ctypes.c_double), ("r_o", ctypes.c_double),
                ("mode", ctypes.c_int32), ("reverse", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("step", ctypes.c_uint64)]


class PackParams(ctypes.Structure):
    _fields_ = [("n_max", ctypes.c_int32), ("L_row", ctypes.c_int32), ("N_win", ctypes.c_int32),
                ("policy", ctypes.c_int32)]


class LossParams(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int64), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("S_max", ctypes.c_int32), ("variant", ctypes.c_int32),
                ("eps_lo", ctypes.c_double), ("eps_hi", ctypes.c_double), ("beta", ctypes.c_double),
                ("temperature", ctypes.c_double), ("no_length_norm", ctypes.c_int32), ("reserved2", ctypes.c_int32),
                ("seq_log_ratio", ctypes.c_void_p)]


class LossKernelChoice(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("ctas_per_row", ctypes.c_int32), ("threads", ctypes.c_int32),
                ("fell_back", ctypes.c_int32)]


KERNEL_GENERAL, KERNEL_WARP, KERNEL_SHARED, KERNEL_STREAM, KERNEL_TILE = 0, 1, 2, 3, 4
KERNEL_NAMES = {KERNEL_GENERAL: "general two-pass", KERNEL_WARP: "warp per row", KERNEL_SHARED: "shared memory",
                KERNEL_STREAM: "streaming (forward only)", KERNEL_TILE: "tiles of rows"}
LOSS_WAIT_SELF_TEST = 1000000      # added to dppo_loss_params.variant
LMHEAD_WAIT_SELF_TEST = 100        # added to dppo_lmhead_params.variant


class LmheadParams(ctypes.Structure):
    _fields_ = [("loss", LossParams), ("H", ctypes.c_int32), ("backward", ctypes.c_int32), ("variant", ctypes.c_int32),
                ("dW_dtype", ctypes.c_int32),
                ("accumulate_dW", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class LogprobParams(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int64), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("top_k", ctypes.c_int32), ("variant", ctypes.c_int32),
                ("temperature", ctypes.c_double)]


class QuantizeParams(ctypes.Structure):
    _fields_ = [("rows_max", ctypes.c_int64), ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("q_stride", ctypes.c_int64)]


class LinearI8Params(ctypes.Structure):
    _fields_ = [("M_max", ctypes.c_int64), ("N", ctypes.c_int32), ("K", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("w_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
                ("out_dtype", ctypes.c_int32), ("variant", ctypes.c_int32)]


class DistillParams(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int64), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("top_k", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("temperature", ctypes.c_double)]


class VerifyParams(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int64), ("n_seqs", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("target_stride", ctypes.c_int64), ("draft_stride", ctypes.c_int64), ("noise_stride", ctypes.c_int64),
                ("temperature", ctypes.c_double), ("draft_temperature", ctypes.c_double)]


class QuantizeF8Params(ctypes.Structure):
    _fields_ = [("rows_max", ctypes.c_int64), ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("q_stride", ctypes.c_int64), ("scale_stride", ctypes.c_int64),
                ("block_rows", ctypes.c_int32)]


class LinearF8Params(ctypes.Structure):
    _fields_ = [("M_max", ctypes.c_int64), ("N", ctypes.c_int32), ("K", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("w_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
                ("x_scale_stride", ctypes.c_int64), ("w_scale_stride", ctypes.c_int64),
                ("out_dtype", ctypes.c_int32), ("variant", ctypes.c_int32)]


DISTILL_GIVEN, DISTILL_NORMALIZED, DISTILL_REST = 0, 1, 2
MAX_LISTED = 128
MAX_TOP_K = 32
LINEAR_I8_WAIT_SELF_TEST = 100     # added to dppo_linear_i8_params.variant
LINEAR_F8_WAIT_SELF_TEST = 100     # added to dppo_linear_f8_params.variant
F8_BLOCK = 128

_vp = ctypes.c_void_p
lib.dppo_version.restype = ctypes.c_int
lib.dppo_last_error.restype = ctypes.c_char_p
lib.dppo_group_advantages.restype = ctypes.c_int
lib.dppo_group_advantages.argtypes = [_vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_double, _vp, _vp, _vp, _vp]
lib.dppo_prune_and_rescale.restype = ctypes.c_int
lib.dppo_prune_and_rescale.argtypes = [ctypes.POINTER(PruneParams)] + [_vp] * 17
lib.dppo_history_gather.restype = ctypes.c_int
lib.dppo_history_gather.argtypes = [_vp, ctypes.c_int, _vp, ctypes.c_int, _vp, _vp, _vp]
lib.dppo_history_scatter.restype = ctypes.c_int
lib.dppo_history_scatter.argtypes = [_vp, ctypes.c_int, _vp, ctypes.c_int, _vp, _vp, _vp]
lib.dppo_pack_workspace_bytes.restype = ctypes.c_size_t
lib.dppo_pack_workspace_bytes.argtypes = [ctypes.POINTER(PackParams)]
lib.dppo_pack_prompts.restype = ctypes.c_int
lib.dppo_pack_prompts.argtypes = [ctypes.POINTER(PackParams)] + [_vp] * 10 + [ctypes.c_size_t, _vp, _vp]
lib.dppo_pack_static_max_units.restype = ctypes.c_int
lib.dppo_pack_prompts_static.restype = ctypes.c_int
lib.dppo_pack_prompts_static.argtypes = [ctypes.POINTER(PackParams)] + [_vp] * 11
lib.dppo_grpo_loss_workspace_bytes.restype = ctypes.c_size_t
lib.dppo_grpo_loss_workspace_bytes.argtypes = [ctypes.POINTER(LossParams)]
lib.dppo_grpo_loss_fwd_bwd.restype = ctypes.c_int
lib.dppo_grpo_loss_fwd_bwd.argtypes = [ctypes.POINTER(LossParams)] + [_vp] * 14 + [ctypes.c_size_t, _vp, _vp]


lib.dppo_grpo_loss_kernel_choice.restype = ctypes.c_int
lib.dppo_grpo_loss_kernel_choice.argtypes = [ctypes.POINTER(LossParams), ctypes.c_int, ctypes.POINTER(LossKernelChoice)]
lib.dppo_sequence_log_ratio.restype = ctypes.c_int
lib.dppo_sequence_log_ratio.argtypes = [_vp, _vp, _vp, ctypes.c_int, _vp, _vp, _vp]
lib.dppo_lmhead_workspace_bytes.restype = ctypes.c_size_t
lib.dppo_lmhead_workspace_bytes.argtypes = [ctypes.POINTER(LmheadParams)]
lib.dppo_lmhead_grpo_loss.restype = ctypes.c_int
lib.dppo_lmhead_grpo_loss.argtypes = [ctypes.POINTER(LmheadParams)] + [_vp] * 16 + [ctypes.c_size_t, _vp, _vp]
lib.dppo_token_logprobs.restype = ctypes.c_int
lib.dppo_token_logprobs.argtypes = [ctypes.POINTER(LogprobParams)] + [_vp] * 11
lib.dppo_token_logprobs_backward.restype = ctypes.c_int
lib.dppo_token_logprobs_backward.argtypes = [ctypes.POINTER(LogprobParams)] + [_vp] * 9
lib.dppo_quantize_rows_i8.restype = ctypes.c_int
lib.dppo_quantize_rows_i8.argtypes = [ctypes.POINTER(QuantizeParams)] + [_vp] * 6
lib.dppo_linear_i8.restype = ctypes.c_int
lib.dppo_linear_i8.argtypes = [ctypes.POINTER(LinearI8Params)] + [_vp] * 8
lib.dppo_distill_topk.restype = ctypes.c_int
lib.dppo_distill_topk.argtypes = [ctypes.POINTER(DistillParams)] + [_vp] * 11
lib.dppo_distill_topk_backward.restype = ctypes.c_int
lib.dppo_distill_topk_backward.argtypes = [ctypes.POINTER(DistillParams)] + [_vp] * 9
lib.dppo_verify_drafts_workspace_bytes.restype = ctypes.c_size_t
lib.dppo_verify_drafts_workspace_bytes.argtypes = [ctypes.POINTER(VerifyParams)]
lib.dppo_verify_drafts.restype = ctypes.c_int
lib.dppo_verify_drafts.argtypes = [ctypes.POINTER(VerifyParams)] + [_vp] * 10 + [ctypes.c_size_t, _vp, _vp]
lib.dppo_quantize_f8.restype = ctypes.c_int
lib.dppo_quantize_f8.argtypes = [ctypes.POINTER(QuantizeF8Params)] + [_vp] * 6
lib.dppo_linear_f8.restype = ctypes.c_int
lib.dppo_linear_f8.argtypes = [ctypes.POINTER(LinearF8Params)] + [_vp] * 8


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    return int(x)


_TORCH_DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
_Tensor, _f32, _i32, _i8, _f8 = torch.Tensor, torch.float32, torch.int32, torch.int8, torch.float8_e4m3fn


def _arr(x, name, device, dtype, n):
    """Device pointer of n dense elements.  A torch tensor is checked: of `dtype`, on `device` (the current one), large
    enough.  The plain case is one expression: these checks are on the path of calls that take 10 us."""
    if x is None:
        return None
    if x.__class__ is _Tensor and x.dtype is dtype and x.get_device() == device and x.numel() >= n and x.is_contiguous():
        return x.data_ptr()
    if not isinstance(x, _Tensor):
        return x
    _check_kind(x, name, device, dtype)
    if n > 0 and (x.numel() < n or not x.is_contiguous()):
        raise DppoError(ERR_BAD_SHAPE, "%s: needs %d contiguous elements, got shape %s, strides %s" % (name, n, tuple(x.shape), x.stride()))
    return x.data_ptr()


def _mat(x, name, device, dtype, rows, cols, stride):
    """The same for [rows x cols] with `stride` elements between rows: the tensor itself must hold them, not only its storage."""
    if (x.__class__ is _Tensor and x.dtype is dtype and x.get_device() == device and x.stride() == (stride, 1)
            and x.shape[0] >= rows and x.shape[1] >= cols):
        return x.data_ptr()
    if not isinstance(x, _Tensor):
        return x
    _check_kind(x, name, device, dtype)
    if rows > 0 and not _holds_rows(x, rows, cols, stride):
        raise DppoError(ERR_BAD_SHAPE, "%s: shape %s, strides %s do not hold %d rows of %d elements, %d apart"
                        % (name, tuple(x.shape), x.stride(), rows, cols, stride))
    return x.data_ptr()


def _holds_rows(x, rows, cols, stride):
    """Whether x, of any rank, holds `rows` rows of `cols` elements that lie `stride` apart."""
    if x.dim() == 2 and x.shape[0] > 1 and x.stride(0) != stride:
        return False
    runs = []                                    # x as few dimensions as its strides allow: [size, stride], outermost first
    for n, s in zip(x.shape, x.stride()):
        if n == 1:
            continue
        if runs and runs[-1][1] == n * s:
            runs[-1] = [runs[-1][0] * n, s]
        else:
            runs.append([n, s])
    if len(runs) == 2 and runs[1][1] == 1:       # rows of their own
        (r, pitch), (c, _) = runs
        return (pitch == stride or rows == 1) and r >= rows and c >= cols
    if len(runs) == 1 and runs[0][1] == stride and cols == 1:
        return runs[0][0] >= rows
    dense = not runs or len(runs) == 1 and runs[0][1] == 1
    return dense and x.numel() >= (rows - 1) * stride + cols


def _check_kind(x, name, device, dtype):
    if x.dtype is not dtype:
        raise DppoError(ERR_INVALID_ARG, "%s: dtype %s, expected %s" % (name, x.dtype, dtype))
    if x.get_device() != device:
        raise DppoError(ERR_INVALID_ARG, "%s: on %s, the current device is cuda:%d" % (name, x.device, device))


_cuda = None                        # whether there is a CUDA device; asked once


def _device():
    global _cuda
    if _cuda is None:
        _cuda = torch.cuda.is_available()
    return _get_device() if _cuda else -1


# torch.cuda.current_device() and current_stream().cuda_stream without their Python layers (3 us of a small call)
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream):
    if stream is None:
        device = _device()
        return _current_stream(device) if device >= 0 else None
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _check(rc):
    if rc != 0:
        raise DppoError(rc, lib.dppo_last_error().decode("utf-8", "replace"))


def version():
    return lib.dppo_version()


def last_error():
    return lib.dppo_last_error().decode("utf-8", "replace")


def group_advantages(rewards, P, G, adv, mean_abs_adv, std_ddof=0, std_eps=1e-6, status=None, stream=None):
    _check(lib.dppo_group_advantages(_ptr(rewards), P, G, std_ddof, std_eps, _ptr(adv), _ptr(mean_abs_adv),
                                     _ptr(status), _stream(stream)))


def prune_and_rescale(params, adv, mean_abs_adv, H_prev, u_q, u_o, cand_q, cand_o, keep_q, keep_o,
                      n_keep_q, n_keep_o, gamma_q, gamma_o, w_seq, H_next, status=None, stream=None):
    _check(lib.dppo_prune_and_rescale(ctypes.byref(params), _ptr(adv), _ptr(mean_abs_adv), _ptr(H_prev),
                                      _ptr(u_q), _ptr(u_o), _ptr(cand_q), _ptr(cand_o), _ptr(keep_q),
                                      _ptr(keep_o), _ptr(n_keep_q), _ptr(n_keep_o), _ptr(gamma_q),
                                      _ptr(gamma_o), _ptr(w_seq), _ptr(H_next), _ptr(status), _stream(stream)))


def history_gather(H_table, N, prompt_ids, P, H_batch, status=None, stream=None):
    _check(lib.dppo_history_gather(_ptr(H_table), N, _ptr(prompt_ids), P, _ptr(H_batch), _ptr(status), _stream(stream)))


def history_scatter(H_table, N, prompt_ids, P, H_next, status=None, stream=None):
    _check(lib.dppo_history_scatter(_ptr(H_table), N, _ptr(prompt_ids), P, _ptr(H_next), _ptr(status), _stream(stream)))


def pack_workspace_bytes(params):
    return lib.dppo_pack_workspace_bytes(ctypes.byref(params))


def pack_prompts(params, len_, keep, loss_len, order, row_of, off_in_row, row_fill, cu_seqlens, counts,
                 workspace, workspace_bytes, status=None, stream=None):
    _check(lib.dppo_pack_prompts(ctypes.byref(params), _ptr(len_), _ptr(keep), _ptr(loss_len), _ptr(order),
                                 _ptr(row_of), _ptr(off_in_row), _ptr(row_fill), _ptr(cu_seqlens),
                                 _ptr(counts), _ptr(workspace), workspace_bytes, _ptr(status), _stream(stream)))


def pack_static_max_units():
    return lib.dppo_pack_static_max_units()


def pack_prompts_static(params, len_, keep, loss_len, order, row_of, off_in_row, row_fill, cu_seqlens, counts,
                        status=None, stream=None):
    """dppo_pack_prompts without a workspace argument: scratch is a fixed array inside the library
    (at most pack_static_max_units() units); nothing is allocated by the call."""
    _check(lib.dppo_pack_prompts_static(ctypes.byref(params), _ptr(len_), _ptr(keep), _ptr(loss_len), _ptr(order),
                                        _ptr(row_of), _ptr(off_in_row), _ptr(row_fill), _ptr(cu_seqlens),
                                        _ptr(counts), _ptr(status), _stream(stream)))


def grpo_loss_workspace_bytes(params):
    return lib.dppo_grpo_loss_workspace_bytes(ctypes.byref(params))


def grpo_loss_fwd_bwd(params, logits, target, logp_old, logp_ref, cu_seqlens, n_tokens_dev, adv, w, seg_map,
                      dlogits, logp_out, lse_out, loss_out, workspace, workspace_bytes, status=None,
                      stream=None):
    _check(lib.dppo_grpo_loss_fwd_bwd(ctypes.byref(params), _ptr(logits), _ptr(target), _ptr(logp_old),
                                      _ptr(logp_ref), _ptr(cu_seqlens), _ptr(n_tokens_dev), _ptr(adv), _ptr(w),
                                      _ptr(seg_map), _ptr(dlogits), _ptr(logp_out), _ptr(lse_out),
                                      _ptr(loss_out), _ptr(workspace), workspace_bytes, _ptr(status),
                                      _stream(stream)))


def grpo_loss_kernel_choice(params, forward_only=False):
    """The kernel dppo_grpo_loss_fwd_bwd runs for these parameters on the current device (forward_only: the call
    will pass no dlogits), as a LossKernelChoice."""
    out = LossKernelChoice()
    _check(lib.dppo_grpo_loss_kernel_choice(ctypes.byref(params), int(bool(forward_only)), ctypes.byref(out)))
    return out


def lmhead_workspace_bytes(params):
    return lib.dppo_lmhead_workspace_bytes(ctypes.byref(params))


def lmhead_grpo_loss(params, hidden, W, target, logp_old, logp_ref, cu_seqlens, n_tokens_dev, adv, w, seg_map,
                     dhidden, dW, logp_out, lse_out, loss_out, workspace, workspace_bytes, status=None, stream=None):
    _check(lib.dppo_lmhead_grpo_loss(ctypes.byref(params), _ptr(hidden), _ptr(W), _ptr(target), _ptr(logp_old),
                                     _ptr(logp_ref), _ptr(cu_seqlens), _ptr(n_tokens_dev), _ptr(adv), _ptr(w),
                                     _ptr(seg_map), _ptr(dhidden), _ptr(dW), _ptr(logp_out), _ptr(lse_out),
                                     _ptr(loss_out), _ptr(workspace), workspace_bytes, _ptr(status), _stream(stream)))


def sequence_log_ratio(logp, logp_old, cu_seqlens, S_max, out, status=None, stream=None):
    _check(lib.dppo_sequence_log_ratio(_ptr(logp), _ptr(logp_old), _ptr(cu_seqlens), S_max, _ptr(out), _ptr(status),
                                       _stream(stream)))


class _NoNative:
    """Stands in for the native marshalling: nothing is the plain case."""
    token_logprobs = token_logprobs_backward = quantize_rows_i8 = linear_i8 = staticmethod(lambda *a: None)
    distill_topk = distill_topk_backward = verify_drafts = quantize_f8 = linear_f8 = token_logprobs


def _load_native():
    """The native marshalling, if it was built for this interpreter and this torch: it reads their structures."""
    try:
        from . import _marshal
    except ImportError:
        return _NoNative
    if getattr(_marshal, "built_for", None) != build.built_for():
        return _NoNative
    _marshal.bind((LogprobParams, QuantizeParams, LinearI8Params, DistillParams, VerifyParams, QuantizeF8Params, LinearF8Params),
                  tuple(ctypes.cast(f, ctypes.c_void_p).value for f in (
                      lib.dppo_token_logprobs, lib.dppo_token_logprobs_backward, lib.dppo_quantize_rows_i8, lib.dppo_linear_i8,
                      lib.dppo_distill_topk, lib.dppo_distill_topk_backward, lib.dppo_verify_drafts, lib.dppo_quantize_f8, lib.dppo_linear_f8)))
    return _marshal


_native = _load_native()


def _done(rc):
    """Whether the native marshalling has made the call (rc: its return code, None where it was not the plain case)."""
    if rc is None:
        return False
    _check(rc)
    return True


def token_logprobs(params, logits, target, n_tokens_dev, logp_out, entropy_out, lse_out, top_ids, top_logp, stats,
                   status=None, stream=None):
    rc = _native.token_logprobs(params, logits, target, n_tokens_dev, logp_out, entropy_out, lse_out, top_ids, top_logp, stats,
                                status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    T, V = p.T_max, p.V
    k = p.top_k * T
    _check(lib.dppo_token_logprobs(
        ctypes.byref(p), _mat(logits, "logits", d, _TORCH_DTYPE.get(p.dtype), T, V, p.row_stride),
        _arr(target, "target", d, _i32, T), _arr(n_tokens_dev, "n_tokens_dev", d, _i32, 1), _arr(logp_out, "logp_out", d, _f32, T),
        _arr(entropy_out, "entropy_out", d, _f32, T), _arr(lse_out, "lse_out", d, _f32, T), _arr(top_ids, "top_ids", d, _i32, k),
        _arr(top_logp, "top_logp", d, _f32, k), _arr(stats, "stats", d, _f32, 4 * T), _arr(status, "status", d, _i32, 1),
        _stream(stream)))


def token_logprobs_backward(params, logits, target, n_tokens_dev, stats, dlogp, dentropy, dlogits, status=None,
                            stream=None):
    rc = _native.token_logprobs_backward(params, logits, target, n_tokens_dev, stats, dlogp, dentropy, dlogits, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    T, V, dt, ld = p.T_max, p.V, _TORCH_DTYPE.get(p.dtype), p.row_stride
    _check(lib.dppo_token_logprobs_backward(
        ctypes.byref(p), _mat(logits, "logits", d, dt, T, V, ld), _arr(target, "target", d, _i32, T),
        _arr(n_tokens_dev, "n_tokens_dev", d, _i32, 1), _arr(stats, "stats", d, _f32, 4 * T), _arr(dlogp, "dlogp", d, _f32, T),
        _arr(dentropy, "dentropy", d, _f32, T), _mat(dlogits, "dlogits", d, dt, T, V, ld), _arr(status, "status", d, _i32, 1),
        _stream(stream)))


def quantize_rows_i8(params, x, q, scale, n_rows_dev=None, status=None, stream=None):
    rc = _native.quantize_rows_i8(params, x, q, scale, n_rows_dev, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    M, K = p.rows_max, p.K
    _check(lib.dppo_quantize_rows_i8(
        ctypes.byref(p), _mat(x, "x", d, _TORCH_DTYPE.get(p.dtype), M, K, p.x_stride), _mat(q, "q", d, _i8, M, K, p.q_stride),
        _arr(scale, "scale", d, _f32, M), _arr(n_rows_dev, "n_rows_dev", d, _i32, 1), _arr(status, "status", d, _i32, 1),
        _stream(stream)))


def linear_i8(params, x, x_scale, w, w_scale, out, n_rows_dev=None, status=None, stream=None):
    rc = _native.linear_i8(params, x, x_scale, w, w_scale, out, n_rows_dev, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    M, N, K = p.M_max, p.N, p.K
    _check(lib.dppo_linear_i8(
        ctypes.byref(p), _mat(x, "x", d, _i8, M, K, p.x_stride), _arr(x_scale, "x_scale", d, _f32, M),
        _mat(w, "w", d, _i8, N, K, p.w_stride), _arr(w_scale, "w_scale", d, _f32, N),
        _mat(out, "out", d, _TORCH_DTYPE.get(p.out_dtype), M, N, p.out_stride), _arr(n_rows_dev, "n_rows_dev", d, _i32, 1),
        _arr(status, "status", d, _i32, 1),
        _stream(stream)))


def distill_topk(params, logits, top_ids, top_logp, n_tokens_dev, weight, loss_out, lse_out, stats, dlogits, status=None, stream=None):
    rc = _native.distill_topk(params, logits, top_ids, top_logp, n_tokens_dev, weight, loss_out, lse_out, stats, dlogits, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    T, V, dt, ld, k = p.T_max, p.V, _TORCH_DTYPE.get(p.dtype), p.row_stride, p.T_max * p.top_k
    _check(lib.dppo_distill_topk(
        ctypes.byref(p), _mat(logits, "logits", d, dt, T, V, ld), _arr(top_ids, "top_ids", d, _i32, k), _arr(top_logp, "top_logp", d, _f32, k),
        _arr(n_tokens_dev, "n_tokens_dev", d, _i32, 1), _arr(weight, "weight", d, _f32, T), _arr(loss_out, "loss_out", d, _f32, T),
        _arr(lse_out, "lse_out", d, _f32, T), _arr(stats, "stats", d, _f32, 4 * T), _mat(dlogits, "dlogits", d, dt, T, V, ld),
        _arr(status, "status", d, _i32, 1), _stream(stream)))


def distill_topk_backward(params, logits, top_ids, top_logp, n_tokens_dev, stats, dloss, dlogits, status=None, stream=None):
    rc = _native.distill_topk_backward(params, logits, top_ids, top_logp, n_tokens_dev, stats, dloss, dlogits, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    T, V, dt, ld, k = p.T_max, p.V, _TORCH_DTYPE.get(p.dtype), p.row_stride, p.T_max * p.top_k
    _check(lib.dppo_distill_topk_backward(
        ctypes.byref(p), _mat(logits, "logits", d, dt, T, V, ld), _arr(top_ids, "top_ids", d, _i32, k), _arr(top_logp, "top_logp", d, _f32, k),
        _arr(n_tokens_dev, "n_tokens_dev", d, _i32, 1), _arr(stats, "stats", d, _f32, 4 * T), _arr(dloss, "dloss", d, _f32, T),
        _mat(dlogits, "dlogits", d, dt, T, V, ld), _arr(status, "status", d, _i32, 1), _stream(stream)))


def verify_drafts_workspace_bytes(params):
    return lib.dppo_verify_drafts_workspace_bytes(ctypes.byref(params))


def verify_drafts(params, target_logits, draft_logits, drafts, cu_drafts, uniforms, noise, n_accepted, tokens_out, logp_out, workspace,
                  workspace_bytes, status=None, stream=None):
    rc = _native.verify_drafts(params, target_logits, draft_logits, drafts, cu_drafts, uniforms, noise, n_accepted, tokens_out, logp_out,
                               workspace, workspace_bytes, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    T, B, V, dt = p.T_max, p.n_seqs, p.V, _TORCH_DTYPE.get(p.dtype)
    _check(lib.dppo_verify_drafts(
        ctypes.byref(p), _mat(target_logits, "target_logits", d, dt, T + B, V, p.target_stride),
        _mat(draft_logits, "draft_logits", d, dt, T, V, p.draft_stride), _arr(drafts, "drafts", d, _i32, T),
        _arr(cu_drafts, "cu_drafts", d, _i32, B + 1), _arr(uniforms, "uniforms", d, _f32, T),
        _mat(noise, "noise", d, _f32, B, V, p.noise_stride), _arr(n_accepted, "n_accepted", d, _i32, B),
        _arr(tokens_out, "tokens_out", d, _i32, T + B), _arr(logp_out, "logp_out", d, _f32, T + B),
        _arr(workspace, "workspace", d, torch.uint8, workspace_bytes), workspace_bytes, _arr(status, "status", d, _i32, 1), _stream(stream)))


def quantize_f8(params, x, q, scale, n_rows_dev=None, status=None, stream=None):
    rc = _native.quantize_f8(params, x, q, scale, n_rows_dev, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    M, K, blocks = p.rows_max, p.K, (p.K + 127) // 128
    rows, cols = (blocks, M) if p.block_rows == 1 else ((M + 127) // 128, blocks)
    _check(lib.dppo_quantize_f8(
        ctypes.byref(p), _mat(x, "x", d, _TORCH_DTYPE.get(p.dtype), M, K, p.x_stride), _mat(q, "q", d, _f8, M, K, p.q_stride),
        _mat(scale, "scale", d, _f32, rows, cols, p.scale_stride), _arr(n_rows_dev, "n_rows_dev", d, _i32, 1),
        _arr(status, "status", d, _i32, 1), _stream(stream)))


def linear_f8(params, x, x_scale, w, w_scale, out, n_rows_dev=None, status=None, stream=None):
    rc = _native.linear_f8(params, x, x_scale, w, w_scale, out, n_rows_dev, status, stream)
    if rc == 0 or _done(rc):
        return
    p, d = params, _device()
    M, N, K, blocks = p.M_max, p.N, p.K, (p.K + 127) // 128
    _check(lib.dppo_linear_f8(
        ctypes.byref(p), _mat(x, "x", d, _f8, M, K, p.x_stride), _mat(x_scale, "x_scale", d, _f32, blocks, M, p.x_scale_stride),
        _mat(w, "w", d, _f8, N, K, p.w_stride), _mat(w_scale, "w_scale", d, _f32, (N + 127) // 128, blocks, p.w_scale_stride),
        _mat(out, "out", d, _TORCH_DTYPE.get(p.out_dtype), M, N, p.out_stride), _arr(n_rows_dev, "n_rows_dev", d, _i32, 1),
        _arr(status, "status", d, _i32, 1), _stream(stream)))
