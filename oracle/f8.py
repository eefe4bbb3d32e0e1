"""8-bit floating point (e4m3: 4 exponent bits of bias 7, 3 mantissa bits, no infinities, largest 448) with block scales, from the
definitions in include/dppo.h."""
import numpy as np


def decode(code):
    """Values of e4m3 codes (uint8) as float64."""
    code = code.astype(np.int64)
    e, m = code >> 3 & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(code & 128, -v, v)


_TABLE = decode(np.arange(127, dtype=np.uint8))                      # 0 .. 448, ascending


def encode(x):
    """Nearest codes of float values, ties to the even code, held at +-448."""
    a = np.minimum(np.abs(x.astype(np.float64)), 448.0)
    hi = np.searchsorted(_TABLE, a)                                  # first value >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _TABLE[lo], _TABLE[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return (np.where(up, hi, lo) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantize(x, block_rows):
    """x float32 [M, K].  Returns codes [M, K] and scales: [ceil(K / 128), M] for block_rows 1, [ceil(M / 128), ceil(K / 128)] for 128."""
    M, K = x.shape
    kb, mb = -(-K // 128), -(-M // block_rows)
    pad = np.zeros((mb * block_rows, kb * 128), dtype=np.float32)
    pad[:M, :K] = x
    blocks = pad.reshape(mb, block_rows, kb, 128)
    amax = np.abs(blocks).max(axis=(1, 3))
    with np.errstate(all="ignore"):
        s = np.maximum(amax * (np.float32(1.0) / np.float32(448.0)), np.float32(2.0 ** -126)).astype(np.float32)
        fine = np.isfinite(amax)
        s = np.where(fine, s, np.float32(np.nan))
        y = (blocks / s[:, None, :, None]).astype(np.float32)
    q = encode(np.where(fine[:, None, :, None], np.nan_to_num(y), 0.0).reshape(-1)).reshape(mb * block_rows, kb * 128)[:M, :K]
    return q, (s.T if block_rows == 1 else s)


def linear(q, xs, w, ws):
    """Products [M, N] in float64 and the sum of the magnitudes of their terms."""
    K = q.shape[1]
    x = decode(q) * np.repeat(xs.astype(np.float64), 128, axis=0)[:K].T
    y = decode(w) * np.repeat(np.repeat(ws.astype(np.float64), 128, axis=0)[:w.shape[0]], 128, axis=1)[:, :K]
    return x @ y.T, np.abs(x) @ np.abs(y).T
