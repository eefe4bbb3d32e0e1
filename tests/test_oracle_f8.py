"""The 8-bit floating-point oracle (CPU): codes against torch's conversion and against the value table."""
import numpy as np
import torch

from oracle import f8


def test_codes_are_those_of_the_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = f8.decode(codes)
    assert np.array_equal(got, want, equal_nan=True)
    fine = ~np.isnan(got)
    assert np.array_equal(f8.encode(got[fine]), codes[fine])


def test_rounding():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(0, 100, 20000), rng.normal(0, 0.01, 20000), np.linspace(-448, 448, 9001)]).astype(np.float32)
    mid = (f8._TABLE[:-1] + f8._TABLE[1:]) / 2                       # ties
    x = np.concatenate([x, mid, -mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9)]).astype(np.float32)
    x = np.clip(x, -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(f8.encode(x), want)


def test_blocks():
    rng = np.random.default_rng(1)
    x = rng.normal(0, 1, (130, 300)).astype(np.float32)
    x[3, 200:] *= 1e4
    for rows in (1, 128):
        q, s = f8.quantize(x, rows)
        assert s.shape == ((3, 130) if rows == 1 else (2, 3))
        full = s.T if rows == 1 else np.repeat(s, 128, axis=0)[:130]
        back = f8.decode(q) * np.repeat(full, 128, axis=1)[:, :300]
        amax = np.repeat(full, 128, axis=1)[:, :300] * 448
        assert (np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, amax * 2.0 ** -10 / 448) * (1 + 1e-6)).all()
