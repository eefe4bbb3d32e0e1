"""Block-scaled 8-bit floating-point product and quantisation on the GPU against the oracle.

Codes and scales are defined by f32 operations: they are compared bit for bit.  Product: a block's 128 products are exact in f32; each of
the 128 additions of its sum is off by at most one step, 2^-23 of the magnitudes; the factor and the block's fma are 2 roundings, the
sum over nb blocks nb more, a join of 8 parts 3:
    |error| <= (128 2^-23 + (nb + 5) 2^-24) sum |x w| + half a step of the output.
"""
import numpy as np
import pytest
import torch

from oracle import f8 as oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


def pad(n, per):
    return (n + per - 1) // per * per


def quantize(B, x, K, rows, n_dev=None, extra=0):
    M = x.shape[0]
    kb = (K + 127) // 128
    q = torch.full((M + 1, pad(K, 16) + 16 * extra), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((kb + 1, pad(M, 4) + 4 * extra) if rows == 1 else ((M + 127) // 128 + 1, kb + extra), -7.5, device="cuda")
    B.quantize_f8(B.QuantizeF8Params(M, K, B.BF16 if x.dtype is torch.bfloat16 else B.F32, x.stride(0), q.stride(0), s.stride(0), rows), x,
                  q.view(F8), s, n_dev)
    return q, s


def check_quantize(B, x, K, rows, extra=3):
    M, kb = x.shape[0], (K + 127) // 128
    q, s = quantize(B, x, K, rows, extra=extra)
    wq, ws = oracle.quantize(x[:, :K].float().cpu().numpy(), rows)
    q, s = q.cpu().numpy(), s.cpu().numpy()
    r, c = ws.shape
    np.testing.assert_array_equal(s[:r, :c].view(np.uint32) & 0x7fffffff, ws.view(np.uint32) & 0x7fffffff if not np.isnan(ws).any() else s[:r, :c].view(np.uint32) & 0x7fffffff)
    assert np.array_equal(s[:r, :c], ws, equal_nan=True)
    assert np.array_equal(q[:M, :K], wq)
    assert (q[M:] == 0x55).all() and (q[:, K:] == 0x55).all() and (s[r:] == -7.5).all() and (s[:, c:] == -7.5).all()


@pytest.mark.parametrize("M,K", [(1, 1), (3, 127), (5, 128), (129, 129), (300, 2563), (64, 4096), (2, 20000), (1000, 515)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_bit_for_bit(B, M, K, dtype, rows):
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    x = torch.empty(M, pad(K, 8), device="cuda").normal_(0.0, 1.0, generator=g)
    x *= torch.exp(torch.empty(x.shape[1], device="cuda").normal_(0.0, 2.0, generator=g))
    x[:, K:] = 1e30                                                  # padding is not looked at
    check_quantize(B, x.to(DT[dtype]), K, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_values_where_it_can_go_wrong(B, dtype):
    x = torch.zeros(12, 256, device="cuda")
    steps = torch.from_numpy(np.concatenate([oracle._TABLE, (oracle._TABLE[:-1] + oracle._TABLE[1:]) / 2])[:253]).float()
    x[0, :253] = steps.cuda()                                        # codes and ties, scale 1 (448 is among them)
    x[1] = -x[0]
    x[2] = x[0] * 2.0 ** -130
    x[3] = x[0] * 2.0 ** 100
    x[4, 7] = float("nan")
    x[5, 200] = float("inf")
    x[6, 3] = 1e-42
    x[7] = torch.linspace(-1, 1, 256, device="cuda")
    x[8, 0], x[8, 1:] = 3e38, 1.0
    x[9] = torch.exp(torch.linspace(-20, 3, 256, device="cuda"))
    x[10, :] = -0.0
    x[11] = 448.0 * 3
    for rows in (1, 128):
        check_quantize(B, x.to(DT[dtype]), 256, rows, extra=0)


def make(B, M, K, N, seed, dtype="f32"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty(M, pad(K, 8), device="cuda").normal_(0.0, 1.0, generator=g)
    x *= torch.exp(torch.empty(x.shape[1], device="cuda").normal_(0.0, 1.5, generator=g))
    w = torch.empty(N, pad(K, 8), device="cuda").normal_(0.0, 0.02, generator=g)
    q, qs = quantize(B, x.to(DT[dtype]), K, 1, extra=1)
    p, ps = quantize(B, w.to(DT[dtype]), K, 128, extra=2)
    q[:, K:] = 0x7f                                                  # NaN codes behind the columns: not part of the product
    p[:, K:] = 0x7f
    return q, qs, p, ps


def product(B, M, K, N, q, qs, p, ps, out="f32", variant=0, n_dev=None, pitch=0):
    y = torch.full((M + 1, N + pitch), -7.5, dtype=DT[out], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.linear_f8(B.LinearF8Params(M, N, K, q.stride(0), p.stride(0), y.stride(0), qs.stride(0), ps.stride(0), B.BF16 if out == "bf16" else B.F32, variant),
                q.view(F8), qs, p.view(F8), ps, y, n_dev, status)
    return y, status


def check_product(y, M, K, N, q, qs, p, ps, rows=None):
    kb = (K + 127) // 128
    T = M if rows is None else rows
    h = lambda t: t.cpu().numpy()
    want, mag = oracle.linear(h(q)[:T, :K], h(qs)[:kb, :T], h(p)[:N, :K], h(ps)[:(N + 127) // 128, :kb])
    got = y[:T, :N].double().cpu().numpy()
    half = 2.0 ** -8 if y.dtype is torch.bfloat16 else U
    tol = (128 * 2.0 ** -23 + (kb + 5) * U) * mag
    bad = np.abs(got - want) > tol + half * (np.abs(want) + tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])
    assert bool((y[T:] == -7.5).all()) and bool((y[:, N:] == -7.5).all())


SHAPES = [(1, 1, 1), (1, 128, 128), (2, 129, 130), (16, 640, 257), (17, 1000, 100), (33, 2563, 300), (64, 4096, 1000), (65, 384, 129),
          (128, 1280, 2000), (129, 256, 512), (200, 2560, 3001), (513, 777, 1111), (1003, 2563, 501), (300, 8192, 70), (5, 20000, 40)]


@pytest.mark.parametrize("M,K,N", SHAPES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("variant", [0, 1, 2])
def test_product(B, M, K, N, out, variant):
    q, qs, p, ps = make(B, M, K, N, M + K + N)
    y, status = product(B, M, K, N, q, qs, p, ps, out, variant, pitch=5)
    check_product(y, M, K, N, q, qs, p, ps)
    again, _ = product(B, M, K, N, q, qs, p, ps, out, variant, pitch=5)
    assert torch.equal(y, again) and int(status) == 0


@pytest.mark.parametrize("variant", [1, 2])
def test_many_tiles(B, variant):
    """More tiles than CTAs, more blocks than slots and stages."""
    M, K, N = 700, 3200, 9000
    q, qs, p, ps = make(B, M, K, N, 3, "bf16")
    y, _ = product(B, M, K, N, q, qs, p, ps, "f32", variant)
    check_product(y, M, K, N, q, qs, p, ps)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(512, 700, 1024), (300, 5000, 1000), (257, 256, 4056)])
def test_aligned_outputs(B, out, M, K, N):
    """Rows of the output on 16 bytes: whole tiles leave by tiled copies."""
    q, qs, p, ps = make(B, M, K, N, 9)
    for pitch in (0, 8):
        y, _ = product(B, M, K, N, q, qs, p, ps, out, 1, pitch=pitch)
        check_product(y, M, K, N, q, qs, p, ps)


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("rows", [0, 1, 100, 299])
def test_true_count_on_the_device(B, rows, variant):
    M, K, N = 299, 300, 700
    q, qs, p, ps = make(B, M, K, N, 4)
    qs[:, rows:] = float("nan")                                      # rows behind the count are not part of anything
    y, _ = product(B, M, K, N, q, qs, p, ps, "f32", variant, torch.tensor([rows], dtype=torch.int32, device="cuda"))
    if rows:
        check_product(y, M, K, N, q, qs, p, ps, rows)
    else:
        assert bool((y == -7.5).all())


def test_invalid_blocks_make_their_products_invalid(B):
    M, K, N = 20, 300, 200
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.empty(M, 304, device="cuda").normal_(0.0, 1.0, generator=g)
    x[3, 290] = float("inf")
    x[9, 0] = float("nan")
    q, qs = quantize(B, x, K, 1)
    _, _, p, ps = make(B, M, K, N, 6)
    for variant in (1, 2):
        y, _ = product(B, M, K, N, q, qs, p, ps, "f32", variant)
        bad = y[:M].isnan().all(1)
        assert bad.nonzero().flatten().tolist() == [3, 9] and not bool(y[[t for t in range(M) if t not in (3, 9)]].isnan().any())


def test_captured_and_on_another_stream(B):
    M, K, N = 40, 500, 600
    q, qs, p, ps = make(B, M, K, N, 7)
    y, status = product(B, M, K, N, q, qs, p, ps)
    prm = B.LinearF8Params(M, N, K, q.stride(0), p.stride(0), N, qs.stride(0), ps.stride(0), B.F32)
    z = torch.zeros(M, N, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.linear_f8(prm, q.view(F8), qs, p.view(F8), ps, z)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(z, y[:M])
    side = torch.cuda.Stream()
    z.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        B.linear_f8(prm, q.view(F8), qs, p.view(F8), ps, z)
    side.synchronize()
    assert torch.equal(z, y[:M])


@pytest.mark.parametrize("variant", [1, 2])
def test_waits_are_bounded(B, variant):
    M, K, N = 300, 1024, 1000
    q, qs, p, ps = make(B, M, K, N, 8)
    _, status = product(B, M, K, N, q, qs, p, ps, "f32", B.LINEAR_F8_WAIT_SELF_TEST + variant)
    torch.cuda.synchronize()
    assert int(status) == B.STATUS_TIMEOUT
    y, status = product(B, M, K, N, q, qs, p, ps, "f32", variant)
    check_product(y, M, K, N, q, qs, p, ps)
    assert int(status) == 0
