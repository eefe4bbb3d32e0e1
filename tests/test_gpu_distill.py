"""Distillation from a teacher's top log-probs on the GPU against the float64 oracle.

Tolerances.  u = 2^-24.  A term e = 2^((z - m) c) carries the roundings of z - m, of c and of the product (3 u |x|, x = (z - m)/tau)
and the exponential (4 u); a thread adds n of them and rescales at most once per vector (5 u each), joins add 16 more.  So a
sum S of terms has a relative error of at most eS = (3 E|x| + 3 + 6 n + 16) u with E|x| = the mean of |x| under the terms, and so
has the sum over what is not listed, eR with its own mean.  The loss adds P ln S + r (ln S - ln S_rest) to sums in 64 bits:
    |loss error| <= P eS + r (eS + eR) + u |loss|.
A gradient entry w (s (G - share) - p): s carries eS + (3 |x| + 4) u, share eS + eR, and G, share, w and the products 8 roundings:
    |error| <= w s (G + share) (eS + eR + (3 |x| + 12) u) + 4 u w p + half a step of the type,
and where an exponential is below the normal numbers, 2^-126 w times what it is multiplied by: at most G + 17, since a share - G above 16
goes into the exponent.  The call that returns loss and gradient at once keeps the
exponentials of bf16 rows in 16 bits between its two passes: 2^-11 more relative to s, and, below 2^-14 of the largest unlisted entry
of the row, 2^-25 of that.
"""
import math

import numpy as np
import pytest
import torch

from oracle import distill as oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


def pad16(n, dtype):
    per = 8 if dtype == "bf16" else 4
    return (n + per - 1) // per * per


def make(T, V, dtype, K, seed, mask="none", extra=0):
    """Logits [T, padded V] and a teacher that mostly agrees with them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.empty(T, pad16(V, dtype) + extra, device="cuda").normal_(0.0, 2.0, generator=g)
    hot = (torch.randint(0, V, (T, 1), device="cuda", generator=g) + torch.arange(6, device="cuda") * max(1, V // 6)) % V
    z.scatter_add_(1, hot, torch.full((T, 6), 7.0, device="cuda"))
    if mask == "tail":
        z[:, V - V // 3:] = -math.inf
    elif mask == "sparse":
        z.masked_fill_(torch.rand(z.shape, device="cuda", generator=g) < 0.9, -math.inf)
    elif mask == "lowest":
        z.masked_fill_(torch.rand(z.shape, device="cuda", generator=g) < 0.7, float(torch.finfo(DT[dtype]).min))
    z = z.to(DT[dtype])
    t = z[:, :V].double().nan_to_num(neginf=-1e300) + torch.empty(T, V, device="cuda", dtype=torch.float64).normal_(0.0, 0.7, generator=g)
    lt = torch.log_softmax(t, 1)
    k = min(K, V)
    val, at = torch.topk(lt, k, dim=1)
    ids = torch.full((T, K), -1, dtype=torch.int32, device="cuda")
    lp = torch.full((T, K), -math.inf, device="cuda")
    dead = val < -1e30
    ids[:, :k] = torch.where(dead, -1, at).int()
    lp[:, :k] = torch.where(dead, torch.full_like(val, -math.inf), val).float()
    return z, ids, lp


class Run:
    """The three calls on the same inputs, every output in a field of marks."""

    def __init__(self, B, z, V, ids, lp, mode, tau, w=None, n_dev=None):
        T, K = ids.shape
        f32 = dict(dtype=torch.float32, device="cuda")
        prm = B.DistillParams(T, V, B.BF16 if z.dtype is torch.bfloat16 else B.F32, z.stride(0), K, mode, tau)
        mark = lambda: {n: torch.full((T + 16, c), -7.5, **f32) for n, c in (("loss", 1), ("lse", 1), ("stats", 4))}
        grad = lambda: torch.full((T + 2, z.stride(0)), -7.5, dtype=z.dtype, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.one, self.two = mark(), mark()
        self.g_bwd, self.g_step = grad(), grad()
        B.distill_topk(prm, z, ids, lp, n_dev, None, self.one["loss"], self.one["lse"], self.one["stats"], None, self.status)
        B.distill_topk_backward(prm, z, ids, lp, n_dev, self.one["stats"], w, self.g_bwd, self.status)
        B.distill_topk(prm, z, ids, lp, n_dev, w, self.two["loss"], self.two["lse"], self.two["stats"], self.g_step, self.status)
        inplace = z.clone()
        B.distill_topk_backward(prm, inplace, ids, lp, n_dev, self.one["stats"], w, inplace, self.status)
        instep = z.clone()
        B.distill_topk(prm, instep, ids, lp, n_dev, w, None, None, self.two["stats"], instep, self.status)
        torch.cuda.synchronize()
        n = T if n_dev is None else int(n_dev.item())
        for o in (self.one, self.two):
            for name, x in o.items():
                assert bool((x[n:] == -7.5).all()), name
        for x in (self.g_bwd, self.g_step):
            assert bool((x[n:] == -7.5).all()) and bool((x[:, V:] == -7.5).all())
        same = lambda a, b: bool(((a == b) | (a.isnan() & b.isnan())).all())
        assert same(inplace[:n, :V], self.g_bwd[:n, :V]) and same(instep[:n, :V], self.g_step[:n, :V])
        assert same(inplace[n:], z[n:]) and same(instep[:, V:], z[:, V:])


def check(r, z, V, ids, lp, mode, tau, w=None, rows=None):
    dtype = "bf16" if z.dtype is torch.bfloat16 else "f32"
    zh = z[:, :V].double().cpu().numpy()
    T = zh.shape[0] if rows is None else rows
    want = oracle.distill_topk(zh[:T], ids.cpu().numpy()[:T], lp.cpu().numpy()[:T], mode, tau)
    n = math.ceil(V / (32 if V <= 4096 else 128))
    wt = np.ones(T) if w is None else w.double().cpu().numpy()[:T]
    half = 2.0 ** -8 if dtype == "bf16" else U
    got = {k: {n_: x[:T].cpu().numpy() for n_, x in o.items()} for k, o in (("one", r.one), ("two", r.two))}
    grads = {"backward": r.g_bwd, "step": r.g_step}
    grads = {k: x[:T, :V].double().cpu().numpy() for k, x in grads.items()}
    for t in range(T):
        row = zh[t]
        if not np.isfinite(want["lse"][t]):
            for o in got.values():
                for name in ("loss", "lse"):
                    np.testing.assert_array_equal(o[name][t, 0], want[name][t])
            for k, g in grads.items():
                np.testing.assert_array_equal(g[t], want["dz"][t], err_msg=k)
            continue
        m = row.max()
        with np.errstate(all="ignore"):
            x = np.where(row > -np.inf, (row - m) / tau, 0.0)
            e = np.where(row > -np.inf, np.exp(x), 0.0)
        listed = np.zeros(V, dtype=bool)
        listed[ids[t].cpu().numpy()[ids[t].cpu().numpy() >= 0]] = True
        base = (3 + 6 * n + 16) * U
        eS = base + 3 * U * (e * np.abs(x)).sum() / e.sum()
        xr = x[~listed & (row > -np.inf)]                            # relative to their own maximum: their sum does not underflow
        mr = xr.max() if xr.size else 0.0
        er = np.where(listed | (row == -np.inf), 0.0, np.exp(np.minimum(x - mr, 0.0)))
        rest = er.sum()
        eR = base + (3 * U * (er * np.abs(x - mr)).sum() / rest + 3 * U * abs(mr) if rest > 0 else 0.0)
        P, rr = want["P"][t], want["r"][t]
        tol = P * eS + rr * (eS + eR)
        for o in got.values():
            a, b = o["loss"][t, 0], want["loss"][t]
            assert a == b or abs(a - b) <= tol + U * abs(b), ("loss", t, a, b, tol)
            a, b = o["lse"][t, 0], want["lse"][t]
            assert abs(a - b) <= eS + 4 * U * abs(np.log(e.sum())) + 3 * U * abs(m) / tau + U * abs(b), ("lse", t, a, b)
        s, G, ww = e / e.sum(), P + rr, abs(wt[t]) / tau
        to_rest = rr * er / rest if rest > 0 else er                 # s r / sigma
        p = np.abs(want["dz"][t] * tau - s * G + to_rest)
        size = s * G + to_rest
        tol = ww * size * (eS + eR + (3 * np.abs(x) + 12) * U) + 4 * U * ww * p + ww * (G + 17) * 2.0 ** -126
        b = want["dz"][t] * wt[t]
        for k, g in grads.items():
            more = tol
            if k == "step" and dtype == "bf16":
                more = tol + ww * (size * 2.0 ** -11 + 2.0 ** -25 * size[~listed].max(initial=0.0))
            bad = np.abs(g[t] - b) > more * (1 + half) + half * np.abs(b) + 1e-40
            assert not bad.any(), (k, t, np.flatnonzero(bad)[:5], g[t][bad][:5], b[bad][:5], more[bad][:5] if np.ndim(more) else more)


CASES = [
    # T, V, dtype, K, mode, tau, mask
    (1, 1, "f32", 1, 2, 1.0, "none"), (2, 5, "bf16", 3, 1, 1.0, "none"), (3, 7, "bf16", 7, 2, 0.7, "none"), (5, 33, "f32", 32, 2, 1.0, "tail"),
    (9, 250, "bf16", 20, 2, 0.7, "sparse"), (40, 1021, "f32", 5, 1, 0.7, "sparse"), (7, 1024, "bf16", 128, 2, 1.0, "none"),
    (300, 777, "bf16", 2, 0, 2.0, "tail"), (6, 4097, "f32", 33, 2, 1.0, "none"), (3, 5003, "bf16", 32, 2, 1.5, "lowest"),
    (5, 10001, "f32", 100, 0, 1.0, "lowest"), (4, 32003, "bf16", 20, 2, 1.0, "tail"), (2, 50304, "f32", 32, 2, 1.0, "none"),
    (3, 100003, "f32", 64, 1, 1.0, "sparse"), (2, 151936, "bf16", 20, 2, 1.0, "none"), (2, 151936, "f32", 1, 2, 0.5, "tail"),
    (1, 300007, "bf16", 128, 2, 1.0, "none"), (1, 1 << 20, "f32", 17, 2, 1.0, "none"), (700, 8200, "bf16", 9, 2, 1.0, "none"),
    (600, 20011, "bf16", 9, 2, 1.0, "sparse"), (320, 40000, "f32", 9, 1, 1.0, "none"),
]


@pytest.mark.parametrize("T,V,dtype,K,mode,tau,mask", CASES)
def test_against_oracle(B, T, V, dtype, K, mode, tau, mask):
    z, ids, lp = make(T, V, dtype, K, T + V, mask, extra=16)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    w = torch.empty(T, device="cuda").normal_(0.0, 1.0, generator=g)
    r = Run(B, z, V, ids, lp, mode, tau, w)
    rows = min(T, max(4, 400000 // V))
    check(r, z, V, ids, lp, mode, tau, w, rows)
    assert int(r.status.item()) == 0


@pytest.mark.parametrize("V,dtype", [(40, "f32"), (1000, "bf16"), (9001, "f32"), (60001, "bf16")])
@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("K", [8, 40])
def test_rows_where_it_can_go_wrong(B, V, dtype, mode, K):
    """Rows without entries, listed twice, all of their mass listed, masked, empty, invalid, far from zero, very peaked."""
    K = min(K, V)
    z, ids, lp = make(14, V, dtype, K, V + mode)
    low = float(torch.finfo(DT[dtype]).min)
    ids[0] = -1
    ids[1, 1] = ids[1, 0]
    ids[1, K - 1] = ids[1, 0]
    ids[2, :] = ids[2, 0].item()                                     # one token, K times
    lp[2, :] = math.log(0.9 / K)
    z[3] = -math.inf
    z[4] = -math.inf
    z[4, ids[4].clamp_min(0).long()] = 1.0                           # nothing left that is not listed
    lp[5, :] = -math.inf                                             # listed, all with probability 0
    z[6, ids[6, 0].long()] = -math.inf                               # a listed token that the student's mask forbids
    z[7, V // 2] = math.nan
    z[8, V - 1] = math.inf
    z[9] = low
    z[9, 3] = 2.0
    z[10, ids[10, 0].long()] = 60.0                                  # a student that leaves nothing: sigma around e^-50
    z[11] = (z[11].float() + 3e5 * (1 if dtype == "f32" else 1)).to(z.dtype)
    z[12] = low                                                      # all masked by the type's lowest value: uniform
    ids[13, ::2] = -1
    r = Run(B, z, V, ids, lp, mode, 1.0)
    check(r, z, V, ids, lp, mode, 1.0)


@pytest.mark.parametrize("V,dtype", [(500, "f32"), (3001, "bf16"), (60001, "f32")])
@pytest.mark.parametrize("tau", [0.02, 0.004, 30.0])
def test_far_temperatures(B, V, dtype, tau):
    """A cold student's unlisted tokens are far below the listed ones (sigma down to e^-2000): the loss and its gradient stay finite."""
    z, ids, lp = make(6, V, dtype, 6, V)
    lp -= 0.3                                                        # the teacher leaves a remainder
    r = Run(B, z, V, ids, lp, 2, tau)
    assert bool(r.one["loss"][:6].isfinite().all())
    check(r, z, V, ids, lp, 2, tau)


@pytest.mark.parametrize("V,dtype", [(40, "f32"), (250, "bf16"), (500, "f32"), (1000, "f32"), (1000, "bf16"), (2000, "bf16"), (5000, "f32"), (9001, "bf16"),
                                     (100003, "f32"), (151936, "bf16")])
@pytest.mark.parametrize("K", [8, 40])
def test_largest_logit(B, V, dtype, K):
    """The statistics' maximum, of rows with entries and without."""
    for T, mode in ((30, 0), (30, 1), (30, 2), (500, 2)):
        z, ids, lp = make(T, V, dtype, K, V + mode)
        ids[0], ids[5], ids[17] = -1, -1, -1
        r = Run(B, z, V, ids, lp, mode, 1.0)
        for o in (r.one, r.two):
            assert torch.equal(o["stats"][:T, 0], z[:, :V].float().amax(1))


@pytest.mark.parametrize("V,dtype,K", [(500, "f32", 6), (3001, "bf16", 6), (60001, "f32", 40), (151936, "bf16", 6)])
def test_normalized_lists_of_low_probability(B, V, dtype, K):
    """A list of unlikely tokens (e^-600 together) normalises as any other does."""
    z, ids, lp = make(6, V, dtype, K, V + 1)
    lp -= torch.tensor([0.0, 60.0, 90.0, 150.0, 400.0, 600.0], device="cuda")[:, None]
    r = Run(B, z, V, ids, lp, 1, 1.0)
    check(r, z, V, ids, lp, 1, 1.0)


@pytest.mark.parametrize("V,dtype", [(300, "f32"), (70001, "bf16")])
def test_bad_ids(B, V, dtype):
    z, ids, lp = make(6, V, dtype, 5, 3)
    good = Run(B, z, V, ids, lp, 2, 1.0)
    ids[2, 1], ids[4, 0] = V, -2
    r = Run(B, z, V, ids, lp, 2, 1.0)
    assert int(r.status.item()) == B.STATUS_BAD_TARGET
    for t in range(6):
        if t in (2, 4):
            assert float(r.one["loss"][t]) == 0 and float(r.two["loss"][t]) == 0
            assert bool((r.g_bwd[t, :V] == 0).all()) and bool((r.g_step[t, :V] == 0).all())
        else:
            assert torch.equal(r.g_bwd[t], good.g_bwd[t]) and torch.equal(r.g_step[t], good.g_step[t])


@pytest.mark.parametrize("T,V,dtype", [(50, 1021, "f32"), (9, 151936, "bf16")])
def test_true_count_on_the_device(B, T, V, dtype):
    z, ids, lp = make(T, V, dtype, 6, 4)
    n = torch.tensor([T - 4], dtype=torch.int32, device="cuda")
    ids[T - 4:] = V + 5                                              # not looked at
    r = Run(B, z, V, ids, lp, 2, 1.0, n_dev=n)
    check(r, z, V, ids, lp, 2, 1.0, rows=min(T - 4, 20))
    assert int(r.status.item()) == 0
    n.zero_()
    Run(B, z, V, ids, lp, 2, 1.0, n_dev=n)


def test_offsets_beyond_32_bits(B):
    T, V, ld = 3, 1000, (1 << 30) + 8
    z, ids, lp = make(T, V, "bf16", 4, 6)
    big = torch.empty((T - 1) * ld + pad16(V, "bf16"), dtype=torch.bfloat16, device="cuda").as_strided((T, V), (ld, 1))
    out = torch.empty((T - 1) * ld + pad16(V, "bf16"), dtype=torch.bfloat16, device="cuda").as_strided((T, V), (ld, 1))
    big.copy_(z[:, :V])
    want = Run(B, z, V, ids, lp, 2, 1.0)
    stats = torch.zeros(T, 4, device="cuda")
    prm = B.DistillParams(T, V, B.BF16, ld, 4, 2, 1.0)
    B.distill_topk(prm, big, ids, lp, None, None, None, None, stats, out)
    assert torch.equal(out, want.g_step[:T, :V])
    B.distill_topk_backward(prm, big, ids, lp, None, stats, None, out)
    assert torch.equal(out, want.g_bwd[:T, :V])


def test_captured_and_on_another_stream(B):
    T, V = 20, 20000
    z, ids, lp = make(T, V, "bf16", 10, 8)
    want = Run(B, z, V, ids, lp, 2, 1.0)
    prm = B.DistillParams(T, V, B.BF16, z.stride(0), 10, 2, 1.0)
    loss, stats, g = torch.zeros(T, device="cuda"), torch.zeros(T, 4, device="cuda"), torch.zeros_like(z)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.distill_topk(prm, z, ids, lp, None, None, loss, None, stats, g)
    z2, ids2, lp2 = make(T, V, "bf16", 10, 9)
    z.copy_(z2); ids.copy_(ids2); lp.copy_(lp2)
    graph.replay()
    torch.cuda.synchronize()
    second = Run(B, z2, V, ids2, lp2, 2, 1.0)
    assert torch.equal(loss, second.two["loss"][:T, 0]) and torch.equal(g[:, :V], second.g_step[:T, :V])
    assert not torch.equal(loss, want.two["loss"][:T, 0])
    side = torch.cuda.Stream()
    loss.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.distill_topk(prm, z, ids, lp, None, None, loss, None, stats, None)
    side.synchronize()
    assert torch.equal(loss, second.one["loss"][:T, 0])
    again = torch.zeros_like(z)
    B.distill_topk(prm, z, ids, lp, None, None, loss, None, stats, again, stream=side)
    side.synchronize()
    assert torch.equal(again[:, :V], second.g_step[:T, :V])
