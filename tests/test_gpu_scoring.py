"""The scoring operators on the GPU against the float64 oracle.

Tolerances.  u = 2^-24 is half an f32 step, relative.  A term e = 2^((z - m) c) carries the roundings of z - m, of c and of
the product (3 u |x| for x = (z - m)/tau) and the 2-ulp exponential (4 u); a thread adds n of them one after the other and
rescales its sums at most once per vector (5 u each: difference, product, exponential, two products), the joins of at most
512 partial sums add 16 more roundings.  So S = sum e has a relative error of at most
    eS = (3 E|x| + 3 + adds + 5 rescales + 16) u,   E|x| = sum p |x|,
which is the absolute error of l = ln S besides l's own rounding; Q/S = -E|x| carries twice that.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import scoring

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


def pad16(n, elem):
    per = 16 // elem
    return (n + per - 1) // per * per


GUARD = 64


class Fwd:
    """Buffers of one forward call, every output between guard bands."""

    def __init__(self, B, z, V, target, k, tau, variant=0, n_dev=None, status=None, skip=()):
        T = z.shape[0]
        self.T, self.k = T, k
        f32 = dict(dtype=torch.float32, device="cuda")
        self.raw = {n: torch.full((T * w + 2 * GUARD,), -7.5, **f32) for n, w in
                    dict(logp=1, entropy=1, lse=1, stats=4, top_logp=k).items()}
        self.raw["top_ids"] = torch.full((T * k + 2 * GUARD,), -77, dtype=torch.int32, device="cuda")
        o = {n: r[GUARD:r.numel() - GUARD] for n, r in self.raw.items()}
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda") if status is None else status
        prm = B.LogprobParams(T, V, B.BF16 if z.dtype is torch.bfloat16 else B.F32, z.stride(0), k, variant, tau)
        g = lambda n: None if n in skip else o[n]
        B.token_logprobs(prm, z, target, n_dev, g("logp") if target is not None else None, g("entropy"), g("lse"),
                         o["top_ids"] if k else None, o["top_logp"] if k else None, g("stats"), self.status)
        torch.cuda.synchronize()
        self.dev = o
        self.stats = o["stats"]

    def host(self):
        for n, r in self.raw.items():                                # nothing is written outside the arrays
            want = -77 if n == "top_ids" else -7.5
            assert bool((r[:GUARD] == want).all()) and bool((r[r.numel() - GUARD:] == want).all()), n
        o = {n: v.cpu().numpy() for n, v in self.dev.items()}
        o["stats"] = o["stats"].reshape(self.T, 4)
        o["top_ids"], o["top_logp"] = (o[n].reshape(self.T, self.k) for n in ("top_ids", "top_logp"))
        return o


def row_eps(z, tau, V, variant):
    """eS of each row (see above)."""
    with np.errstate(all="ignore"):
        m = z.max(axis=1, keepdims=True)
        x = np.where(z > -np.inf, (z - m) / tau, 0.0)
        e = np.where(z > -np.inf, np.exp(x), 0.0)
        ex = np.abs(e * x).sum(1) / np.maximum(e.sum(1), 1e-300)
    threads = 32 if (variant == 32 or (variant == 0 and V <= 12295)) else 128     # a warp per row, at most 1,536 vectors and a tail
    n = math.ceil(V / threads)
    return (3 * ex + 3 + n + 5 * n + 16) * U, ex, e.sum(1)


def check(got, want, z, target, tau, V, k, variant=0, rows=None):
    eS, ex, S = row_eps(z, tau, V, variant)
    rows = range(z.shape[0]) if rows is None else rows
    for t in rows:
        m = z[t].max()
        l = math.log(S[t]) if S[t] > 0 and math.isfinite(S[t]) else 0.0

        def near(a, b, tol, what):
            if abs(b) > 3.4028235677973366e38:                       # 2^128 - 2^103: rounds to an infinity in f32
                b = math.copysign(math.inf, b)
            if math.isnan(b):
                assert math.isnan(a), (what, t, a, b)
            elif math.isinf(b):
                assert a == b, (what, t, a, b)
            else:
                assert abs(a - b) <= tol, (what, t, a, b, abs(a - b), tol)
        base = eS[t] + 4 * U * abs(l)
        near(got["lse"][t], want["lse"][t], base + 3 * U * abs(m) / tau + U * abs(want["lse"][t]), "lse")
        near(got["entropy"][t], want["entropy"][t], base + ex[t] * (2 * eS[t] + 6 * U), "entropy")
        if target is not None and math.isfinite(m):
            d = abs(z[t, target[t]] - m) / tau if math.isfinite(z[t, target[t]]) else 0.0
            near(got["logp"][t], want["logp"][t], base + 4 * U * d + U * abs(want["logp"][t]) if math.isfinite(want["logp"][t]) else 0, "logp")
        elif target is not None:
            near(got["logp"][t], want["logp"][t], 0, "logp")
        assert list(got["top_ids"][t]) == list(want["top_ids"][t]), (t, got["top_ids"][t], want["top_ids"][t])
        for j in range(k):
            w = want["top_logp"][t, j]
            near(got["top_logp"][t, j], w, base + (5 * U * (abs(w) + abs(l)) if math.isfinite(w) else 0), "top_logp")


def make(T, V, dtype, seed, sigma=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.empty(T, pad16(V, 2 if dtype == "bf16" else 4), dtype=DT[dtype], device="cuda").normal_(0.0, sigma, generator=g)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    return z, y


def run(B, z, V, y, k, tau, variant=0):
    got = Fwd(B, z, V, y, k, tau, variant).host()
    zh = z[:, :V].double().cpu().numpy()
    yh = None if y is None else y.cpu().numpy()
    check(got, scoring.token_logprobs(zh, yh, k, tau), zh, yh, tau, V, k, variant)
    return got


# ---- forward ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, V, k, tau", [
    (1, 1, 1, 1.0), (3, 2, 5, 1.0), (2, 7, 7, 0.5), (5, 8, 3, 1.0), (9, 9, 0, 2.0), (17, 31, 32, 1.0), (4, 33, 32, 1.0),
    (33, 255, 20, 0.7), (70, 1021, 5, 0.7), (8, 1024, 8, 1.0), (3, 2048, 20, 1.0), (3, 4095, 20, 1.3), (3, 4104, 20, 1.0),
    (5, 8192, 32, 1.0), (2, 32001, 20, 1.0), (300, 5003, 4, 1.0), (1, 151936, 20, 1.0), (3, 151936, 32, 0.8)])
def test_forward(B, T, V, k, tau, dtype):
    z, y = make(T, V, dtype, T * 1000 + V)
    run(B, z, V, y, k, tau)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("variant", [32, 10128, 10256, 10512, 20128, 20256, 20512, 40128, 40256, 40512, 80128, 80256, 80512])
def test_every_launch_shape(B, variant, dtype):
    for T, V in ((3, 5003), (2, 40), (1, 3)):                        # fewer vectors than CTAs too
        z, y = make(T, V, dtype, V)
        run(B, z, V, y, 20, 0.9, variant)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, variant", [(8203, 0), (8203, 32), (20003, 10128), (20003, 10512), (151936, 10256), (151936, 0), (151937, 40256)])
def test_maxima_that_move(B, V, variant, dtype):
    """Rows whose maximum grows all along, or that most threads see nothing of: the lanes of a warp share their maximum."""
    lowest = float(torch.finfo(DT[dtype]).min)
    g = torch.Generator().manual_seed(V)
    z = torch.full((9, pad16(V, 2 if dtype == "bf16" else 4)), 7.0)
    z[0, :V] = torch.linspace(-30, 30, V)
    z[1, :V] = torch.linspace(30, -30, V)
    z[2, :V] = -math.inf
    z[2, V - 3:] = torch.tensor([1.0, 2.0, -5.0] + [0.0] * (z.shape[1] - V))
    z[3, :V] = torch.randn(V, generator=g).masked_fill(torch.rand(V, generator=g) < 0.99, -math.inf)
    z[4, :V] = torch.full((V,), -math.inf).masked_fill(torch.rand(V, generator=g) < 0.01, lowest)
    z[5, :V] = torch.full((V,), lowest).masked_fill(torch.rand(V, generator=g) < 0.5, -math.inf)
    z[5, V // 2] = 3.0
    z[6, :V] = torch.linspace(-400, 400, V)[torch.randperm(V, generator=g)]
    z[7, :V] = torch.where(torch.arange(V) // 8 % 32 == 5, torch.linspace(-9, 9, V), torch.tensor(-math.inf))     # one lane of each warp
    z[8, :V] = lowest
    z[8, V // 3] = -math.inf
    z = z.to(DT[dtype]).cuda()
    y = torch.tensor([5, V - 1, V - 2, 0, 1, V // 2, 7, 40, V // 3], dtype=torch.int32, device="cuda")
    run(B, z, V, y, 7, 0.9, variant)


@pytest.mark.parametrize("k", [0, 9])
@pytest.mark.parametrize("T", [19, 37, 49, 61, 91, 149, 184, 300, 371, 500, 745, 1490])
def test_many_row_shapes(B, T, k):
    """Counts of rows for which the library picks every split of a row and size of a CTA; first, last and some rows between."""
    for V, dtype in ((50003, "f32"), (17003, "bf16"), (6001, "f32")):
        z, y = make(T, V, dtype, T + V)
        z[1, 7:] = -math.inf
        got = Fwd(B, z, V, y, k, 0.8).host()
        pick = sorted({0, 1, 2, T // 3, T // 2, T - 2, T - 1})
        zh, yh = z[pick, :V].double().cpu().numpy(), y.cpu().numpy()[pick]
        check({n: v[pick] for n, v in got.items()}, scoring.token_logprobs(zh, yh, k, 0.8), zh, yh, 0.8, V, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1000, 20003])
@pytest.mark.parametrize("tau", [1e-6, 1e-3, 1e3, 1e6])
def test_extreme_temperatures(B, V, tau, dtype):
    """Temperatures at which the distribution is a single token, or uniform; masked entries too."""
    z, y = make(4, V, dtype, 17)
    z[1, : V // 2] = -math.inf
    z[2, :] = 0
    z[2, 5] = -1e10
    z[3, ::3] = float(torch.finfo(DT[dtype]).min)
    z[1, int(y[1])] = 1.0
    run(B, z, V, y, 5, tau)
    a, b = torch.randn(4, device="cuda"), torch.randn(4, device="cuda")
    zh, yh = z[:, :V].double().cpu().numpy(), y.cpu().numpy()
    want = scoring.token_logprobs_backward(zh, yh, a.double().cpu().numpy(), b.double().cpu().numpy(), tau)
    check_grad(backward(B, z, V, y, a, b, tau)[:, :V].double().cpu().numpy(), want, zh, yh, a.double().cpu().numpy(),
               b.double().cpu().numpy(), tau, dtype, V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, variant", [(151936, 10128), (151936, 10256), (300001, 10128), (131077, 20128), (600003, 10256), (40003, 32)])
def test_more_rounds_than_slots(B, V, variant, dtype):
    """Rows of more rounds than there are slots for their maxima: several rounds share one."""
    z, y = make(2, V, dtype, V)
    z[1, :V] = z[1, :V].round()                                      # and with many ties
    run(B, z, V, y, 20, 1.0, variant)


def special_rows(V, dtype):
    """Rows where a softmax or a selection goes wrong, as f32 [n, V]."""
    g = torch.Generator().manual_seed(V)
    low = torch.finfo(DT[dtype]).min
    rnd = torch.empty(V).normal_(0, 2, generator=g)
    rows = []
    rows.append(torch.full((V,), -math.inf))                                    # a mask that leaves nothing
    rows.append(torch.full((V,), float(low)))                                   # nothing but the type's lowest value
    rows.append(torch.where(torch.rand(V, generator=g) < 0.9, torch.tensor(-math.inf), rnd))
    rows.append(torch.where(torch.rand(V, generator=g) < 0.9, torch.tensor(float(low)), rnd))
    r = torch.full((V,), -math.inf); r[V // 2] = 1.5; rows.append(r)            # one entry
    r = torch.full((V,), float(low)); r[V - 1] = 3.0; rows.append(r)
    r = rnd.clone(); r[V // 3] = math.nan; rows.append(r)
    r = rnd.clone(); r[V - 1] = math.inf; rows.append(r)
    r = torch.full((V,), -math.inf); r[0] = math.nan; rows.append(r)
    rows.append(torch.zeros(V))                                                 # all tied
    r = torch.zeros(V); r[::2] = -0.0; rows.append(r)                           # -0 ties with +0
    rows.append(torch.full((V,), -3.25))
    rows.append(torch.arange(V).float() / 7)                                    # the maximum grows all the way
    rows.append(-torch.arange(V).float() / 7)
    rows.append(torch.randint(-2, 3, (V,), generator=g).float())                # a handful of values
    rows.append((torch.arange(V) % 37).float())
    r = rnd * 0.01; r[: max(1, V // 2)] += 5; rows.append(r)                    # half of the row far above the rest
    r = torch.zeros(V); r[torch.arange(V) % (512 * 8) < 24] = 1; r += rnd * 0.1; rows.append(r)   # three threads hold the large ones
    r = torch.zeros(V); r[torch.arange(V) % (256 * 4) < 16] = 1; r += rnd * 0.1; rows.append(r)
    r = torch.zeros(V); r[torch.arange(V) % (32 * 8) < 8] = 4; r += torch.arange(V) * 1e-3; rows.append(r)
    rows.append(rnd * 1e4)                                                      # large magnitudes
    rows.append(rnd + 3e4)
    rows.append(rnd * 1e37)
    rows.append(rnd * 1e-38)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, k, variant", [(9, 4, 0), (1000, 20, 0), (1500, 20, 0), (2001, 32, 0), (3500, 8, 0), (4099, 32, 0), (8200, 5, 0), (20000, 20, 10128), (20003, 20, 0),
                                           (20003, 32, 10512), (20003, 7, 40256), (20003, 20, 80128), (1027, 32, 32), (20003, 32, 32), (150003, 20, 10128)])
def test_special_rows(B, V, k, variant, dtype):
    rows = special_rows(V, dtype)
    z = torch.zeros(rows.shape[0], pad16(V, 2 if dtype == "bf16" else 4), dtype=DT[dtype], device="cuda")
    z[:, :V] = rows.to(DT[dtype])
    y = torch.arange(rows.shape[0], dtype=torch.int32, device="cuda") * 7919 % V
    run(B, z, V, y, k, 1.0, variant)
    run(B, z, V, y, k, 0.25, variant)


def test_forward_is_deterministic_and_stream_ordered(B):
    z, y = make(64, 20003, "bf16", 5)
    a = Fwd(B, z, 20003, y, 20, 1.0).host()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = Fwd(B, z, 20003, y, 20, 1.0).host()
    for n in a:
        assert np.array_equal(a[n].view(np.int32), b[n].view(np.int32)), n


@pytest.mark.parametrize("V", [1021, 20000])
def test_token_count_on_the_device_leaves_later_rows(B, V):
    z, y = make(40, V, "bf16", 1)
    z[23:] = math.nan
    y[23:] = -5
    for n in (0, 1, 23, 40):
        n_dev = torch.tensor([n], dtype=torch.int32, device="cuda")
        f = Fwd(B, z, V, y, 4, 1.0, n_dev=n_dev)
        o = f.host()
        m = min(n, 23)
        zh = z[:m, :V].double().cpu().numpy()
        check({k: v[:m] for k, v in o.items()}, scoring.token_logprobs(zh, y[:m].cpu().numpy(), 4, 1.0), zh, y[:m].cpu().numpy(), 1.0, V, 4)
        for name in ("logp", "entropy", "lse", "stats", "top_logp"):
            assert (o[name][n:] == -7.5).all(), name
        assert (o["top_ids"][n:] == -77).all()
        assert f.status.item() == (0 if n <= 23 else B.STATUS_BAD_TARGET)
    many = torch.tensor([1000], dtype=torch.int32, device="cuda")          # more than T_max: T_max rows
    assert np.isfinite(Fwd(B, z[:23], V, y[:23], 4, 1.0, n_dev=many).host()["logp"]).all()


@pytest.mark.parametrize("V", [1021, 20000])
def test_bad_targets_and_absent_outputs(B, V):
    z, y = make(6, V, "f32", 2)
    ref = Fwd(B, z, V, y, 3, 1.0).host()
    y2 = y.clone()
    y2[1], y2[4] = -1, V
    f = Fwd(B, z, V, y2, 3, 1.0)
    o = f.host()
    assert f.status.item() == B.STATUS_BAD_TARGET and o["logp"][1] == 0 and o["logp"][4] == 0
    keep = [0, 2, 3, 5]
    assert np.array_equal(o["logp"][keep], ref["logp"][keep])
    for n in ("entropy", "lse", "top_ids", "top_logp", "stats"):
        assert np.array_equal(o[n], ref[n]), n
    o = Fwd(B, z, V, None, 3, 1.0).host()                                  # no tokens given
    assert (o["logp"] == -7.5).all() and np.array_equal(o["top_ids"], ref["top_ids"])
    o = Fwd(B, z, V, y, 0, 1.0, skip=("entropy", "stats")).host()
    assert (o["entropy"] == -7.5).all() and (o["stats"] == -7.5).all() and np.array_equal(o["logp"], ref["logp"])


def test_rows_past_4_gib(B):
    V, T = 151936, 9000                                                    # 5.5 GB of f32 logits
    z = torch.zeros(T, V, dtype=torch.float32, device="cuda")
    y = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    z[8999, V - 1] = 20.0
    z[8998, 17] = 20.0
    f = Fwd(B, z, V, y, 2, 1.0)
    o = f.host()
    l = math.log1p((V - 1) * math.exp(-20.0))
    assert abs(o["logp"][8999] + l) < 1e-4 and abs(o["logp"][8998] + l + 20) < 1e-4 and abs(o["lse"][0] - math.log(V)) < 1e-4
    assert o["top_ids"][8999].tolist() == [V - 1, 0] and o["top_ids"][8998].tolist() == [17, 0] and o["top_ids"][5].tolist() == [0, 1]
    d = torch.zeros_like(z)
    a = torch.ones(T, device="cuda")
    B.token_logprobs_backward(B.LogprobParams(T, V, B.F32, V, 0, 0, 1.0), z, y, None, f.stats, a, None, d)
    p = math.exp(o["logp"][8998] + 20)
    assert abs(d[8998, 17].item() + p) < 1e-4 and abs(d[8998, V - 1].item() - 1) < 1e-4 and abs(d[8999, V - 1].item() - (1 - p)) < 1e-4


@pytest.mark.parametrize("T, V, dtype", [(4737, 37, "bf16"), (20011, 260, "f32"), (40001, 9, "f32"), (9000, 1500, "bf16"), (4999, 5003, "bf16"), (5000, 3001, "f32"), (4800, 20000, "bf16")])
def test_many_short_rows(B, T, V, dtype):
    """A warp takes several rows here: every row is what it is in a call of its own."""
    z, y = make(T, V, dtype, T)
    y[T - 3] = -1
    f = Fwd(B, z, V, y, 6, 1.0)
    o = f.host()
    assert f.status.item() == B.STATUS_BAD_TARGET
    few = [0, 1, 7, 8, 4735, T // 2, T - 3, T - 2, T - 1]            # (the same launch shape sums in the same order)
    for t in few:
        one = Fwd(B, z[t:t + 1], V, y[t:t + 1], 6, 1.0, 10128 if V == 20000 else 32).host()
        for n in o:
            assert np.array_equal(o[n][t:t + 1], one[n]), (n, t)
    z64 = z[:, :V].double()
    lnp = torch.log_softmax(z64, 1)
    ok = torch.arange(T) != T - 3
    want = lnp.gather(1, y.clamp_min(0).long()[:, None])[:, 0].cpu()
    # row_eps at its largest here: E|x| < 10 and 4 u |l| + 4 u |x_y| + u |logp| < 150 u
    tol = (3 * 10 + 6 * max(48, math.ceil(V / 32)) + 19 + 150) * U
    assert float((torch.from_numpy(o["logp"]).double() - want)[ok].abs().max()) < tol
    key = torch.sort(z64, dim=1, descending=True, stable=True)
    assert torch.equal(torch.from_numpy(o["top_ids"]).long(), key.indices[:, :6].cpu())


# ---- backward --------------------------------------------------------------------------------------
def check_grad(g, want, z, target, a, b, tau, dtype, V, variant=0):
    """|error| <= p-relative part (the exponent: 3 u |x| + l's own error and rounding, the exponential) x |dz|, plus the
    bracket's roundings x p, plus the token's own element, plus the output's rounding (half a step)."""
    eS, ex, S = row_eps(z, tau, V, variant)
    with np.errstate(all="ignore"):
        m = z.max(axis=1, keepdims=True)
        x = np.where(z > -np.inf, np.maximum((z - m) / tau, -1e6), 0.0)
        l = np.log(np.maximum(S, 1e-300))[:, None]
        p = np.where(z > -np.inf, np.exp(x - l), 0.0)
        plnp = np.where(p > 0, p * np.where(p > 0, x - l, 0.0), 0.0)
    H = -plnp.sum(1, keepdims=True)
    aa = np.abs(a)[:, None] if a is not None else 0.0
    bb = np.abs(b)[:, None] if b is not None else 0.0
    e = eS[:, None]
    bracket = aa + bb * (np.abs(np.where(p > 0, x - l, 0.0)) + H)
    tol = p / tau * (bracket * (3 * U * np.abs(x) + e + 4 * U * np.abs(l) + 16 * U)
                     + bb * (8 * U * (np.abs(x) + np.abs(l) + H) + 3 * e + ex[:, None] * (2 * e + 6 * U)) + 4 * U * aa)
    if a is not None:
        tol[np.arange(len(target)), target] += 6 * U * np.abs(a) / tau
    half = 2.0 ** -8 if dtype == "bf16" else U
    # a probability below the smallest normal f32, 2^-126, counts as 0: the element then lacks p x bracket / tau
    tol = tol * (1 + half) + half * np.abs(want) + 2.0 ** -126 * (1 + bracket / tau)
    bad = np.abs(g - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], g[bad][:3], want[bad][:3], tol[bad][:3])


def backward(B, z, V, y, a, b, tau, in_place=False, n_dev=None, status=None):
    f = Fwd(B, z, V, y, 0, tau, n_dev=n_dev)
    out = z if in_place else torch.full_like(z, 9.0)
    prm = B.LogprobParams(z.shape[0], V, B.BF16 if z.dtype is torch.bfloat16 else B.F32, z.stride(0), 0, 0, tau)
    B.token_logprobs_backward(prm, z, y, n_dev, f.stats, a, b, out, status)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, V, tau, terms", [(1, 1, 1.0, "ab"), (3, 9, 0.5, "ab"), (5, 31, 1.0, "a"), (70, 1021, 0.7, "ab"), (4, 4096, 1.0, "b"),
                                              (3, 4104, 1.0, "ab"), (2, 16392, 1.3, "ab"), (2, 32001, 1.0, "a"), (2, 151936, 1.0, "ab"), (3, 40, 1.0, "")])
def test_backward(B, T, V, tau, terms, dtype):
    z, y = make(T, V, dtype, V + T)
    a = torch.randn(T, device="cuda") if "a" in terms else None
    b = torch.randn(T, device="cuda") if "b" in terms else None
    zh = z[:, :V].double().cpu().numpy()
    ah, bh = (None if v is None else v.double().cpu().numpy() for v in (a, b))
    want = scoring.token_logprobs_backward(zh, y.cpu().numpy(), ah, bh, tau)
    out = backward(B, z, V, y, a, b, tau)
    check_grad(out[:, :V].double().cpu().numpy(), want, zh, y.cpu().numpy(), ah, bh, tau, dtype, V)
    assert bool((out[:, V:] == 9.0).all())                                 # the padding of the rows is left alone
    pad = z[:, V:].clone()
    same = backward(B, z, V, y, a, b, tau, in_place=True)
    assert torch.equal(same[:, :V], out[:, :V]) and torch.equal(z[:, V:], pad)


@pytest.mark.parametrize("T, V, dtype", [(100, 1000, "bf16"), (2000, 1000, "bf16"), (3000, 1203, "f32"), (1500, 2603, "bf16"), (1500, 5003, "bf16"), (1500, 2501, "f32"),
                                         (1200, 9603, "bf16"), (700, 17003, "bf16"), (60, 200003, "bf16"), (300, 20001, "f32")])
def test_backward_many_row_shapes(B, T, V, dtype):
    """Counts of rows for which the library takes every cut of a row and size of a CTA; sampled rows, masked ones and in place too."""
    z, y = make(T, V, dtype, T + V)
    z[2, 5:] = -math.inf
    z[3] = -math.inf                                                       # an empty row
    y[2], y[0], y[T - 1] = 3, V - 1, V // 2
    a, b = torch.randn(T, device="cuda"), torch.randn(T, device="cuda")
    pick = sorted({0, 1, 2, 3, T // 3, T // 2, T - 2, T - 1})
    zh, yh, ah, bh = (v.cpu().numpy()[pick] for v in (z[:, :V].double(), y, a.double(), b.double()))
    want = scoring.token_logprobs_backward(zh, yh, ah, bh, 0.8)
    out = backward(B, z, V, y, a, b, 0.8)
    check_grad(out[:, :V].double().cpu().numpy()[pick], want, zh, yh, ah, bh, 0.8, dtype, V)
    assert bool((out[:, V:] == 9.0).all()) and bool((out[3, :V] == 0).all())
    pad = z[:, V:].clone()
    same = backward(B, z, V, y, a, b, 0.8, in_place=True)
    assert torch.equal(same[:, :V], out[:, :V]) and torch.equal(z[:, V:], pad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 1000, 8200])
def test_backward_special_rows(B, V, dtype):
    rows = special_rows(V, dtype)
    keep = [i for i in range(rows.shape[0]) if not torch.isnan(rows[i]).any() and not torch.isposinf(rows[i]).any()]
    rows = rows[keep]
    z = torch.zeros(rows.shape[0], pad16(V, 2 if dtype == "bf16" else 4), dtype=DT[dtype], device="cuda")
    z[:, :V] = rows.to(DT[dtype])
    T = z.shape[0]
    zh = z[:, :V].double().cpu().numpy()
    yh = np.array([int(np.argmax(zh[t] > -np.inf)) for t in range(T)])      # a token that the mask allows, where there is one
    y = torch.tensor(yh, dtype=torch.int32, device="cuda")
    a, b = torch.randn(T, device="cuda"), torch.randn(T, device="cuda")
    want = scoring.token_logprobs_backward(zh, yh, a.double().cpu().numpy(), b.double().cpu().numpy(), 1.0)
    got = backward(B, z, V, y, a, b, 1.0)[:, :V].double().cpu().numpy()
    assert (got[0] == 0).all() and (got[zh == -np.inf] == 0).all()
    check_grad(got, want, zh, yh, a.double().cpu().numpy(), b.double().cpu().numpy(), 1.0, dtype, V)


def test_backward_of_invalid_rows_is_nan(B):
    z, y = make(2, 500, "f32", 3)
    z[0, 7] = math.nan
    z[1, 9] = math.inf
    one = torch.ones(2, device="cuda")
    assert bool(torch.isnan(backward(B, z, 500, y, one, one, 1.0)[:, :500]).all())


@pytest.mark.parametrize("V", [500, 20000])
def test_backward_bad_target_and_token_count(B, V):
    z, y = make(8, V, "f32", 4)
    y[2], y[5] = -3, V + 1
    a = torch.ones(8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n_dev = torch.tensor([7], dtype=torch.int32, device="cuda")
    out = backward(B, z, V, y, a, a, 1.0, n_dev=n_dev, status=status)
    assert status.item() == B.STATUS_BAD_TARGET
    assert bool((out[2, :V] == 0).all()) and bool((out[5, :V] == 0).all()) and bool((out[7] == 9.0).all())
    assert bool((out[0, :V] != 9.0).all())


def test_gradient_against_differences(B):
    """<dz, d> against central differences of the oracle's value: the error of the difference is at most h^2/6 |f'''| with
    |f'''| <= 6 (sum |a| + |b| (ln V + 6)) for |d| <= 1, tau = 1; h = 2^-8."""
    T, V, h = 4, 600, 2.0 ** -8
    z, y = make(T, V, "f32", 11)
    a, b, d = torch.randn(T), torch.randn(T), torch.rand(T, V) * 2 - 1
    g = backward(B, z, V, y, a.cuda(), b.cuda(), 1.0)[:, :V].double().cpu()
    zh, yh = z[:, :V].double().cpu().numpy(), y.cpu().numpy()

    def f(x):
        r = scoring.token_logprobs(x, yh, 0, 1.0)
        return (a.double().numpy() * r["logp"] + b.double().numpy() * r["entropy"]).sum()
    diff = (f(zh + h * d.double().numpy()) - f(zh - h * d.double().numpy())) / (2 * h)
    bound = h * h * float((a.abs() + b.abs() * (math.log(V) + 6)).sum())
    assert abs(float((g * d.double()).sum()) - diff) <= bound + 1e-4 * float((a.abs() + b.abs() * 8).sum())


# ---- 8-bit product: exact, bit for bit --------------------------------------------------------------
def f32_product(q, qs, w, ws):
    acc = (q.double() @ w.double().t()).cpu().numpy()                      # |sum| < 2^31: exact in f64
    s = (qs.cpu().numpy()[:, None] * ws.cpu().numpy()[None, :]).astype(np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        return (acc.astype(np.float32) * s).astype(np.float32)


def codes(rows, K, ld, seed, full=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-128, 128, (rows, ld), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M, N, K, variant", [
    (1, 1, 1, 0), (1, 5, 3, 0), (3, 128, 128, 0), (16, 129, 127, 0), (17, 300, 129, 0), (1, 4096, 2560, 0), (5, 100, 4097, 0),
    (33, 1000, 640, 0), (64, 4096, 4096, 0), (100, 257, 700, 0), (128, 640, 256, 0), (129, 640, 256, 0), (300, 130, 2000, 0),
    (257, 20000, 384, 0), (700, 3001, 513, 0), (1003, 5003, 2563, 0), (5000, 700, 200, 0), (1, 151936, 64, 0),
    (1, 1, 1, 1), (7, 300, 129, 1), (300, 513, 640, 1), (300, 513, 640, 2), (20, 64, 131071, 0), (130, 256, 131071, 1)])
def test_linear_i8(B, M, N, K, variant, out_dtype):
    ldx, ldw, ldo = (K + 15) // 16 * 16, (K + 15) // 16 * 16 + 16, N + 3
    x, w = codes(M, K, ldx, M + K), codes(N, K, ldw, N + K + 1)
    xs = torch.rand(M, device="cuda") * 0.01
    ws = torch.rand(N, device="cuda") * 0.01
    out = torch.full((M + 2, ldo), 5.0, dtype=DT[out_dtype], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.linear_i8(B.LinearI8Params(M, N, K, ldx, ldw, ldo, B.BF16 if out_dtype == "bf16" else B.F32, variant), x, xs, w, ws, out, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    want = torch.from_numpy(f32_product(x[:, :K], xs, w[:, :K], ws)).to(DT[out_dtype])
    assert torch.equal(out[:M, :N].cpu(), want)
    assert bool((out[:M, N:] == 5.0).all()) and bool((out[M:] == 5.0).all())


@pytest.mark.parametrize("M", [33, 64, 65, 96, 128, 160, 192, 224, 250, 256, 480])
def test_linear_i8_every_token_tile(B, M):
    """594 channel tiles: the pair kernel takes the token tile that holds M with the least waves (64, 96, ... 256)."""
    N, K = 151936, 48
    x, w = codes(M, K, K, M), codes(N, K, K, 7)
    xs, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    out = torch.zeros(M, N, device="cuda")
    B.linear_i8(B.LinearI8Params(M, N, K, K, K, N, B.F32, 1), x, xs, w, ws, out)
    assert torch.equal(out.cpu(), torch.from_numpy(f32_product(x, xs, w, ws)))


def test_quantize_then_product_is_ordered(B):
    """The product starts setting up while the quantisation runs: it must still see all of its rows, call after call."""
    M, N, K = 3000, 512, 1024
    w = codes(N, K, K, 7)
    ws = torch.rand(N, device="cuda")
    xs = [torch.randn(M, K, device="cuda") * (i + 1) for i in range(4)]
    q, s = torch.zeros(M, K, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda")
    outs = [torch.zeros(M, N, device="cuda") for _ in xs]
    for _ in range(3):
        for x, out in zip(xs, outs):
            B.quantize_rows_i8(B.QuantizeParams(M, K, B.F32, K, K), x, q, s)
            B.linear_i8(B.LinearI8Params(M, N, K, K, K, N, B.F32), q, s, w, ws, out)
    for x, out in zip(xs, outs):
        wq, wsc = scoring.quantize_rows_i8(x.cpu().numpy())
        want = f32_product(torch.from_numpy(wq).cuda(), torch.from_numpy(wsc), w, ws)
        assert torch.equal(out.cpu(), torch.from_numpy(want))


@pytest.mark.parametrize("M, variant", [(1, 2), (16, 2), (40, 2), (100, 2), (256, 1), (256, 2)])
def test_linear_i8_extreme_sums(B, M, variant):
    """Every product is (-128)^2 or -128 * 127: the sums reach the ends of int32."""
    K, N = 131071, 130
    ld = 131072
    x = torch.full((M, ld), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, ld), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    out = torch.zeros(M, N, device="cuda")
    one = torch.ones(max(M, N), device="cuda")
    B.linear_i8(B.LinearI8Params(M, N, K, ld, ld, N, B.F32, variant), x, one, w, one, out)
    assert bool((out[:, 0::2] == np.float32(16384 * K)).all()) and bool((out[:, 1::2] == np.float32(-128 * 127 * K)).all())


@pytest.mark.parametrize("M, variant", [(40, 0), (300, 1), (300, 2)])
def test_linear_i8_token_count_on_the_device(B, M, variant):
    N, K = 300, 256
    x, w = codes(M, K, K, 1), codes(N, K, K, 2)
    xs, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    want = torch.from_numpy(f32_product(x, xs, w, ws))
    for n in (0, 1, M // 2, M, M + 9):
        n_dev = torch.tensor([n], dtype=torch.int32, device="cuda")
        out = torch.full((M, N), 5.0, device="cuda")
        B.linear_i8(B.LinearI8Params(M, N, K, K, K, N, B.F32, variant), x, xs, w, ws, out, n_dev)
        m = min(n, M)
        assert torch.equal(out[:m].cpu(), want[:m]) and bool((out[m:] == 5.0).all())


def test_linear_i8_scales_that_are_no_numbers(B):
    x, w = codes(4, 64, 64, 1), codes(32, 64, 64, 2)
    xs, ws = torch.ones(4, device="cuda"), torch.ones(32, device="cuda")
    xs[1], ws[3] = math.nan, math.inf
    out = torch.zeros(4, 32, device="cuda")
    B.linear_i8(B.LinearI8Params(4, 32, 64, 64, 64, 32, B.F32), x, xs, w, ws, out)
    nan = torch.isnan(out)
    assert bool(nan[1].all()) and not bool(nan[0, :3].any()) and bool(torch.isinf(out[0, 3]) | torch.isnan(out[0, 3]))


@pytest.mark.parametrize("variant", [101, 102])
def test_linear_i8_bounded_waits(B, variant):
    x, w = codes(200, 256, 256, 1), codes(300, 256, 256, 2)
    xs, ws = torch.ones(200, device="cuda"), torch.ones(300, device="cuda")
    out = torch.zeros(200, 300, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.linear_i8(B.LinearI8Params(200, 300, 256, 256, 256, 300, B.F32, variant), x, xs, w, ws, out, status=status)
    torch.cuda.synchronize()
    assert status.item() == B.STATUS_TIMEOUT
    status.zero_()                                                          # the device goes on working
    B.linear_i8(B.LinearI8Params(200, 300, 256, 256, 256, 300, B.F32, variant - 100), x, xs, w, ws, out, status=status)
    assert status.item() == 0 and torch.equal(out.cpu(), torch.from_numpy(f32_product(x, xs, w, ws)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M, K", [(1, 1), (3, 7), (5, 8), (2, 129), (9, 2560), (4, 4097), (2, 30001), (300, 64), (5000, 1000), (2, 4096), (6, 4104),
                                  (700, 500), (2001, 1003), (1000, 2005), (300, 4001), (20, 4003), (700, 7001), (701, 8200), (1300, 16003), (300, 12001), (40, 40003)])
def test_quantize_rows(B, M, K, dtype):
    ldx, ldq = pad16(K, 2 if dtype == "bf16" else 4), (K + 15) // 16 * 16 + 16
    x = torch.empty(M, ldx, device="cuda").normal_(0, 3).to(DT[dtype])
    x[:, K:] = math.nan                                                     # the rows' padding is not looked at
    if M > 2:
        x[0, :K] = 0
        x[1, K // 2] = math.inf
        x[2, :K] = (torch.arange(K, device="cuda") % 255 - 127).to(DT[dtype]) * 0.5      # many exact ties
    if M > 4:
        x[3, K - 1] = math.nan
        x[4, :K] = 1e-42                                                    # the scale underflows
    q = torch.full((M + 1, ldq), 99, dtype=torch.int8, device="cuda")
    s = torch.full((M + 1,), 5.0, device="cuda")
    B.quantize_rows_i8(B.QuantizeParams(M, K, B.BF16 if dtype == "bf16" else B.F32, ldx, ldq), x, q, s)
    wq, ws = scoring.quantize_rows_i8(x[:, :K].float().cpu().numpy())
    assert np.array_equal(q[:M, :K].cpu().numpy(), wq) and np.array_equal(s[:M].cpu().numpy(), ws, equal_nan=True)
    assert bool((q[:M, K:] == 99).all()) and bool((q[M] == 99).all()) and s[M].item() == 5.0
    n_dev = torch.tensor([M // 2], dtype=torch.int32, device="cuda")
    q.fill_(99)
    B.quantize_rows_i8(B.QuantizeParams(M, K, B.BF16 if dtype == "bf16" else B.F32, ldx, ldq), x, q, s, n_dev)
    assert np.array_equal(q[:M // 2, :K].cpu().numpy(), wq[:M // 2]) and bool((q[M // 2:] == 99).all())


# ---- together, as a step uses them ------------------------------------------------------------------
def make_step(V, T, dtype="f32", n=None):
    from paper_2603_04135_b200.step import DppoStep
    st = DppoStep(2, 2, 512, 4, 0.0, 0.0, V, dtype, T, temperature=0.9)
    st.counts[3] = T if n is None else n
    return st


@pytest.mark.parametrize("T, n, chunk", [(50, 50, 16), (50, 33, 16), (300, 290, 2048), (1, 1, 2048)])
def test_step_scores_hidden_states(B, T, n, chunk):
    """hidden -> codes -> product -> scores, against the oracle on the same codes: the f32 logits carry 3 roundings."""
    from paper_2603_04135_b200.step import quantize_rows_i8
    H, V, k = 136, 1003, 6
    st = make_step(V, T, n=n)
    hidden = torch.randn(T, H, device="cuda").to(torch.bfloat16)
    W = torch.randn(V, H, device="cuda").to(torch.bfloat16) / math.sqrt(H) * 2
    Wq, Ws = quantize_rows_i8(W)
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    got = st.score_hidden_i8(hidden, Wq, Ws, y, top_k=k, chunk_tokens=chunk)
    again = st.score_hidden_i8(hidden, Wq, Ws, y, top_k=k, chunk_tokens=chunk, out={x: v.clone() for x, v in got.items()})
    assert st.status.item() == 0
    q, s = scoring.quantize_rows_i8(hidden.float().cpu().numpy())
    wq, ws = scoring.quantize_rows_i8(W.float().cpu().numpy())
    assert np.array_equal(wq, Wq.cpu().numpy())
    z = f32_product(torch.from_numpy(q).cuda(), torch.from_numpy(s), torch.from_numpy(wq).cuda(), torch.from_numpy(ws)).astype(np.float64)[:n]
    want = scoring.token_logprobs(z, y.cpu().numpy(), k, 0.9)
    o = {x: v.cpu().numpy() for x, v in got.items()}
    check({x: v[:n] for x, v in o.items()}, want, z, y.cpu().numpy(), 0.9, V, k)
    assert (o["logp"][n:] == 0).all() and (o["top_ids"][n:] == -1).all()
    for x in got:
        assert torch.equal(got[x], again[x]), x


def test_step_scores_feed_the_loss_and_its_gradient(B):
    """score() of the current policy as logp_old makes every ratio 1 in the loss sweep; score_backward with
    dlogp = -A W is then the gradient that the loss sweep writes (beta = 0)."""
    from paper_2603_04135_b200 import synth
    from paper_2603_04135_b200.step import DppoStep
    w = synth.WORKLOADS["config0"]
    batch = synth.make_batch(w, 0)
    T_max = int(batch.loss_len.sum())
    st = DppoStep(w.P, w.G, w.L_row, w.N_win, 0.0, 0.0, w.V, w.dtype, T_max, beta=0.0)
    st.set_batch(batch.rewards, batch.unit_len, batch.loss_len)
    st.prune_pack()
    T = st.n_tokens()
    tok = synth.make_token_inputs(w, T_max, 0, device="cuda:0")
    scored = st.score(tok.logits, tok.target, top_k=4)
    d_loss = torch.zeros_like(tok.logits)
    st.loss(tok.logits, tok.target, scored["logp"], scored["logp"], d_loss)
    assert st.status.item() == 0
    assert torch.allclose(st.logp_out[:T], scored["logp"][:T], rtol=0, atol=2e-5) and torch.allclose(st.lse_out[:T], scored["lse"][:T], rtol=0, atol=2e-5)
    cu = st.cu_seqlens.cpu().numpy()
    order = st.order.cpu().numpy()
    dlogp = torch.zeros(T_max)
    for s in range(int(st.counts[0])):
        lo, hi, unit = int(cu[s]), int(cu[s + 1]), int(order[s])
        if hi > lo:
            dlogp[lo:hi] = -float(st.adv[unit]) * float(st.w_seq[unit]) / (hi - lo)
    d = st.score_backward(tok.logits, tok.target, scored, dlogp=dlogp.cuda())
    # both are f32 evaluations of the same expression: the ratio exp(logp - logp_old) is 1 within 2e-5
    scale = float(dlogp.abs().max())
    assert float((d[:T] - d_loss[:T]).abs().max()) <= 4e-5 * scale
    st.score_backward(tok.logits, tok.target, scored, dlogp=dlogp.cuda(), dlogits=tok.logits)        # in place
    assert torch.equal(tok.logits[:T], d[:T])


def test_captured_and_replayed(B):
    V, T, H, k = 4001, 24, 256, 5
    ld = pad16(V, 4)
    x = torch.randn(T, H, device="cuda")
    W = codes(V, H, H, 3)
    ws = torch.rand(V, device="cuda") * 1e-3
    f32 = dict(dtype=torch.float32, device="cuda")
    q, s, z, dz = torch.zeros(T, H, dtype=torch.int8, device="cuda"), torch.zeros(T, **f32), torch.zeros(T, ld, **f32), torch.zeros(T, ld, **f32)
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    logp, H_, lse, stats = torch.zeros(T, **f32), torch.zeros(T, **f32), torch.zeros(T, **f32), torch.zeros(T, 4, **f32)
    ids, tl = torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(T, k, **f32)
    a = torch.ones(T, **f32)

    def work():
        B.quantize_rows_i8(B.QuantizeParams(T, H, B.F32, H, H), x, q, s)
        B.linear_i8(B.LinearI8Params(T, V, H, H, H, ld, B.F32), q, s, W, ws, z)
        prm = B.LogprobParams(T, V, B.F32, ld, k, 0, 1.0)
        B.token_logprobs(prm, z, y, None, logp, H_, lse, ids, tl, stats)
        B.token_logprobs_backward(prm, z, y, None, stats, a, a, dz)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in (1, 2):
        torch.manual_seed(seed)
        x.copy_(torch.randn(T, H, device="cuda"))
        outs = (q, s, z, logp, H_, lse, ids, tl, dz)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        work()
        torch.cuda.synchronize()
        for r, o in zip(replayed, outs):
            assert torch.equal(r, o)


def test_calls_on_two_streams_at_once(B):
    """Nothing is shared between calls: the same work on two streams at a time gives what it gives alone."""
    V, T, K, N = 20003, 37, 640, 3000
    z, y = make(T, V, "bf16", 9)
    x, w = codes(T, K, K, 1), codes(N, K, K, 2)
    xs, ws = torch.rand(T, device="cuda"), torch.rand(N, device="cuda")

    def work():
        o = torch.zeros(T, N, device="cuda")
        logp, ids, tl = torch.zeros(T, device="cuda"), torch.zeros(T, 8, dtype=torch.int32, device="cuda"), torch.zeros(T, 8, device="cuda")
        return o, logp, ids, tl

    def go(b):
        B.linear_i8(B.LinearI8Params(T, N, K, K, K, N, B.F32), x, xs, w, ws, b[0])
        B.token_logprobs(B.LogprobParams(T, V, B.BF16, z.stride(0), 8, 0, 1.0), z, y, None, b[1], None, None, b[2], b[3], None)
    alone = work()
    go(alone)
    streams = [torch.cuda.Stream() for _ in range(2)]
    bufs = [[work() for _ in range(8)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(8):
        for s, bs in zip(streams, bufs):
            with torch.cuda.stream(s):
                go(bs[i])
    torch.cuda.synchronize()
    for bs in bufs:
        for b in bs:
            for got, want in zip(b, alone):
                assert torch.equal(got, want)


@pytest.mark.parametrize("T, V, dtype", [(1, 20000, "bf16"), (40, 20000, "bf16"), (3000, 300, "f32"), (4000, 4001, "f32")])
def test_dependent_calls_back_to_back(B, T, V, dtype):
    """A call may be set up while the one before it runs: chains in which each reads what the last wrote (in place, into
    shared buffers) give what the same calls give with a wait after each."""
    z0, y = make(T, V, dtype, T + V)
    f32 = dict(dtype=torch.float32, device="cuda")

    def chain(wait):
        z = z0.clone()
        logp, H, lse, stats = torch.zeros(T, **f32), torch.zeros(T, **f32), torch.zeros(T, **f32), torch.zeros(T, 4, **f32)
        ids, tl = torch.zeros(T, 6, dtype=torch.int32, device="cuda"), torch.zeros(T, 6, **f32)
        n_dev = torch.tensor([T], dtype=torch.int32, device="cuda")
        kept = []
        torch.cuda.synchronize()
        for i in range(6):
            prm = B.LogprobParams(T, V, B.BF16 if dtype == "bf16" else B.F32, z.stride(0), 6, 0, 1.0)
            B.token_logprobs(prm, z, y, n_dev, logp, H, lse, ids, tl, stats)
            if wait:
                torch.cuda.synchronize()
            B.token_logprobs_backward(prm, z, y, n_dev, stats, logp, H, z)        # in place: the next call's logits
            if wait:
                torch.cuda.synchronize()
            if i % 2:
                z.mul_(3.0).add_(0.25)                                            # a kernel that knows nothing of it
                kept += [x.clone() for x in (logp, H, lse, ids, tl, z)]
        torch.cuda.synchronize()
        return kept
    for a, b in zip(chain(True), chain(False)):
        assert torch.equal(a, b)


def test_events_between_calls_are_kept(B):
    """A call that may be set up early still waits for another stream's event (and a copy) in front of it."""
    V, T = 5003, 20
    z, y = make(T, V, "f32", 1)
    z2, _ = make(T, V, "f32", 2)
    want = Fwd(B, z2, V, y, 4, 1.0).host()
    prm = B.LogprobParams(T, V, B.F32, z.stride(0), 0, 0, 1.0)
    one, stats, dz = torch.ones(T, device="cuda"), torch.zeros(T, 4, device="cuda"), torch.zeros_like(z)
    side = torch.cuda.Stream()
    for _ in range(3):
        buf = z.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                            # about 10 ms
            buf.copy_(z2)
            done = torch.cuda.Event()
            done.record()
        B.token_logprobs(prm, z, y, None, one, None, None, None, None, stats)          # lets its successor start early
        torch.cuda.current_stream().wait_event(done)
        f = Fwd(B, buf, V, y, 4, 1.0)
        got = f.host()
        for n in want:
            assert np.array_equal(got[n], want[n]), n


def test_native_marshalling_takes_the_plain_case_only(B):
    """The plain case is marshalled natively; addresses, parameters, views and explicit streams go through Python and do the
    same; what is wrong is named by the same errors either way."""
    T, V, k = 6, 1003, 3
    z, y = make(T, V, "f32", 3)
    f = lambda *s: torch.zeros(*s, device="cuda")
    logp, ent, lse, stats, tl = f(T), f(T), f(T), f(T, 4), f(T, k)
    ids = torch.zeros(T, k, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    prm = B.LogprobParams(T, V, B.F32, z.stride(0), k, 0, 1.0)
    plain = (z, y, None, logp, ent, lse, ids, tl, stats)
    native = getattr(B._native, "__name__", "").endswith("_marshal")
    assert B._native.token_logprobs(prm, *plain, status, None) == (0 if native else None)
    B.token_logprobs(prm, *plain, status)
    want = [t.clone() for t in (logp, ent, lse, ids, tl, stats)]
    others = [((z[:, :V],) + plain[1:], None), ((torch.nn.Parameter(z),) + plain[1:], None), (plain, torch.cuda.current_stream()),
              ((z.data_ptr(), y.data_ptr(), None) + tuple(t.data_ptr() for t in plain[3:]), None)]
    for args, stream in others:
        for t in (logp, ent, lse, ids, tl, stats):
            t.zero_()
        assert B._native.token_logprobs(prm, *args, status, stream) is None
        B.token_logprobs(prm, *args, status, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (logp, ent, lse, ids, tl, stats)))

    def code(prm, *args):
        with pytest.raises(B.DppoError) as e:
            B.token_logprobs(prm, *args, status)
        return e.value.code
    assert code(prm, z.double(), *plain[1:]) == B.ERR_INVALID_ARG
    assert code(prm, z.cpu(), *plain[1:]) == B.ERR_INVALID_ARG
    assert code(prm, z[:5].clone(), *plain[1:]) == B.ERR_BAD_SHAPE
    assert code(prm, z, y[:5].clone(), *plain[2:]) == B.ERR_BAD_SHAPE
    assert code(prm, z, y, None, f(2 * T)[::2], *plain[4:]) == B.ERR_BAD_SHAPE
    assert code(prm, None, *plain[1:]) == B.ERR_INVALID_ARG
    assert code(B.LogprobParams(T, V, B.F32, z.stride(0), k, 77, 1.0), *plain) == B.ERR_UNSUPPORTED
    assert code(B.LogprobParams(T, V, 9, z.stride(0), k, 0, 1.0), *plain) in (B.ERR_UNSUPPORTED, B.ERR_INVALID_ARG)
    with pytest.raises((AttributeError, ctypes.ArgumentError)):          # the params of another call
        B.token_logprobs(B.LinearI8Params(T, V, 64, 64, 64, V, 0), *plain, status)
    assert status.item() == 0


def test_calls_from_two_threads(B):
    """Two Python threads, a stream each, the same work at the same time."""
    import threading
    V, T = 20003, 31
    z, y = make(T, V, "bf16", 12)
    want = Fwd(B, z, V, y, 8, 1.0).host()
    got, errors = {}, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    got[i] = Fwd(B, z, V, y, 8, 1.0).host()
        except Exception as e:                                       # noqa: BLE001  (reported by the main thread)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for o in got.values():
        for n in want:
            assert np.array_equal(o[n].view(np.int32), want[n].view(np.int32)), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 1000, 8200])
@pytest.mark.parametrize("m, tau", [(-1e30, 1.0), (-1e12, 1.0), (1e11, 1.0), (1e36, 1.0), (7e5, 1.0), (7.5e5, 1.0), (-7.5e5, 1.0), (-1e9, 0.01),
                                    (1e8, 1e-3), (33024.0, 1e-6), (4e4, 1e-6), (-1e11, 1e6)])
def test_backward_of_a_maximum_far_from_zero(B, m, tau, V, dtype):
    """Rows whose maximum is large against the temperature: entries below it, masked ones too, keep their own probability
    (0 here: `lower` is more than 104 tau below m)."""
    m = float(torch.tensor(m).to(DT[dtype]))
    g = torch.Generator().manual_seed(V)
    kind = torch.randint(0, 4, (5, V), generator=g)
    lower = float(torch.tensor(m - abs(m) * 2.0 ** -6).to(DT[dtype]))
    rows = torch.where(kind == 0, m, torch.where(kind == 1, lower, torch.tensor(-math.inf)))
    rows[0] = m
    rows[0, V // 2:] = -math.inf
    rows[1] = -math.inf
    rows[1, V - 1] = m                                                     # one token
    rows[2] = lower
    rows[2, V // 3] = m
    rows[3, 0], rows[4, 1] = m, m
    rows[4, V - 2] = lower                                                 # the given token is not the most likely one
    z = torch.zeros(5, pad16(V, 2 if dtype == "bf16" else 4), dtype=DT[dtype], device="cuda")
    z[:, :V] = rows.to(DT[dtype])
    yh = np.array([0, V - 1, V // 3, 0, V - 2])
    a, b = torch.randn(5, device="cuda"), torch.randn(5, device="cuda")
    zh = z[:, :V].double().cpu().numpy()
    ah, bh = a.double().cpu().numpy(), b.double().cpu().numpy()
    want = scoring.token_logprobs_backward(zh, yh, ah, bh, tau)
    out = backward(B, z, V, torch.tensor(yh, dtype=torch.int32, device="cuda"), a, b, tau)
    got = out[:, :V].double().cpu().numpy()
    assert (got[zh == -np.inf] == 0).all()
    check_grad(got, want, zh, yh, ah, bh, tau, dtype, V)


def test_matrices_of_other_ranks_and_slices(B):
    """A matrix is taken in any shape whose own elements are the rows; rows of its storage that were not passed are refused, and
    not written."""
    T, V, ld, k = 10, 1003, 1008, 3
    z, y = make(T, V, "bf16", 21)
    assert z.shape[1] == ld
    want = Fwd(B, z, V, y, k, 1.0).host()
    prm = B.LogprobParams(T, V, B.BF16, ld, k, 0, 1.0)
    f = lambda *s: torch.zeros(*s, device="cuda")
    stats, a = f(T, 4), torch.ones(T, device="cuda")
    dz = torch.full_like(z, 9.0)

    def call(logits):
        logp, ids, tl = f(T), torch.zeros(T, k, dtype=torch.int32, device="cuda"), f(T, k)
        B.token_logprobs(prm, logits, y, None, logp, None, None, ids, tl, stats)
        return logp.cpu().numpy(), ids.cpu().numpy()
    for logits in (z, z[:, :V], z.view(2, 5, ld), z.view(2, 5, ld)[:, :, :V], z.view(-1), z.view(T, 1, ld)):
        logp, ids = call(logits)
        assert np.array_equal(logp, want["logp"]) and np.array_equal(ids, want["top_ids"])
    B.token_logprobs_backward(prm, z, y, None, stats, a, None, dz)
    grad = dz[:, :V].clone()
    seqs = torch.full((2, 6, ld), 9.0, dtype=z.dtype, device="cuda")
    for dlogits in (dz.view(2, 5, ld), dz.view(2, 5, ld)[:, :, :V]):
        dz.fill_(9.0)
        B.token_logprobs_backward(prm, z.view(2, 5, ld), y, None, stats, a, None, dlogits)
        assert torch.equal(dz[:, :V], grad)
    for wrong in (seqs[:, :-1], seqs[:, 1:], seqs.view(12, ld)[:9], seqs.view(12, ld)[:9, :V], seqs.view(-1)[:9 * ld]):
        for args in ((wrong, dz), (z, wrong)):
            with pytest.raises(B.DppoError) as e:
                B.token_logprobs_backward(prm, args[0], y, None, stats, a, None, args[1])
            assert e.value.code == B.ERR_BAD_SHAPE
        with pytest.raises(B.DppoError):
            call(wrong)
    torch.cuda.synchronize()
    assert bool((seqs == 9.0).all())


def hidden_case(V, H, T, seed):
    from paper_2603_04135_b200.step import quantize_rows_i8
    g = torch.Generator(device="cuda").manual_seed(seed)
    hidden = torch.empty(T, H, device="cuda").normal_(0, 1, generator=g).to(torch.bfloat16)
    W_q, W_scale = quantize_rows_i8(torch.empty(V, H, device="cuda").normal_(0, 0.1, generator=g))
    return hidden, W_q, W_scale, torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=g)


def test_hidden_states_scored_on_two_streams_at_once(B):
    """Two frozen policies side by side, each on its own stream, give what they give alone."""
    V, H, T = 20003, 256, 700
    st = make_step(V, T)
    cases = [hidden_case(V, H, T, s) for s in (1, 2)]
    alone = {n: [st.score_hidden_i8(*c, top_k=4, chunk_tokens=n) for c in cases] for n in (300, 128)}    # each sums in its own order
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[{n: torch.zeros_like(v) for n, v in alone[300][0].items()} for _ in range(6)] for _ in cases]
    torch.cuda.synchronize()
    for i in range(6):
        for s, c, o in zip(streams, cases, outs):
            with torch.cuda.stream(s):
                st.score_hidden_i8(*c, top_k=4, chunk_tokens=300 if i % 3 else 128, out=o[i])
    torch.cuda.synchronize()
    assert st.status.item() == 0
    for j, os in enumerate(outs):
        for i, o in enumerate(os):
            for n, v in alone[300 if i % 3 else 128][j].items():
                assert torch.equal(o[n], v), (i, j, n)


def test_hidden_states_scored_in_two_graphs(B):
    """Two captured calls replayed on two streams at once, with eager calls of other sizes in between."""
    V, H, T = 8003, 256, 300
    st = make_step(V, T)
    cases = [hidden_case(V, H, T, s) for s in (3, 4)]
    want = [st.score_hidden_i8(*c, top_k=4) for c in cases]
    outs = [{n: torch.zeros_like(v) for n, v in w.items()} for w in want]
    torch.cuda.synchronize()
    graphs = []
    for c, o in zip(cases, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            st.score_hidden_i8(*c, top_k=4, out=o)
    streams = [torch.cuda.Stream() for _ in graphs]
    for i in range(4):
        for o in outs:
            for v in o.values():
                v.zero_()
        st.score_hidden_i8(*cases[0], top_k=2, chunk_tokens=64 + 32 * i)
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
                g.replay()
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            for n in w:
                assert torch.equal(o[n], w[n]), n
    assert st.status.item() == 0


@pytest.mark.parametrize("n", [-3, 0, 1, 40, 1000])
def test_hidden_states_of_any_token_count(B, n):
    """A count on the device beyond the rows, none or below none, in one chunk and in several, as i32 [1], i32 [] and i64 [1]."""
    V, H, T = 1003, 128, 41
    st = make_step(V, T)
    c = hidden_case(V, H, T, 5)
    full = st.score_hidden_i8(*c, top_k=3)
    m = min(max(n, 0), T)
    for chunk in (2048, 41, 16):
        for count in (torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor(n, dtype=torch.int32, device="cuda"),
                      torch.tensor([n], device="cuda")):
            got = st.score_hidden_i8(*c, top_k=3, n_tokens_dev=count, chunk_tokens=chunk)
            for name, v in got.items():
                assert torch.equal(v[:m], full[name][:m]), name
                assert bool((v[m:] == (-1 if name == "top_ids" else 0)).all()), name
    assert st.status.item() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_step_gradient_of_padded_rows(B, dtype):
    """score and score_backward on a [T, V] view of rows padded to 16 bytes, an odd vocabulary."""
    T, V = 9, 1003
    st = make_step(V, T, dtype)
    z, y = make(T, V, dtype, 30)
    z[:, V:] = math.nan                                              # the padding is not looked at
    a, b = torch.randn(T, device="cuda"), torch.randn(T, device="cuda")
    zh, yh = z[:, :V].double().cpu().numpy(), y.cpu().numpy()
    ah, bh = a.double().cpu().numpy(), b.double().cpu().numpy()
    want = scoring.token_logprobs_backward(zh, yh, ah, bh, 0.9)
    for logits in (z[:, :V], z):
        scored = st.score(logits, y, top_k=2, row_stride=z.shape[1])
        d = st.score_backward(logits, y, scored, dlogp=a, dentropy=b, row_stride=z.shape[1])
        assert d.shape == logits.shape and d.stride() == logits.stride() and bool((d[:, V:] == 0).all())
        check_grad(d[:, :V].double().cpu().numpy(), want, zh, yh, ah, bh, 0.9, dtype, V)
    assert st.status.item() == 0


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("N", [1, 31, 33, 97, 129, 255, 257, 383])
def test_linear_i8_last_channels(B, N, variant):
    """Some lanes of a warp have no channel, or a block of tokens is the last: the others' sums are read all the same, in
    contractions of one CTA, of a cluster and of a pair, call after call."""
    for M, K in ((1, 130), (15, 1024), (47, 4096), (130, 515), (300, 640)):
        x, w = codes(M, K, (K + 15) // 16 * 16, M), codes(N, K, (K + 15) // 16 * 16, N)
        xs, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
        out = torch.full((M + 1, N + 5), 5.0, device="cuda")
        prm = B.LinearI8Params(M, N, K, x.shape[1], w.shape[1], N + 5, B.F32, variant)
        want = torch.from_numpy(f32_product(x[:, :K], xs, w[:, :K], ws))
        for _ in range(3):
            out[:M, :N] = 0
            B.linear_i8(prm, x, xs, w, ws, out)
            assert torch.equal(out[:M, :N].cpu(), want)
        assert bool((out[M:] == 5.0).all()) and bool((out[:, N:] == 5.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V, variant", [(1021, 0), (1021, 32), (8203, 32), (20003, 0), (20003, 10512), (50304, 20256), (151936, 0), (151937, 10128),
                                        (151937, 40256), (151937, 80512)])
def test_every_entry_counts_once(B, V, variant, dtype):
    """Rows of n entries at 0 and nothing else that counts (-inf, the type's lowest value, -5,000): 2^0 = 1 is exact, so are
    sums of up to 2^24 ones, and 2^-5000 is 0.  What is left is logf's error of one step, 2 U l for l = ln n, where one entry
    lost or counted twice moves l by 1 / n > 6e-6.  The gradient's exponent has l's error (2 U l) and three roundings
    (log2(e), product, fma: 3 U l), the exponential 4 U, the product with a and the sum at the token one each."""
    lowest = float(torch.finfo(DT[dtype]).min)
    g = torch.Generator().manual_seed(V)
    live = [torch.ones(V, dtype=torch.bool), torch.rand(V, generator=g) < 0.5, torch.arange(V) < V - 1, torch.arange(V) > 0,
            torch.arange(V) % 977 == 5, torch.arange(V) == V - 1, torch.rand(V, generator=g) < 0.9]
    T = len(live)
    z = torch.zeros(T, pad16(V, 2 if dtype == "bf16" else 4))
    for t, on in enumerate(live):
        other = torch.tensor([-math.inf, lowest, -5000.0])[torch.randint(0, 3, (V,), generator=g)]
        z[t, :V] = torch.where(on, torch.tensor(0.0), other)
    n = torch.stack([on.sum() for on in live]).double().numpy()
    y = torch.tensor([int(torch.nonzero(on)[-1]) for on in live], dtype=torch.int32, device="cuda")
    z = z.to(DT[dtype]).cuda()
    f = Fwd(B, z, V, y, 3, 1.0, variant)
    o, l = f.host(), np.log(n)
    for got, want in ((o["lse"], l), (o["entropy"], l), (o["logp"], -l), (o["top_logp"][:, 0], -l)):
        assert (np.abs(got - want) <= 2 * U * l).all(), (got - want, l)
    first = [torch.nonzero(on)[:3, 0].tolist() for on in live]
    assert [[i for i, p in zip(ids, lp) if p > -100] for ids, lp in zip(o["top_ids"].tolist(), o["top_logp"].tolist())] == first
    a = torch.randn(T, device="cuda")
    dz = torch.full_like(z, 9.0)
    B.token_logprobs_backward(B.LogprobParams(T, V, B.BF16 if dtype == "bf16" else B.F32, z.stride(0), 0, 0, 1.0), z, y, None, f.stats, a, None, dz)
    ah, got = a.double().cpu().numpy(), dz[:, :V].double().cpu().numpy()
    half = 2.0 ** -8 if dtype == "bf16" else 0.0                           # f32: the product's rounding is the output's
    for t, on in enumerate(live):
        p = on.double().numpy() / n[t]
        want = -ah[t] * p
        tol = np.abs(want) * (5 * l[t] + 6) * U
        want[int(y[t])] += ah[t]
        tol[int(y[t])] += 2 * U * abs(ah[t])
        assert (np.abs(got[t] - want) <= tol * (1 + half) + half * np.abs(want)).all(), t
