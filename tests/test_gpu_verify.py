"""Verification of drafted tokens on the GPU against the float64 oracle.

Tokens and counts have to be the oracle's wherever its decisions have a margin: u q < p and the race compare f64 values that rest on
sums S with a relative error of at most eS = (3 E|x| + 3 + 6 n + 16) 2^-24 (n terms per thread, E|x| the mean exponent), so a
decision whose two sides are further apart than 1e-4 of each other, or 1e-4 / kappa where p - q cancels, cannot turn; the oracle's
margin tells, and sequences below it are counted: there are hardly any.  Log-probs carry eS, the f64 difference and the f32 result.
"""
import math

import numpy as np
import pytest
import torch

from oracle import verify as oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


def pad(n, per):
    return (n + per - 1) // per * per


class Case:
    def __init__(self, lens, V, dtype, copied, tau, dtau, seed, mask="none", spare=3, spread=0.6):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.V, self.dtype, self.tau, self.dtau, self.nB = V, dtype, tau, dtau, len(lens)
        per = 8 if dtype == "bf16" else 4
        self.T = sum(lens)
        self.T_max = self.T + spare                                  # rows behind the last sequence
        cu = np.concatenate([[0], np.cumsum(lens)])
        self.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        rows = self.T_max + self.nB
        z = torch.empty(rows, pad(V, per) + 8, device="cuda").normal_(0.0, 2.0, generator=g)
        seq = torch.tensor(np.repeat(np.arange(self.nB), lens), device="cuda")
        trow = torch.arange(self.T, device="cuda") + seq
        d = torch.full((self.T_max, z.shape[1]), math.nan, device="cuda")
        d[:self.T] = z[trow] + spread * torch.empty(self.T, z.shape[1], device="cuda").normal_(0.0, 1.0, generator=g)
        if mask == "sparse":
            z.masked_fill_(torch.rand(z.shape, device="cuda", generator=g) < 0.8, -math.inf)
        z[self.T + self.nB:] = math.nan
        self.target, self.draft = z.to(DT[dtype]), d.to(DT[dtype])
        q = torch.softmax(self.draft[:self.T, :V].double() / dtau, 1)
        e = torch.empty(q.shape, device="cuda", dtype=torch.float64).exponential_(generator=g)
        self.drafts = torch.full((self.T_max,), -9, dtype=torch.int32, device="cuda")
        self.drafts[:self.T] = (self.target[trow, :V].float().argmax(1) if copied else (q / e).argmax(1)).int()
        if copied:
            self.draft = None
        self.u = torch.rand(self.T_max, device="cuda", generator=g)
        self.noise = torch.empty(self.nB, pad(V, 4) + 4, device="cuda").exponential_(generator=g)

    def run(self, B, stream=None, out=None):
        prm = B.VerifyParams(self.T_max, self.nB, self.V, B.BF16 if self.dtype == "bf16" else B.F32, self.target.stride(0),
                             self.draft.stride(0) if self.draft is not None else 0, self.noise.stride(0), self.tau, self.dtau)
        n = B.verify_drafts_workspace_bytes(prm)
        if out is None:
            out = dict(n=torch.full((self.nB + 4,), -77, dtype=torch.int32, device="cuda"), tokens=torch.full((self.T_max + self.nB + 4,), -77, dtype=torch.int32, device="cuda"),
                       logp=torch.full((self.T_max + self.nB + 4,), -7.5, device="cuda"), status=torch.zeros(1, dtype=torch.int32, device="cuda"),
                       ws=torch.full((n,), 0xff, dtype=torch.uint8, device="cuda"))
        B.verify_drafts(prm, self.target, self.draft, self.drafts, self.cu, self.u, self.noise, out["n"], out["tokens"], out["logp"], out["ws"], n,
                        status=out["status"], stream=stream)
        return out

    def want(self):
        V = self.V
        return oracle.verify_drafts(self.target[:self.T + self.nB, :V].double().cpu().numpy(),
                                    None if self.draft is None else self.draft[:self.T, :V].double().cpu().numpy(), self.drafts[:self.T].cpu().numpy(),
                                    self.cu.cpu().numpy().astype(np.int64), self.u.double().cpu().numpy(), self.noise[:, :V].double().cpu().numpy(),
                                    self.tau, self.dtau)

    def check(self, out, status=0, all_close=False):
        torch.cuda.synchronize()
        w = self.want()
        got = {k: v.cpu().numpy() for k, v in out.items()}
        assert int(got["status"][0]) == status
        n = self.T + self.nB
        assert (got["n"][self.nB:] == -77).all() and (got["tokens"][n:] == -77).all() and (got["logp"][n:] == -7.5).all()
        z = self.target[:n, :self.V].double().cpu().numpy()
        cu = self.cu.cpu().numpy()
        close = 0
        for b in range(self.nB):
            lo, hi = cu[b] + b, cu[b + 1] + b + 1
            if w["margin"][b] < 1e-4:
                close += 1
                continue
            assert got["n"][b] == w["n_accepted"][b], (b, got["n"][b], w["n_accepted"][b], w["margin"][b])
            assert list(got["tokens"][lo:hi]) == list(w["tokens"][lo:hi]), b
            for t in range(lo, hi):
                a, x = got["logp"][t], w["logp"][t]
                if not math.isfinite(x):
                    np.testing.assert_array_equal(a, x)
                    continue
                row = z[t][z[t] > -np.inf]
                d = (row - row.max()) / self.tau if row.size else np.zeros(1)
                e = np.exp(d)
                eS = (3 * (e * np.abs(d)).sum() / e.sum() + 3 + 6 * math.ceil(self.V / (32 if self.V <= 2055 else 128)) + 16) * U
                assert abs(a - x) <= (eS + U * abs(x) if got["tokens"][t] >= 0 else 0), (t, a, x)
        assert close == self.nB if all_close else close <= max(1, self.nB // 50)
        return got, w


CASES = [
    # drafts per sequence, V, dtype, copied, tau, draft tau, mask
    ([4], 151936, "bf16", False, 1.0, 1.0, "none"), ([0], 7, "f32", False, 1.0, 1.0, "none"), ([0, 0, 3], 1, "f32", False, 1.0, 1.0, "none"),
    ([5, 0, 1, 7, 33, 2], 250, "bf16", False, 0.7, 1.0, "none"), ([31, 32, 33, 64, 65], 1021, "f32", False, 1.0, 0.8, "none"),
    ([3, 1, 8, 2] * 20, 2049, "bf16", False, 1.0, 1.0, "sparse"), ([6] * 30, 5003, "f32", True, 0.5, 1.0, "none"),
    ([100, 40], 777, "bf16", True, 0.25, 1.0, "none"), ([2, 9], 50304, "f32", False, 1.3, 1.3, "none"), ([1], 33001, "bf16", False, 1.0, 2.0, "sparse"),
    ([3] * 400, 300, "f32", False, 1.0, 1.0, "none"), ([7, 3] * 8, 32003, "bf16", True, 0.4, 1.0, "sparse"),
]


@pytest.mark.parametrize("lens,V,dtype,copied,tau,dtau,mask", CASES)
def test_against_oracle(B, lens, V, dtype, copied, tau, dtau, mask):
    c = Case(lens, V, dtype, copied, tau, dtau, V + len(lens), mask)
    c.check(c.run(B))


def test_all_accepted_and_all_rejected(B):
    c = Case([9, 40], 3001, "f32", False, 1.0, 1.0, 3, spread=0.0)
    got, _ = c.check(c.run(B))                                       # the same policies: everything is accepted
    assert list(got["n"][:2]) == [9, 40]
    c.u.fill_(1.0 - 2.0 ** -24)                                      # p = q, bit for bit: (p - u q) / p = 2^-24 for every draft
    got, _ = c.check(c.run(B), all_close=True)
    assert list(got["n"][:2]) == [9, 40]
    c.draft[:c.T] = -math.inf                                        # q = 0: accepted wherever p > 0
    got, _ = c.check(c.run(B))
    assert list(got["n"][:2]) == [9, 40]
    c.draft[:c.T, :] = 0.0
    c.target[:c.T + 2, :c.V] = -math.inf
    c.target[:c.T + 2, 5] = 1.0                                      # one token is allowed, and no draft is that one
    c.drafts[:c.T] = 6
    got, _ = c.check(c.run(B))
    assert list(got["n"][:2]) == [0, 0] and got["tokens"][0] == 5


@pytest.mark.parametrize("V", [300, 70001])
def test_rows_where_it_can_go_wrong(B, V):
    lens = [4] * 8
    c = Case(lens, V, "f32", False, 1.0, 1.0, 9, spread=0.0)         # without what follows everything is accepted
    rows = [b * 5 for b in range(8)]
    c.target[rows[0] + 1, 7] = math.nan
    c.target[rows[1] + 2, V - 1] = math.inf
    c.target[rows[2], :V] = -math.inf
    c.draft[3 * 4 + 2, 0] = math.nan
    c.target[rows[4] + 4, :V] = -math.inf                            # the row after the last draft
    low = torch.finfo(torch.float32).min
    c.target[rows[5] + 1, :V] = low                                  # all masked by the lowest value: uniform
    c.target[rows[6] + 1, c.drafts[6 * 4 + 1].long()] = -math.inf    # the drafted token is not allowed
    c.draft[7 * 4 + 1, :V] = -math.inf
    got, w = c.check(c.run(B))
    assert list(got["n"][:5]) == [1, 2, 0, 2, 4] and got["n"][6] == 1 and got["n"][7] == 4


def test_residual_that_is_empty(B):
    """p <= q everywhere where p has mass (the target is masked to one token that the draft is sure of) and u close to 1."""
    c = Case([1], 64, "f32", True, 1.0, 1.0, 2)
    c.target[0, :64] = -math.inf
    c.target[0, 9] = 3.0
    c.drafts[0] = 9
    c.u.fill_(1.0)                                                   # not below p = 1: a rejection with nothing left over
    got, _ = c.check(c.run(B))
    assert got["n"][0] == 0 and got["tokens"][0] == 9 and got["logp"][0] == 0.0


@pytest.mark.parametrize("V,dtype", [(1000, "f32"), (40000, "bf16")])
def test_ties_go_to_the_lower_index(B, V, dtype):
    c = Case([0, 2], V, dtype, False, 1.0, 1.0, 4)
    c.target[:, :V] = 0.0
    c.noise.fill_(0.5)
    got, _ = c.run(B), None
    torch.cuda.synchronize()
    assert int(got["tokens"][0]) == 0                                # all alike: the first
    c.noise[0, 11:V] = 0.25
    got = c.run(B)
    torch.cuda.synchronize()
    assert int(got["tokens"][0]) == 11
    # f32 rounds both to the same value, 64 bits tell them apart
    c.noise[0, 11:V] = 0.5
    c.noise[0, 20] = float(np.nextafter(np.float32(0.5), np.float32(0)))
    c.noise[0, V - 1] = float(np.nextafter(np.nextafter(np.float32(0.5), np.float32(0)), np.float32(0)))
    got = c.run(B)
    torch.cuda.synchronize()
    assert int(got["tokens"][0]) == V - 1


def test_bad_ids_and_segments(B):
    c = Case([3, 3, 3], 500, "f32", False, 1.0, 1.0, 6, spread=0.0)
    good, _ = c.check(c.run(B))
    c.drafts[4] = 500
    out = c.run(B)
    torch.cuda.synchronize()
    assert int(out["status"]) == B.STATUS_BAD_TARGET
    assert out["n"][:3].tolist() == [3, 1, 3] and 0 <= int(out["tokens"][5]) < 500
    assert out["tokens"][8:12].tolist() == good["tokens"][8:12].tolist()
    c.drafts[4] = 1
    for cu in ([0, 5, 3, 9], [0, 3, 6, 13], [0, -2, 6, 9], [-1, 3, 6, 9]):
        c.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        out = c.run(B)
        torch.cuda.synchronize()
        assert int(out["status"]) == B.STATUS_BAD_SEGMENTS
    c.cu = torch.tensor([0, 0, 0, 0], dtype=torch.int32, device="cuda")
    out = c.run(B)
    torch.cuda.synchronize()
    assert int(out["status"]) == 0 and out["n"][:3].tolist() == [0, 0, 0] and bool((out["tokens"][3:] == -77).all())


def test_offsets_beyond_32_bits(B):
    c = Case([2], 900, "bf16", False, 1.0, 1.0, 5, spare=0)
    want = c.run(B)
    ld = (1 << 30) + 8
    for name, rows in (("target", 3), ("draft", 2)):
        x = torch.empty((rows - 1) * ld + 1024, dtype=torch.bfloat16, device="cuda").as_strided((rows, 900), (ld, 1))
        x.copy_(getattr(c, name)[:, :900])
        setattr(c, name, x)
    out = c.run(B)
    torch.cuda.synchronize()
    for k in ("n", "tokens", "logp"):
        assert torch.equal(out[k], want[k])


def test_captured_and_on_another_stream(B):
    c, d = (Case([4, 6, 2], 20000, "bf16", False, 1.0, 1.0, s) for s in (1, 2))
    out = c.run(B)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(B, out=out)
    for n in ("target", "draft", "drafts", "u", "noise"):
        getattr(c, n).copy_(getattr(d, n))
    out["tokens"].fill_(-77)
    graph.replay()
    c.check(out)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    o2 = c.run(B, stream=side)
    c.check(o2)
