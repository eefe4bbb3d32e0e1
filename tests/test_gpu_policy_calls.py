"""Calls around a second policy as a program makes them: on two streams at once, in two captured graphs, with no drafts and with very many, with
outputs and row counts of every alignment.  Results are compared bit for bit with the same call made alone, or with the oracle."""
import numpy as np
import pytest
import torch

from oracle import f8, verify

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def B():
    from paper_2603_04135_b200 import binding
    return binding


class Calls:
    """One of each call on inputs of its own."""

    def __init__(self, B, seed, V=20003, T=37, K=700, M=150):
        g = torch.Generator(device="cuda").manual_seed(seed)
        ld = (V + 7) // 8 * 8
        self.B, self.V, self.T, self.K, self.M, self.ld = B, V, T, K, M, ld
        self.z = torch.empty(2 * T, ld, device="cuda").normal_(0, 2, generator=g).bfloat16()
        self.ids = torch.randint(0, V, (T, 9), device="cuda", generator=g, dtype=torch.int32)
        self.lp = torch.full((T, 9), -3.0, device="cuda")
        self.w = torch.rand(T, device="cuda", generator=g)
        self.drafts = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
        self.cu = torch.tensor([0, 5, 5, 20, T], dtype=torch.int32, device="cuda")
        self.u, self.noise = torch.rand(T, device="cuda", generator=g), torch.empty(4, ld, device="cuda").exponential_(generator=g)
        self.x = torch.empty(M, K + 4, device="cuda").normal_(0, 1, generator=g)
        self.wq = torch.empty(V, 768, device="cuda").normal_(0, 100, generator=g).clamp_(-448, 448).to(F8)
        self.ws = torch.rand((V + 127) // 128, 6, device="cuda", generator=g)

    def outputs(self):
        z = lambda *n, dtype=torch.float32: torch.zeros(*n, dtype=dtype, device="cuda")
        return dict(loss=z(self.T), stats=z(self.T, 4), dz=torch.zeros_like(self.z[:self.T]), dz2=torch.zeros_like(self.z[:self.T]), n=z(4, dtype=torch.int32),
                    tok=z(self.T + 4, dtype=torch.int32), logp=z(self.T + 4), ws=z(8 * (2 * self.T + 4), dtype=torch.uint8),
                    q=torch.zeros(self.M, 768, dtype=F8, device="cuda"), qs=z(6, (self.M + 3) // 4 * 4), y=z(self.M, self.V), y1=z(9, self.V, dtype=torch.bfloat16),
                    status=z(1, dtype=torch.int32))

    def run(self, o, stream=None):
        B, T, V, ld = self.B, self.T, self.V, self.ld
        d = B.DistillParams(T, V, B.BF16, ld, 9, B.DISTILL_REST, 1.0)
        B.distill_topk(d, self.z, self.ids, self.lp, None, self.w, o["loss"], None, o["stats"], o["dz"], o["status"], stream=stream)
        B.distill_topk_backward(d, self.z, self.ids, self.lp, None, o["stats"], self.w, o["dz2"], o["status"], stream=stream)
        p = B.VerifyParams(T, 4, V, B.BF16, ld, ld, ld, 1.0, 1.0)
        B.verify_drafts(p, self.z, self.z[4:], self.drafts, self.cu, self.u, self.noise, o["n"], o["tok"], o["logp"], o["ws"], o["ws"].numel(), o["status"],
                        stream=stream)
        B.quantize_f8(B.QuantizeF8Params(self.M, self.K, B.F32, self.x.stride(0), 768, o["qs"].stride(0), 1), self.x, o["q"], o["qs"], None, o["status"], stream=stream)
        for out, M, dt in ((o["y"], self.M, B.F32), (o["y1"], 9, B.BF16)):
            B.linear_f8(B.LinearF8Params(M, V, self.K, 768, 768, V, o["qs"].stride(0), 6, dt), o["q"], o["qs"], self.wq, self.ws, out, None, o["status"], stream=stream)


def same(a, b):
    for k in a:
        if k != "ws":
            assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), k


def test_two_streams_at_once(B):
    one, two = Calls(B, 1), Calls(B, 2, V=5001, T=61, K=768, M=300)
    want = []
    for c in (one, two):
        want.append(c.outputs())
        c.run(want[-1])
    torch.cuda.synchronize()
    streams, got = (torch.cuda.Stream(), torch.cuda.Stream()), (one.outputs(), two.outputs())
    torch.cuda.synchronize()
    for _ in range(20):
        for c, o, s in zip((one, two), got, streams):
            c.run(o, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        same(a, b)
        assert int(b["status"].item()) == 0


def test_two_graphs_at_once(B):
    """Captured calls keep nothing between them: two graphs of the same inputs replay side by side."""
    c = Calls(B, 3)
    want = c.outputs()
    c.run(want)
    torch.cuda.synchronize()
    got, graphs, streams = [c.outputs(), c.outputs()], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for o in got:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run(o)
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o in got:
        same(want, o)


def test_sequences_without_drafts(B):
    n, V = 5, 1003
    g = torch.Generator(device="cuda").manual_seed(4)
    z, noise = torch.empty(n, 1004, device="cuda").normal_(0, 2, generator=g), torch.empty(n, 1004, device="cuda").exponential_(generator=g)
    prm = B.VerifyParams(0, n, V, B.F32, 1004, 0, 1004, 0.7, 1.0)
    need = B.verify_drafts_workspace_bytes(prm)
    acc, tok, logp = (torch.full((n,), -7, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32))
    empty_i, empty_f = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    B.verify_drafts(prm, z, None, empty_i, torch.zeros(n + 1, dtype=torch.int32, device="cuda"), empty_f, noise, acc, tok, logp,
                    torch.empty(need, dtype=torch.uint8, device="cuda"), need)
    h = lambda t: t.cpu().numpy()
    want = verify.verify_drafts(h(z)[:, :V].astype(np.float64), None, h(empty_i), np.zeros(n + 1, dtype=np.int64), h(empty_f), h(noise)[:, :V].astype(np.float64), 0.7, 1.0)
    assert (want["margin"] > 1e-12).all() and np.array_equal(h(tok), want["tokens"]) and (h(acc) == 0).all()
    assert np.abs(h(logp) - want["logp"]).max() < 1e-5


def test_one_sequence_of_very_many_drafts(B):
    """Accepted to the end, and up to a place far beyond the first 32."""
    T, V = 5000, 40
    g = torch.Generator(device="cuda").manual_seed(5)
    z = torch.empty(T + 1, V, device="cuda").normal_(0, 1, generator=g)
    y = z[:T].argmax(1).int()
    noise, u = torch.empty(1, V, device="cuda").exponential_(generator=g), torch.zeros(T, device="cuda")
    prm = B.VerifyParams(T, 1, V, B.F32, V, 0, V, 1.0, 1.0)
    need = B.verify_drafts_workspace_bytes(prm)
    ws, cu = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda")
    for stop in (T, 4321, 31, 32):
        if stop < T:
            u[stop] = 1.0                                            # never below a probability
        acc, tok, logp = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((T + 1,), -7, dtype=torch.int32, device="cuda"), torch.zeros(T + 1, device="cuda")
        B.verify_drafts(prm, z, None, y, cu, u, noise, acc, tok, logp, ws, need)
        first = min([stop] + [s for s in (4321, 31) if float(u[min(s, T - 1)]) == 1.0])
        assert int(acc.item()) == first and torch.equal(tok[:first], y[:first])
        p = torch.softmax(z[first].double(), 0)
        if first < T:
            p[y[first].long()] = 0.0
        assert int(tok[first].item()) == int((p / noise[0].double()).argmax()) and bool((tok[first + 1:] == -1).all())
        lp = torch.log_softmax(z.double(), 1)
        at = torch.arange(first, device="cuda")
        assert (logp[:first].double() - lp[at, y[:first].long()]).abs().max() < 1e-5 if first else True
        assert bool((logp[first + 1:] == 0).all())


@pytest.mark.parametrize("M,K", [(3000, 2563), (20011, 515), (700, 4096), (2500, 640)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_many_rows(B, M, K, dtype):
    """Rows in numbers, four blocks at a time: bit for bit, with the true count on the device."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.empty(M, (K + 7) // 8 * 8, device="cuda").normal_(0, 1, generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[5, 3], x[6, K - 1] = float("nan"), float("inf")
    kb, ld = (K + 127) // 128, (K + 15) // 16 * 16
    q, s = torch.full((M, ld), 0x55, dtype=torch.uint8, device="cuda"), torch.full((kb, M + 5), -7.5, device="cuda")
    n = torch.tensor([M - 3], dtype=torch.int32, device="cuda")
    B.quantize_f8(B.QuantizeF8Params(M, K, B.BF16 if dtype == "bf16" else B.F32, x.stride(0), ld, s.stride(0), 1), x, q.view(F8), s, n)
    rows = np.concatenate([np.arange(40), np.arange(M // 2, M // 2 + 40), np.arange(M - 43, M - 3)])
    want_q, want_s = f8.quantize(x.float().cpu().numpy()[rows][:, :K], 1)
    at = torch.from_numpy(rows).cuda()
    np.testing.assert_array_equal(q[at, :K].cpu().numpy(), want_q)
    np.testing.assert_array_equal(s[:, at].cpu().numpy(), want_s)
    assert bool((q[M - 3:] == 0x55).all()) and bool((q[:, K:] == 0x55).all()) and bool((s[:, M - 3:] == -7.5).all())


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("M,N,shift,pitch", [(300, 1024, 1, 0), (257, 1000, 0, 3), (512, 513, 4, 7), (130, 2056, 8, 8), (256, 300, 0, 4)])
def test_outputs_of_any_alignment(B, out, variant, M, N, shift, pitch):
    """The same numbers wherever they are written, and nothing beside them."""
    K, g = 640, torch.Generator(device="cuda").manual_seed(N)
    dt = torch.bfloat16 if out == "bf16" else torch.float32
    x, w = (torch.empty(n, K, device="cuda").normal_(0, 100, generator=g).clamp_(-448, 448).to(F8) for n in (M, N))
    xs, ws = torch.rand(5, (M + 3) // 4 * 4, device="cuda", generator=g), torch.rand((N + 127) // 128, 5, device="cuda", generator=g)
    plain = torch.zeros(M, (N + 255) // 256 * 256, dtype=dt, device="cuda")
    call = lambda y, ld: B.linear_f8(B.LinearF8Params(M, N, K, K, K, ld, xs.shape[1], 5, B.BF16 if out == "bf16" else B.F32, variant), x, xs, w, ws, y)
    call(plain, plain.stride(0))
    flat = torch.full((shift + M * (N + pitch) + 64,), -7.5, dtype=dt, device="cuda")
    y = flat[shift:shift + M * (N + pitch)].view(M, N + pitch)
    call(y, N + pitch)
    assert torch.equal(y[:, :N], plain[:, :N]) and bool((plain[:, N:] == 0).all())
    y[:, :N] = -7.5
    assert bool((flat == -7.5).all())
