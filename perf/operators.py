"""Cases of the scoring operators: log-probs of given tokens (with entropy and top alternatives), their gradient with
respect to the logits, and the 8-bit matrix product of a frozen policy's LM-head.

`own` chooses between the plain torch form of each operator and the library's calls.
"""
import math

import torch

own = False

_BYTES = {"bf16": 2, "f32": 4}
_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------
def listed():
    return [
        # one decoded token over the Qwen3 vocabulary, 20 alternatives: latency counts
        dict(name="logprobs_1_token", op="logprobs", T=1, V=151936, dtype="bf16", k=20, tau=1.0, mask="padding"),
        # a decode batch
        dict(name="logprobs_48_tokens", op="logprobs", T=48, V=151936, dtype="bf16", k=8, tau=1.0, mask="none"),
        # a scoring pass over packed completions
        dict(name="logprobs_8192_tokens", op="logprobs", T=8192, V=151936, dtype="bf16", k=4, tau=1.0, mask="padding"),
        # short ragged rows in f32 with a constrained vocabulary
        dict(name="logprobs_short_rows", op="logprobs", T=20011, V=1021, dtype="f32", k=5, tau=0.7, mask="sparse"),
        # gradient for a small micro-batch
        dict(name="backward_64_tokens", op="backward", T=64, V=151936, dtype="bf16", tau=1.0, mask="none"),
        # gradient for a packed batch
        dict(name="backward_8192_tokens", op="backward", T=8192, V=151936, dtype="bf16", tau=1.0, mask="padding"),
        # short ragged rows
        dict(name="backward_short_rows", op="backward", T=20011, V=1021, dtype="f32", tau=0.7, mask="sparse"),
        # f32 rows of a mid-sized vocabulary
        dict(name="backward_f32", op="backward", T=2003, V=50304, dtype="f32", tau=1.0, mask="none"),
        # LM-head of one decoded token: the weights are read once
        dict(name="linear_1_token", op="linear", M=1, K=2560, N=151936, dtype="bf16", out="f32"),
        # a square projection for a decode batch
        dict(name="linear_64_tokens", op="linear", M=64, K=4096, N=4096, dtype="bf16", out="bf16"),
        # LM-head of a scoring chunk: tensor-core bound
        dict(name="linear_2048_tokens", op="linear", M=2048, K=2560, N=151936, dtype="bf16", out="bf16"),
        # nothing divides anything
        dict(name="linear_ragged", op="linear", M=1003, K=2563, N=5003, dtype="f32", out="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "backward", "linear"])
    if op == "linear":
        M, K, N = _log_int(rng, 1, 4096), _log_int(rng, 48, 8192), _log_int(rng, 48, 151936)
        M = max(1, min(M, 2048 * 2560 * 151936 // (K * N), 2048 * 151936 // N))
        return dict(op=op, M=M, K=K, N=N, dtype=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    dtype = rng.choice(["bf16", "f32"])
    V = _log_int(rng, 250, 151936)
    T = min(_log_int(rng, 1, 30000), 8192 * 151936 * 2 // (V * _BYTES[dtype]))
    case = dict(op=op, T=T, V=V, dtype=dtype, tau=round(rng.uniform(0.5, 1.5), 3), mask=rng.choice(["none", "padding", "sparse"]))
    if op == "logprobs":
        case["k"] = rng.randint(0, 20)
    return case


# ---- inputs ---------------------------------------------------------------------------------------
def _logits(case, gen):
    """Logits N(0, 2) in rows padded to 16 bytes, and a sampled token for each row.  `padding`: the last entries of the
    vocabulary are no tokens (-inf); `sparse`: nine of ten entries are not allowed."""
    T, V, dt = case["T"], case["V"], _TORCH[case["dtype"]]
    per = 16 // _BYTES[case["dtype"]]
    stride = (V + per - 1) // per * per
    z = torch.empty(T, stride, dtype=dt, device="cuda").normal_(0.0, 2.0, generator=gen)
    target = torch.randint(0, max(1, V - V // 500), (T,), device="cuda", generator=gen, dtype=torch.int32)
    if case["mask"] == "padding":
        z[:, V - V // 500:] = -math.inf
    elif case["mask"] == "sparse":
        z.masked_fill_(torch.rand(z.shape, device="cuda", generator=gen) < 0.9, -math.inf)
    rows = torch.arange(T, device="cuda")
    z[rows, target.long()] = torch.empty(T, device="cuda").normal_(4.0, 2.0, generator=gen).to(dt)
    return z, target


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    f32 = dict(dtype=torch.float32, device="cuda")
    s = dict(case)
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        per = 16 // _BYTES[case["dtype"]]
        ldx, ldq = (K + per - 1) // per * per, (K + 15) // 16 * 16
        x = torch.empty(M, ldx, **f32).normal_(0.0, 1.0, generator=gen)
        x *= torch.exp(torch.empty(ldx, **f32).normal_(0.0, 0.5, generator=gen))       # channels of different size
        w = torch.randint(-127, 128, (N, ldq), device="cuda", generator=gen, dtype=torch.int8)
        s.update(x=x.to(_TORCH[case["dtype"]]), w=w,
                 w_scale=torch.empty(N, **f32).uniform_(0.5, 1.5, generator=gen) / (127.0 * math.sqrt(K)),
                 q=torch.zeros(M, ldq, dtype=torch.int8, device="cuda"), q_scale=torch.zeros(M, **f32),
                 y=torch.zeros(M, N, dtype=_TORCH[case["out"]], device="cuda"), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
        return s
    z, target = _logits(case, gen)
    T, V = case["T"], case["V"]
    s.update(logits=z, target=target, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if case["op"] == "logprobs":
        k = case["k"]
        s.update(logp=torch.zeros(T, **f32), entropy=torch.zeros(T, **f32), lse=torch.zeros(T, **f32), stats=torch.zeros(T, 4, **f32),
                 top_ids=torch.zeros(T, k, dtype=torch.int32, device="cuda"), top_logp=torch.zeros(T, k, **f32))
        return s
    # what the forward call leaves for the backward: per row the maximum, the log of the sum relative to it, the entropy
    stats = torch.zeros(T, 4, **f32)
    step = max(1, (1 << 27) // V)
    for a in range(0, T, step):
        x = z[a:a + step, :V].double()
        m = x.amax(1, keepdim=True)
        x = (x - m) / case["tau"]
        e = x.exp()
        tot = e.sum(1)
        stats[a:a + step, 0] = m[:, 0].float()
        stats[a:a + step, 1] = tot.log().float()
        stats[a:a + step, 2] = (tot.log() - (e * x.clamp_min(-1e5)).sum(1) / tot).float()
    s.update(stats=stats, dlogp=torch.empty(T, **f32).normal_(0.0, 1.0, generator=gen),
             dentropy=torch.empty(T, **f32).normal_(0.0, 0.1, generator=gen), dlogits=torch.zeros_like(z))
    return s


# ---- one pass ---------------------------------------------------------------------------------------
def run(s):
    if s["op"] == "linear":
        return _run_linear(s)
    if s["op"] == "logprobs":
        return _run_logprobs(s)
    return _run_backward(s)


def _run_linear(s):
    M, K, N = s["M"], s["K"], s["N"]
    if own:
        from paper_2603_04135_b200 import binding as B
        code = {"f32": B.F32, "bf16": B.BF16}
        B.quantize_rows_i8(B.QuantizeParams(M, K, code[s["dtype"]], s["x"].shape[1], s["q"].shape[1]), s["x"], s["q"], s["q_scale"])
        B.linear_i8(B.LinearI8Params(M, N, K, s["q"].shape[1], s["w"].shape[1], N, code[s["out"]]), s["q"], s["q_scale"], s["w"],
                    s["w_scale"], s["y"], status=s["status"])
        return {"y": s["y"]}
    x = s["x"][:, :K].float()
    scale = x.abs().amax(1, keepdim=True) / 127.0
    q = torch.where(scale > 0, torch.clamp(torch.round(x / scale), -127, 127), torch.zeros_like(x))
    acc = q @ s["w"][:, :K].float().t()
    return {"y": (acc * (scale * s["w_scale"])).to(_TORCH[s["out"]])}


def _run_logprobs(s):
    T, V, k, tau = s["T"], s["V"], s["k"], s["tau"]
    if own:
        from paper_2603_04135_b200 import binding as B
        prm = B.LogprobParams(T, V, B.BF16 if s["dtype"] == "bf16" else B.F32, s["logits"].shape[1], k, 0, tau)
        B.token_logprobs(prm, s["logits"], s["target"], None, s["logp"], s["entropy"], s["lse"], s["top_ids"] if k else None,
                         s["top_logp"] if k else None, s["stats"], status=s["status"])
        return {n: s[n] for n in ("logp", "entropy", "lse", "top_ids", "top_logp")}
    z = s["logits"][:, :V].float()
    m = z.amax(1, keepdim=True)
    x = (z - m) / tau
    e = torch.exp(x)
    total = e.sum(1)
    l = torch.log(total)
    out = {"logp": x.gather(1, s["target"].long()[:, None])[:, 0] - l,
           "entropy": l - (e * x.clamp_min(-1e5)).sum(1) / total, "lse": m[:, 0] / tau + l}
    # alternatives by (value, lower index first): one key for each entry whose order is that
    bits = (z + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7fffffff)).long() * (1 << 32) + (V - 1 - torch.arange(V, device=z.device))
    ids = V - 1 - (torch.topk(key, min(k, V), dim=1).values & 0xffffffff)
    val = z.gather(1, ids)
    gone = val == -math.inf
    out["top_ids"] = torch.where(gone, -1, ids).to(torch.int32)
    out["top_logp"] = torch.where(gone, -math.inf, (val - m) / tau - l[:, None])
    return out


def _run_backward(s):
    T, V, tau = s["T"], s["V"], s["tau"]
    if own:
        from paper_2603_04135_b200 import binding as B
        prm = B.LogprobParams(T, V, B.BF16 if s["dtype"] == "bf16" else B.F32, s["logits"].shape[1], 0, 0, tau)
        B.token_logprobs_backward(prm, s["logits"], s["target"], None, s["stats"], s["dlogp"], s["dentropy"], s["dlogits"], status=s["status"])
        return {"dlogits": s["dlogits"][:, :V]}
    z = s["logits"][:, :V].float()
    x = (z - z.amax(1, keepdim=True)) / tau
    lnp = x - torch.log(torch.exp(x).sum(1, keepdim=True))
    p = torch.exp(lnp)
    lnp = lnp.clamp_min(-1e5)
    H = -(p * lnp).sum(1, keepdim=True)
    g = -p * (s["dlogp"][:, None] + s["dentropy"][:, None] * (lnp + H))
    g.scatter_add_(1, s["target"].long()[:, None], s["dlogp"][:, None])
    return {"dlogits": (g / tau).to(s["logits"].dtype)}


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K * _BYTES[case["dtype"]] + N * K + 4 * N + M * N * _BYTES[case["out"]], "flops": 2 * M * N * K}
    T, V, b = case["T"], case["V"], _BYTES[case["dtype"]]
    if case["op"] == "logprobs":
        return {"bytes": T * (V * b + 4 + 28 + 8 * case["k"]), "flops": 6 * T * V}
    return {"bytes": T * (2 * V * b + 28), "flops": 7 * T * V}


# ---- the definition in 64 bits -----------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        K = case["K"]
        w = s["w"][:, :K].double()
        ws = s["w_scale"].double()
        y = torch.empty(case["M"], case["N"], dtype=torch.float64, device="cuda")
        for r in range(0, case["M"], 256):
            x = s["x"][r:r + 256, :K].float()
            sx = x.abs().max(dim=1).values / 127.0                      # the scale and the quotient are f32 by definition
            q = torch.nan_to_num(x / sx[:, None], nan=0.0).round().clamp(-127, 127).double()
            y[r:r + 256] = torch.einsum("mk,nk->mn", q, w) * sx.double()[:, None] * ws
        return {"y": y}
    T, V, tau = case["T"], case["V"], case["tau"]
    y = s["target"].long()
    step = max(1, (1 << 26) // V)
    parts = []
    for a in range(0, T, step):
        z = s["logits"][a:a + step, :V].double()
        lnp = torch.log_softmax(z / tau, dim=1)
        p = lnp.exp()
        H = torch.special.entr(p).sum(1)
        yy = y[a:a + step, None]
        if case["op"] == "logprobs":
            k = case["k"]
            val, ids = (t[:, :k] for t in torch.sort(z, dim=1, descending=True, stable=True)) if k else (z[:, :0], yy[:, :0])
            dead = torch.isinf(val)
            parts.append((lnp.gather(1, yy)[:, 0], H, torch.logsumexp(z / tau, dim=1), torch.where(dead, -1, ids).int(), lnp.gather(1, ids)))
        else:
            da, db = s["dlogp"][a:a + step, None].double(), s["dentropy"][a:a + step, None].double()
            hot = torch.zeros_like(p).scatter_(1, yy, 1.0)
            plnp = -torch.special.entr(p)
            parts.append(((da * (hot - p) - db * (plnp + p * H[:, None])) / tau,))
            if case["dtype"] == "bf16":
                parts[-1] = (parts[-1][0].float(),)
    if case["op"] == "logprobs":
        return dict(zip(("logp", "entropy", "lse", "top_ids", "top_logp"), (torch.cat(c) for c in zip(*parts))))
    return {"dlogits": torch.cat([c[0] for c in parts])}
