"""Cases of the operators around a second policy: distillation from a teacher's top log-probs (loss, loss with its gradient,
gradient alone), verification of drafted tokens, and the 8-bit floating-point product with a scale for each block of 128.

`own` chooses between the plain torch form of each operator and the library's calls.
"""
import math

import torch

own = False

_BYTES = {"bf16": 2, "f32": 4}
_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_MODE = {"given": 0, "normalized": 1, "rest": 2}


# ---- cases ----------------------------------------------------------------------------------------
def listed():
    return [
        # evaluation of a few tokens under a teacher's 20 alternatives: latency counts
        dict(name="distill_loss_16_tokens", op="loss", T=16, V=151936, dtype="bf16", k=20, mode="rest", tau=1.0, mask="none"),
        # the loss of a packed batch over the Qwen3 vocabulary, without training on it
        dict(name="distill_loss_8192_tokens", op="loss", T=8192, V=151936, dtype="bf16", k=32, mode="rest", tau=1.0, mask="padding"),
        # a training step of a small vocabulary under a constraint: short ragged rows, f32
        dict(name="distill_step_short_rows", op="step", T=20011, V=1021, dtype="f32", k=5, mode="normalized", tau=0.7, mask="sparse"),
        # a training step of a packed batch: loss and gradient in one call
        dict(name="distill_step_8192_tokens", op="step", T=8192, V=151936, dtype="bf16", k=20, mode="rest", tau=1.0, mask="padding"),
        # gradient of a small micro-batch
        dict(name="distill_backward_64_tokens", op="backward", T=64, V=151936, dtype="bf16", k=20, mode="rest", tau=1.0, mask="none"),
        # f32 rows of a mid-sized vocabulary, a softened student
        dict(name="distill_backward_f32", op="backward", T=2003, V=50304, dtype="f32", k=32, mode="given", tau=2.0, mask="none"),
        # one sequence with four drafted tokens: the inner step of a rollout, latency counts
        dict(name="verify_1_sequence", op="verify", B=1, n=4, V=151936, dtype="bf16", draft="model", tau=1.0, mask="padding"),
        # a rollout batch of ragged drafts
        dict(name="verify_128_sequences", op="verify", B=128, n=7, V=151936, dtype="bf16", draft="model", tau=1.0, mask="padding"),
        # drafts copied from earlier completions (no draft model), f32 logits of a ragged vocabulary
        dict(name="verify_copied_drafts", op="verify", B=37, n=61, V=32003, dtype="f32", draft="copied", tau=0.8, mask="none"),
        # LM-head of one decoded token: the weights are read once
        dict(name="linear_f8_1_token", op="linear", M=1, K=2560, N=151936, dtype="bf16", out="f32"),
        # a square projection for a decode batch
        dict(name="linear_f8_64_tokens", op="linear", M=64, K=4096, N=4096, dtype="bf16", out="bf16"),
        # LM-head of a scoring chunk: tensor-core bound
        dict(name="linear_f8_2048_tokens", op="linear", M=2048, K=2560, N=151936, dtype="bf16", out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "step", "backward", "verify", "linear"])
    if op == "linear":
        M, K, N = _log_int(rng, 1, 4096), _log_int(rng, 48, 8192), _log_int(rng, 48, 151936)
        M = max(1, min(M, 2048 * 2560 * 151936 // (K * N), 2048 * 151936 // N))
        return dict(op=op, M=M, K=K, N=N, dtype=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    dtype = rng.choice(["bf16", "f32"])
    V = _log_int(rng, 250, 151936)
    mask, tau = rng.choice(["none", "padding", "sparse"]), round(rng.uniform(0.5, 2.0), 3)
    if op == "verify":
        B, n = _log_int(rng, 1, 256), _log_int(rng, 1, 64)
        B = max(1, min(B, 128 * 8 * 151936 * 2 // (V * _BYTES[dtype] * (n + 1))))
        return dict(op=op, B=B, n=n, V=V, dtype=dtype, draft=rng.choice(["model", "copied"]), tau=tau, mask=mask)
    T = min(_log_int(rng, 1, 30000), 8192 * 151936 * 2 // (V * _BYTES[dtype]))
    return dict(op=op, T=T, V=V, dtype=dtype, k=rng.randint(1, 32), mode=rng.choice(["given", "normalized", "rest"]), tau=tau, mask=mask)


# ---- inputs ---------------------------------------------------------------------------------------
def _padded(V, dtype):
    per = 16 // _BYTES[dtype]
    return (V + per - 1) // per * per


def _logits(rows, case, gen):
    """Rows of logits as a language model has them: N(0, 2) over the vocabulary and 24 likely tokens well above, in rows
    padded to 16 bytes.  `padding`: the last entries of the vocabulary are no tokens (-inf)."""
    V, dt = case["V"], _TORCH[case["dtype"]]
    z = torch.empty(rows, _padded(V, case["dtype"]), dtype=dt, device="cuda").normal_(0.0, 2.0, generator=gen)
    top = (torch.randint(0, V, (rows, 1), device="cuda", generator=gen) + torch.arange(24, device="cuda") * (V // 24)) % V
    z.scatter_(1, top, torch.empty(rows, 24, device="cuda").uniform_(6.0, 15.0, generator=gen).to(dt))
    if case["mask"] == "padding":
        z[:, V - V // 500:] = -math.inf
    return z


def _constrain(z, case, gen):
    """`sparse`: nine of ten entries are not allowed."""
    if case["mask"] == "sparse":
        z.masked_fill_(torch.rand(z.shape, device="cuda", generator=gen) < 0.9, -math.inf)


def _like(z, case, spread, gen, a, b):
    """f32 logits of another model that mostly agrees with rows a..b of z."""
    x = z[a:b, :case["V"]].float()
    return x + torch.empty(x.shape, device="cuda").normal_(0.0, spread, generator=gen)


def _rows_at_once(V):
    return max(1, (1 << 27) // V)


def _prepare_distill(case, seed, gen, s):
    T, V, k, tau = case["T"], case["V"], case["k"], case["tau"]
    z = _logits(T, case, gen)
    _constrain(z, case, gen)
    ids = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    logp = torch.full((T, k), -math.inf, dtype=torch.float32, device="cuda")
    kk = min(k, V)
    for a in range(0, T, _rows_at_once(V)):
        b = min(T, a + _rows_at_once(V))
        t = _like(z, case, 0.7, gen, a, b)
        val, at = torch.topk(t, kk, dim=1)
        dead = val == -math.inf
        logp[a:b, :kk] = torch.where(dead, val, val - torch.logsumexp(t, dim=1, keepdim=True)).nan_to_num_(nan=-math.inf)
        ids[a:b, :kk] = torch.where(dead, -1, at).int()
    ids[96::97] = -1                                             # tokens that the teacher did not score
    logp[96::97] = -math.inf
    s.update(logits=z, ids=ids, logp=logp, status=torch.zeros(1, dtype=torch.int32, device="cuda"),
             weight=torch.empty(T, device="cuda").uniform_(0.1, 2.0, generator=gen) / T)
    f32 = dict(dtype=torch.float32, device="cuda")
    if case["op"] != "backward":
        s.update(loss=torch.zeros(T, **f32), lse=torch.zeros(T, **f32), stats=torch.zeros(T, 4, **f32))
    if case["op"] == "step":
        s.update(dlogits=torch.zeros_like(z))
    if case["op"] == "backward":
        # what the forward call leaves for the backward: the maximum, the sum of exponentials relative to it, the teacher's mass,
        # and the remainder over the student's
        stats = torch.zeros(T, 4, **f32)
        for a in range(0, T, _rows_at_once(V)):
            b = min(T, a + _rows_at_once(V))
            x = z[a:b, :V].double()
            m = x.amax(1)
            m0 = torch.where(m == -math.inf, torch.zeros_like(m), m)
            e = ((x - m0[:, None]) / tau).exp_()
            tot = e.sum(1)
            i = ids[a:b].long()
            p = torch.where(i >= 0, logp[a:b].double().exp(), torch.zeros(i.shape, dtype=torch.float64, device="cuda"))
            P = p.sum(1)
            stats[a:b, 0], stats[a:b, 1] = m.float(), tot.float()
            stats[a:b, 2] = P.float() if case["mode"] == "given" else (P > 0).float()
            if case["mode"] == "rest":
                keep = torch.ones(x.shape[0], V + 1, dtype=torch.float64, device="cuda")
                keep.scatter_(1, torch.where(i >= 0, i, V), 0.0)
                sigma = (e * keep[:, :V]).sum(1) / tot
                r = 1.0 - P
                r = torch.where(r > 2.0 ** -16, r, torch.zeros_like(r))
                stats[a:b, 2] = (P + r).float()
                stats[a:b, 3] = torch.where(r > 0, r / sigma, r).float()
        s.update(stats=stats, dlogits=torch.zeros_like(z))


def _lengths(case):
    """Drafted tokens of each sequence: n down to half of it."""
    n = case["n"]
    return [n - i % (n - n // 2 + 1) for i in range(case["B"])]


def _prepare_verify(case, seed, gen, s):
    B, n, V, tau = case["B"], case["n"], case["V"], case["tau"]
    lens = torch.tensor(_lengths(case), device="cuda")[torch.randperm(B, device="cuda", generator=gen)]
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[1:] = lens.cumsum(0)
    T = int(cu[B])
    target = _logits(T + B, case, gen)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), lens)
    trow = torch.arange(T, device="cuda") + seq                   # target row of each drafted token
    if case["draft"] == "copied":
        # mostly what the target would say itself
        drafts = target[trow, :V].float().argmax(1)
        drafts = torch.where(torch.rand(T, device="cuda", generator=gen) < 0.05, torch.randint(0, V, (T,), device="cuda", generator=gen), drafts)
        draft = None
    else:
        draft = torch.full((T, target.shape[1]), -math.inf, dtype=target.dtype, device="cuda")
        drafts = torch.zeros(T, dtype=torch.int64, device="cuda")
        for a in range(0, T, _rows_at_once(V)):
            b = min(T, a + _rows_at_once(V))
            x = target[trow[a:b], :V].float()
            x += torch.empty(x.shape, device="cuda").normal_(0.0, 0.6, generator=gen)
            draft[a:b, :V] = x.to(draft.dtype)
            e = torch.empty(x.shape, device="cuda").exponential_(generator=gen)
            drafts[a:b] = (draft[a:b, :V].float() / tau - e.log()).argmax(1)
    _constrain(target, case, gen)                                 # the target's constraint is not known to the draft
    s.update(T=T, cu=cu, target=target, draft=draft, drafts=drafts.int(), lens=lens,
             u=torch.rand(T, device="cuda", generator=gen), noise=torch.empty(B, (V + 3) // 4 * 4, device="cuda").exponential_(generator=gen),
             n_accepted=torch.zeros(B, dtype=torch.int32, device="cuda"), tokens=torch.zeros(T + B, dtype=torch.int32, device="cuda"),
             logp=torch.zeros(T + B, device="cuda"), status=torch.zeros(1, dtype=torch.int32, device="cuda"),
             workspace=torch.zeros(16 * (2 * T + B) + 256, dtype=torch.uint8, device="cuda"))


def _prepare_linear(case, seed, gen, s):
    M, K, N = case["M"], case["K"], case["N"]
    f32 = dict(dtype=torch.float32, device="cuda")
    ldx, ldq, kb = _padded(K, case["dtype"]), (K + 127) // 128 * 128, (K + 127) // 128
    x = torch.empty(M, ldx, **f32).normal_(0.0, 1.0, generator=gen)
    x *= torch.exp(torch.empty(ldx, **f32).normal_(0.0, 1.0, generator=gen))           # channels of different size
    w = torch.empty(N, ldq, **f32).normal_(0.0, 100.0, generator=gen).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
    s.update(x=x.to(_TORCH[case["dtype"]]), w=w,
             w_scale=torch.empty((N + 127) // 128, kb, **f32).uniform_(0.5, 1.5, generator=gen) / (100.0 * math.sqrt(K)),
             q=torch.zeros(M, ldq, dtype=torch.float8_e4m3fn, device="cuda"), q_scale=torch.zeros(kb, (M + 3) // 4 * 4, **f32),
             y=torch.zeros(M, N, dtype=_TORCH[case["out"]], device="cuda"), status=torch.zeros(1, dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = dict(case)
    {"linear": _prepare_linear, "verify": _prepare_verify}.get(case["op"], _prepare_distill)(case, seed, gen, s)
    return s


# ---- one pass ---------------------------------------------------------------------------------------
def run(s):
    return {"linear": _run_linear, "verify": _run_verify, "backward": _run_backward}.get(s["op"], _run_distill)(s)


def _run_linear(s):
    M, K, N = s["M"], s["K"], s["N"]
    if own:
        from paper_2603_04135_b200 import binding as B
        code = {"f32": B.F32, "bf16": B.BF16}
        ldq, lds = s["q"].shape[1], s["q_scale"].shape[1]
        B.quantize_f8(B.QuantizeF8Params(M, K, code[s["dtype"]], s["x"].shape[1], ldq, lds, 1), s["x"], s["q"], s["q_scale"])
        B.linear_f8(B.LinearF8Params(M, N, K, ldq, s["w"].shape[1], N, lds, s["w_scale"].shape[1], code[s["out"]]), s["q"], s["q_scale"],
                    s["w"], s["w_scale"], s["y"], status=s["status"])
        return {"y": s["y"]}
    kb = s["w_scale"].shape[1]
    x = torch.zeros(M, kb * 128, device="cuda")
    x[:, :K] = s["x"][:, :K].float()
    x = x.view(M, kb, 128)
    scale = (x.abs().amax(2, keepdim=True) * (1.0 / 448.0)).clamp_min(2.0 ** -126)
    q = (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() * scale
    w = s["w"].float().view(N, kb, 128) * s["w_scale"].repeat_interleave(128, 0)[:N, :, None]
    w.view(N, kb * 128)[:, K:] = 0.0
    return {"y": (q.view(M, kb * 128) @ w.view(N, kb * 128).t()).to(_TORCH[s["out"]])}


def _distill_params(s, B):
    return B.DistillParams(s["T"], s["V"], B.BF16 if s["dtype"] == "bf16" else B.F32, s["logits"].shape[1], s["k"], _MODE[s["mode"]], s["tau"])


def _plain_distill(s, gradient, weight):
    """Per-token loss, log-sum-exp and weighted gradient, in f32."""
    V, tau = s["V"], s["tau"]
    z = s["logits"][:, :V].float()
    m = z.amax(1, keepdim=True)
    x = (z - torch.where(m == -math.inf, torch.zeros_like(m), m)) / tau
    e = torch.exp(x)
    total = e.sum(1)
    l = torch.log(total)
    have = s["ids"] >= 0
    ids = torch.where(have, s["ids"], 0).long()
    zero = torch.zeros_like(s["logp"])
    p = torch.where(have, torch.exp(s["logp"]), zero)
    lp = torch.where(have, s["logp"], zero)
    P = p.sum(1, keepdim=True)
    r = torch.zeros_like(P)
    if s["mode"] == "normalized":
        p, lp = torch.where(P > 0, p / P, zero), torch.where(P > 0, lp - torch.log(P), zero)
    elif s["mode"] == "rest":
        r = (1.0 - torch.where(have, torch.exp(s["logp"].double()), zero.double()).sum(1, keepdim=True)).float()
        r = torch.where(r > 2.0 ** -16, r, torch.zeros_like(r))
    ls = x.gather(1, ids) - l[:, None]
    loss = torch.where(p > 0, p * (lp - ls), zero).sum(1)
    share = torch.zeros_like(r)
    if s["mode"] == "rest":
        keep = torch.ones(z.shape[0], V + 1, device=z.device).scatter_(1, torch.where(have, ids, V), 0.0)
        sigma = (e * keep[:, :V]).sum(1, keepdim=True) / total[:, None]
        loss = loss + torch.where(r > 0, r * torch.log(r / sigma), r)[:, 0]
        share = torch.where(r > 0, r / sigma, r)
    lse = torch.where(m[:, 0] == -math.inf, m[:, 0], m[:, 0] / tau + l)
    if not gradient:
        return loss, lse, None
    sm = e / total[:, None]
    G = p.sum(1, keepdim=True) + r
    g = sm * (G - share)
    listed_ = (sm.gather(1, ids) * share) * have                  # what the line above took off there; one entry per id
    g.scatter_add_(1, ids, listed_ - p)
    g = torch.where(m == -math.inf, torch.zeros_like(g), g)
    return loss, lse, (g * (weight[:, None] / tau)).to(s["logits"].dtype)


def _run_distill(s):
    step = s["op"] == "step"
    if own:
        from paper_2603_04135_b200 import binding as B
        B.distill_topk(_distill_params(s, B), s["logits"], s["ids"], s["logp"], None, s["weight"] if step else None, s["loss"], s["lse"],
                       s["stats"], s["dlogits"] if step else None, status=s["status"])
        out = {"loss": s["loss"], "lse": s["lse"]}
        if step:
            out["dlogits"] = s["dlogits"][:, :s["V"]]
        return out
    loss, lse, g = _plain_distill(s, step, s["weight"])
    return {"loss": loss, "lse": lse, "dlogits": g} if step else {"loss": loss, "lse": lse}


def _run_backward(s):
    if own:
        from paper_2603_04135_b200 import binding as B
        B.distill_topk_backward(_distill_params(s, B), s["logits"], s["ids"], s["logp"], None, s["stats"], s["weight"], s["dlogits"],
                                status=s["status"])
        return {"dlogits": s["dlogits"][:, :s["V"]]}
    return {"dlogits": _plain_distill(s, True, s["weight"])[2]}


def _run_verify(s):
    B_, n, V, T, tau = s["B"], s["n"], s["V"], s["T"], s["tau"]
    if own:
        from paper_2603_04135_b200 import binding as B
        prm = B.VerifyParams(T, B_, V, B.BF16 if s["dtype"] == "bf16" else B.F32, s["target"].shape[1],
                             s["draft"].shape[1] if s["draft"] is not None else 0, s["noise"].shape[1], tau, tau)
        B.verify_drafts(prm, s["target"], s["draft"], s["drafts"], s["cu"], s["u"], s["noise"], s["n_accepted"], s["tokens"], s["logp"],
                        s["workspace"], s["workspace"].numel(), status=s["status"])
        return {k: s[k] for k in ("n_accepted", "tokens", "logp")}
    # in 64 bits: both the acceptance and the race compare values that lie close together now and then
    seq = torch.repeat_interleave(torch.arange(B_, device="cuda"), s["lens"], output_size=T)
    at = torch.arange(T, device="cuda")
    place = at - s["cu"][:-1].long()[seq]
    y = s["drafts"].long()
    lse_t = torch.cat([torch.logsumexp(c[:, :V].double() / tau, dim=1) for c in s["target"].split(_rows_at_once(V))])
    lp = s["target"][at + seq, y].double() / tau - lse_t[at + seq]
    if s["draft"] is not None:
        lse_d = torch.cat([torch.logsumexp(c[:, :V].double() / tau, dim=1) for c in s["draft"].split(_rows_at_once(V))])
        lq = s["draft"][at, y].double() / tau - lse_d
    else:
        lq = torch.zeros_like(lp)
    ok = torch.zeros(B_, n + 1, dtype=torch.bool, device="cuda")
    ok[seq, place] = s["u"].double() * lq.exp() < lp.exp()
    n_acc = ok.long().cumprod(1).sum(1)
    # the next token: from the residual at a rejection, from the target after the last drafted token
    row = s["cu"][:-1].long() + torch.arange(B_, device="cuda") + n_acc
    p = (s["target"][row, :V].double() / tau - lse_t[row, None]).exp()
    rejected = n_acc < s["lens"]
    w = p
    if T > 0:
        d = (s["cu"][:-1].long() + n_acc).clamp_max(T - 1)
        if s["draft"] is not None:
            q = (s["draft"][d, :V].double() / tau - lse_d[d, None]).exp()
        else:
            q = torch.zeros_like(p).scatter_(1, y[d][:, None], 1.0)
        res = (p - q).clamp_min(0.0)
        w = torch.where((rejected & (res.amax(1) > 0))[:, None], res, p)
    nxt = (w / s["noise"][:, :V].double()).argmax(1)
    tokens = torch.full((T + B_,), -1, dtype=torch.int32, device="cuda")
    logp = torch.zeros(T + B_, dtype=torch.float64, device="cuda")
    kept = place < n_acc[seq]
    tokens[at + seq] = torch.where(kept, s["drafts"], -1)
    logp[at + seq] = torch.where(kept, lp, torch.zeros_like(lp))
    tokens[row] = nxt.int()
    logp[row] = s["target"][row, nxt].double() / tau - lse_t[row]
    return {"n_accepted": n_acc.int(), "tokens": tokens, "logp": logp.float()}


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        kb = (K + 127) // 128
        return {"bytes": M * K * _BYTES[case["dtype"]] + N * K + 4 * kb * ((N + 127) // 128) + M * N * _BYTES[case["out"]], "flops": 2 * M * N * K}
    V, b = case["V"], _BYTES[case["dtype"]]
    if case["op"] == "verify":
        T = sum(_lengths(case))
        rows = T + case["B"] + (T if case["draft"] == "model" else 0)
        return {"bytes": rows * V * b + case["B"] * V * 4 + 16 * (T + case["B"]), "flops": 3 * rows * V}
    T = case["T"]
    if case["op"] == "loss":
        return {"bytes": T * (V * b + 8 * case["k"] + 8), "flops": 4 * T * V}
    return {"bytes": T * (2 * V * b + 8 * case["k"] + 12), "flops": 6 * T * V}


# ---- the definition in 64 bits -----------------------------------------------------------------------
def _exact_linear(case, s):
    M, K, N = case["M"], case["K"], case["N"]
    if 2 * M * N * K > 6e11:
        return None                                                 # 64-bit products of this size take too long
    y = torch.empty(M, N, dtype=torch.float64, device="cuda")
    first = s["w_scale"].repeat_interleave(128, 1)[:, :K].double()
    rows = max(128, (1 << 27) // K // 128 * 128)
    xs = []
    for a in range(0, K, 128):                                      # the scale and the quotient are f32 by definition
        x = s["x"][:, a:min(a + 128, K)].float()
        sx = torch.maximum(x.abs().max(dim=1).values * (1.0 / 448.0), torch.tensor(2.0 ** -126, device="cuda"))[:, None]
        xs.append(torch.clamp(x / sx, -448.0, 448.0).to(torch.float8_e4m3fn).float().double() * sx.double())
    x = torch.cat(xs, dim=1)
    for a in range(0, N, rows):
        b = min(N, a + rows)
        w = s["w"][a:b, :K].float().double() * first[a // 128:(b + 127) // 128].repeat_interleave(128, 0)[:b - a]
        y[:, a:b] = torch.einsum("mk,nk->mn", x, w)
    return {"y": y}


def _exact_distill(case, s):
    T, V, tau = case["T"], case["V"], case["tau"]
    losses, lses, grads = [], [], []
    step = max(1, (1 << 26) // V)
    for a in range(0, T, step):
        z = s["logits"][a:a + step, :V].double() / tau
        lse = torch.logsumexp(z, dim=1)
        empty = lse == -math.inf
        lnp = z - torch.where(empty, torch.zeros_like(lse), lse)[:, None]
        n = z.shape[0]
        teacher = torch.zeros(n, V + 1, dtype=torch.float64, device="cuda")
        listed_ = torch.zeros(n, V + 1, dtype=torch.bool, device="cuda")
        ids = s["ids"][a:a + step].long()
        at = torch.where(ids < 0, V, ids)
        teacher.scatter_add_(1, at, torch.exp(s["logp"][a:a + step].double()))
        listed_.scatter_(1, at, True)
        teacher, listed_ = teacher[:, :V], listed_[:, :V]
        P = teacher.sum(1, keepdim=True)
        if case["mode"] == "normalized":
            teacher = torch.where(P > 0, teacher / P, teacher)
        sm = lnp.exp()
        loss = -(torch.special.entr(teacher) + torch.where(teacher > 0, teacher * lnp, torch.zeros_like(lnp))).sum(1)
        g = sm * teacher.sum(1, keepdim=True) - teacher
        if case["mode"] == "rest":
            r = 1.0 - P[:, 0]
            r = torch.where(r > 2.0 ** -16, r, torch.zeros_like(r))
            lsig = torch.logsumexp(lnp.masked_fill(listed_, -math.inf), dim=1)
            loss = loss + torch.where(r > 0, r * (torch.log(r) - lsig), r)
            g = g + torch.where(listed_, r[:, None] * sm, torch.where(r > 0, r - r * torch.exp(-lsig), r)[:, None] * sm)
        losses.append(loss)
        lses.append(lse)
        if case["op"] != "loss":
            g = g.masked_fill(empty[:, None], 0.0) * (s["weight"][a:a + step].double() / tau)[:, None]
            grads.append(g.float() if case["dtype"] == "bf16" else g)
    if case["op"] == "backward":
        return {"dlogits": torch.cat(grads)}
    out = {"loss": torch.cat(losses), "lse": torch.cat(lses)}
    if case["op"] == "step":
        out["dlogits"] = torch.cat(grads)
    return out


def _exact_verify(case, s):
    """One sequence after the other, as the definition reads."""
    V, tau, T, B_ = case["V"], case["tau"], s["T"], case["B"]
    cu, u, drafts = s["cu"].tolist(), s["u"].tolist(), s["drafts"].tolist()
    n_acc, tokens = [], [-1] * (T + B_)
    logp = torch.zeros(T + B_, dtype=torch.float64, device="cuda")
    for b in range(B_):
        n = cu[b + 1] - cu[b]
        p = torch.softmax(s["target"][cu[b] + b:cu[b + 1] + b + 1, :V].double() / tau, dim=1)
        y = s["drafts"][cu[b]:cu[b + 1]].long()[:, None]
        py = p[:n].gather(1, y)[:, 0].tolist()
        if s["draft"] is not None:
            q = torch.softmax(s["draft"][cu[b]:cu[b + 1], :V].double() / tau, dim=1)
            qy = q.gather(1, y)[:, 0].tolist()
        else:
            q, qy = None, [1.0] * n
        j = 0
        while j < n and u[cu[b] + j] * qy[j] < py[j]:
            j += 1
        w = p[j]
        if j < n:
            left = p[j].clone()
            if q is None:
                left[drafts[cu[b] + j]] = 0.0
            else:
                left = torch.relu(left - q[j])
            if float(left.max()) > 0:
                w = left
        nxt = int(torch.argmax(w / s["noise"][b, :V].double()))
        at = cu[b] + b
        tokens[at:at + j + 1] = drafts[cu[b]:cu[b] + j] + [nxt]
        n_acc.append(j)
        picked = torch.tensor(tokens[at:at + j + 1], device="cuda")[:, None]
        logp[at:at + j + 1] = p[:j + 1].gather(1, picked)[:, 0].log()
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"n_accepted": torch.tensor(n_acc, **i32), "tokens": torch.tensor(tokens, **i32), "logp": logp}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "verify": _exact_verify}.get(case["op"], _exact_distill)(case, s)
