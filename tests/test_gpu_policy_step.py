"""A training step's run over the operators around a second policy: a teacher's head in block-scaled fp8, its alternatives, distillation on
them with its gradient, and earlier completions verified under the current policy."""
import numpy as np
import pytest
import torch

from oracle import distill, f8, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_teacher_to_gradient_to_verified_tokens(dtype):
    from paper_2603_04135_b200.step import DppoStep, quantize_f8
    P, G, V, H, T, K = 2, 4, 2000, 384, 150, 12
    st = DppoStep(P, G, 512, 4, 0.25, 0.25, V, dtype, T, temperature=0.9)
    st.counts[3] = 140                                               # true tokens; the rest are rows that nothing may touch
    g = torch.Generator(device="cuda").manual_seed(3)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    hidden = torch.empty(T, H, device="cuda").normal_(0, 1, generator=g)
    hidden[:, 5] *= 300.0                                            # an outlier channel
    W = torch.empty(V, H, device="cuda").normal_(0, 0.08, generator=g)
    W[:, 5] /= 300.0
    hidden, W = hidden.to(tdt), W.to(tdt)
    W_q, W_s = quantize_f8(W)
    teacher = st.score_hidden_f8(hidden, W_q, W_s, top_k=K, chunk_tokens=64)
    again = st.score_hidden_f8(hidden, W_q, W_s, top_k=K)            # chunks change no result but the order of a sum
    q, qs = f8.quantize(hidden.float().cpu().numpy(), 1)
    zt, mag = f8.linear(q, qs, W_q.view(torch.uint8).cpu().numpy(), W_s.cpu().numpy())
    lt = zt / 0.9
    lt = lt - np.log(np.exp(lt - lt.max(1, keepdims=True)).sum(1, keepdims=True)) - lt.max(1, keepdims=True)
    ids, lp = teacher["top_ids"][:140].cpu().numpy(), teacher["top_logp"][:140].cpu().numpy()
    tol = 2 * (128 * 2.0 ** -23 + 40 * 2.0 ** -24) * mag[:140].max() / 0.9 + 1e-5
    assert np.abs(lp - np.take_along_axis(lt[:140], ids, 1)).max() < tol
    assert torch.equal(teacher["top_ids"][140:], torch.full((10, K), -1, dtype=torch.int32, device="cuda"))
    assert (teacher["top_logp"][:140] - again["top_logp"][:140]).abs().max() < tol

    student = (torch.from_numpy(zt).to("cuda").float() + torch.empty(T, V, device="cuda").normal_(0, 0.5, generator=g)).to(tdt)
    w = torch.rand(T, device="cuda", generator=g)
    grad = torch.full_like(student, 7.0)
    out = st.distill(student, teacher["top_ids"], teacher["top_logp"], weight=w, dlogits=grad)
    lone = st.distill(student, teacher["top_ids"], teacher["top_logp"])
    back = st.distill_backward(student, teacher["top_ids"], teacher["top_logp"], lone, dloss=w)
    zs = student.double().cpu().numpy()
    want = distill.distill_topk(zs[:140], ids, lp, distill.REST, 0.9)
    assert np.abs(out["loss"][:140].cpu().numpy() - want["loss"]).max() < 2e-5
    ref = want["dz"] * w[:140].double().cpu().numpy()[:, None]
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for x in (grad, back):
        # 16-bit exponentials of bf16 rows 2^-11, f32 arithmetic 1e-4 of a probability at this size
        err = np.abs(x[:140].double().cpu().numpy() - ref)
        assert (err <= half * np.abs(ref) + (2.0 ** -11 if dtype == "bf16" else 0) * 2 * np.abs(ref) + 2e-6).all(), err.max()
    assert bool((grad[140:] == 7.0).all()) and bool((back[140:] == 0).all())

    # the completions of an earlier epoch, verified under the student
    lens = [20, 0, 33, 7, 60]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    rows = sum(lens) + len(lens)
    u, noise = torch.rand(sum(lens), device="cuda", generator=g), torch.empty(len(lens), V, device="cuda").exponential_(generator=g)
    drafts = torch.cat([student[c + b:c + b + n, :V].float().argmax(1) for b, (c, n) in enumerate(zip(cu.tolist(), lens))]).int()
    res = st.verify(student[:rows], drafts, cu, uniforms=u, noise=noise)
    torch.cuda.synchronize()
    wv = verify.verify_drafts(zs[:rows], None, drafts.cpu().numpy(), cu.cpu().numpy().astype(np.int64), u.double().cpu().numpy(),
                              noise.double().cpu().numpy(), 0.9, 1.0)
    sure = wv["margin"] > 1e-4
    assert sure.sum() >= len(lens) - 1 and np.array_equal(res["n_accepted"].cpu().numpy()[sure], wv["n_accepted"][sure])
    if sure.all():
        assert np.array_equal(res["tokens"].cpu().numpy(), wv["tokens"])
        # logp is the student's score of those tokens, as the loss takes it
        sc = st.score(student, res["tokens"].clamp_min(0).new_zeros(T).index_copy(0, torch.arange(rows, device="cuda"), res["tokens"].clamp_min(0)))
        kept = res["tokens"] >= 0
        assert (res["logp"][kept] - sc["logp"][:rows][kept]).abs().max() < 2e-5
    assert int(st.status.item()) == 0
