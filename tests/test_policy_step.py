"""What DppoStep's distillation, verification and block-scaled scoring methods hand to the library, with the library's calls replaced by
recorders (CPU)."""
import types

import pytest
import torch

from paper_2603_04135_b200 import binding as B
from paper_2603_04135_b200 import step as S


@pytest.fixture
def calls(monkeypatch):
    seen = []
    for name in ("token_logprobs", "quantize_f8", "linear_f8", "distill_topk", "distill_topk_backward", "verify_drafts"):
        monkeypatch.setattr(B, name, lambda *a, _n=name, **k: seen.append((_n, a)))
    return seen


def make(T_max, V, dtype=B.F32):
    st = S.DppoStep.__new__(S.DppoStep)                              # the constructor asks for a GPU
    st.V, st.T_max, st.device = V, T_max, torch.device("cpu")
    st.counts = torch.tensor([0, 0, 0, T_max], dtype=torch.int32)
    st.status = torch.zeros(1, dtype=torch.int32)
    st.loss_params = types.SimpleNamespace(dtype=dtype, temperature=0.7)
    return st


def test_distill(calls):
    st = make(6, 16)
    z, ids, lp = torch.zeros(6, 16), torch.zeros(6, 5, dtype=torch.int32), torch.zeros(6, 5)
    out = st.distill(z, ids, lp, "normalized", dlogits=z)
    prm, a = calls[0][1][0], calls[0][1]
    assert (prm.T_max, prm.V, prm.top_k, prm.mode, prm.temperature, prm.row_stride) == (6, 16, 5, B.DISTILL_NORMALIZED, 0.7, 16)
    assert a[1] is z and a[9] is z and a[6] is out["loss"] and a[8] is out["stats"] and a[4].tolist() == [6]
    assert st.distill(z, ids, lp, out=out) is out and calls[1][1][0].mode == B.DISTILL_REST and calls[1][1][9] is None
    n = len(calls)
    with pytest.raises(ValueError):
        st.distill(z, ids, lp, "tail")
    with pytest.raises(ValueError):
        st.distill(z, ids[:5], lp)
    for name in ("loss", "lse", "stats"):
        with pytest.raises(ValueError):
            st.distill(z, ids, lp, out=dict(out, **{name: out[name][:5]}))
    assert len(calls) == n


def test_distill_backward_lays_the_gradient_out_as_the_logits(calls):
    st = make(4, 10)
    z = torch.zeros(4, 12)[:, :10]
    out = st.distill(z, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), row_stride=12)
    g = st.distill_backward(z, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), out, row_stride=12)
    assert g.stride() == (12, 1) and calls[1][1][7] is g and calls[1][1][5] is out["stats"] and calls[1][1][0].row_stride == 12


def test_verify(calls):
    st = make(1, 10, B.BF16)
    cu = torch.tensor([0, 3, 3, 5], dtype=torch.int32)
    t = torch.zeros(8, 16, dtype=torch.bfloat16)[:, :10]
    out = st.verify(t, torch.zeros(5, dtype=torch.int32), cu)
    prm, a = calls[0][1][0], calls[0][1]
    assert (prm.T_max, prm.n_seqs, prm.V, prm.target_stride, prm.noise_stride, prm.temperature) == (5, 3, 10, 16, 12, 0.7)
    assert a[2] is None and a[6].shape == (3, 12) and bool((a[6] > 0).all()) and a[5].shape == (5,) and a[11] == (2 * 5 + 3) * 8
    assert out["tokens"].shape == (8,) and out["n_accepted"].shape == (3,)
    g = torch.Generator().manual_seed(1)
    st.verify(t, torch.zeros(5, dtype=torch.int32), cu, draft_logits=t[:5], draft_temperature=2.0, generator=g, out=out)
    assert calls[1][1][0].draft_temperature == 2.0 and calls[1][1][8] is out["tokens"]
    st.verify(t[:1], torch.zeros(0, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    assert calls[2][1][0].target_stride == 16


def test_score_hidden_f8_in_chunks(calls):
    st = make(10, 40)
    W_q, W_s = torch.zeros(300, 256, dtype=torch.float8_e4m3fn)[:, :200], torch.zeros(3, 2)
    hidden = torch.zeros(10, 200)
    st.score_hidden_f8(hidden, W_q, W_s, chunk_tokens=4, n_tokens_dev=torch.tensor([7], dtype=torch.int32))
    assert [c[0] for c in calls] == ["quantize_f8", "linear_f8", "token_logprobs"] * 3
    assert [c[1][4].tolist() for c in calls if c[0] == "quantize_f8"] == [[4], [3], [0]]
    q, lin = calls[0][1][0], calls[1][1][0]
    assert (q.rows_max, q.K, q.q_stride, q.scale_stride, q.block_rows) == (4, 200, 256, 4, 1)
    assert (lin.M_max, lin.N, lin.K, lin.w_stride, lin.x_scale_stride, lin.w_scale_stride, lin.out_stride) == (4, 300, 200, 256, 4, 2, 300)
    n = len(calls)
    for w, s in ((W_q[:, :100], W_s), (W_q, W_s[:2]), (W_q, torch.zeros(3, 3))):
        with pytest.raises(ValueError):
            st.score_hidden_f8(hidden, w, s)
    with pytest.raises(ValueError):
        st.score_hidden_f8(hidden[:9], W_q, W_s)
    assert len(calls) == n
    st0 = make(0, 40)
    st0.score_hidden_f8(hidden[:0], W_q, W_s)
    assert len(calls) == n
