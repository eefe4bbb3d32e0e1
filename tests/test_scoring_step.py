"""What DppoStep's scoring methods hand to the library, with the library's calls replaced by recorders (CPU)."""
import types

import pytest
import torch

from paper_2603_04135_b200 import binding as B
from paper_2603_04135_b200 import step as S


@pytest.fixture
def calls(monkeypatch):
    """Every call of the binding's scoring functions as (name, arguments); tensors are kept alive."""
    seen = []
    for name in ("token_logprobs", "token_logprobs_backward", "quantize_rows_i8", "linear_i8"):
        monkeypatch.setattr(B, name, lambda *a, _n=name, **k: seen.append((_n, a)))
    return seen


def make(T_max, V, dtype=B.F32):
    st = S.DppoStep.__new__(S.DppoStep)                              # the constructor asks for a GPU
    st.V, st.T_max, st.device = V, T_max, torch.device("cpu")
    st.counts = torch.tensor([0, 0, 0, T_max], dtype=torch.int32)
    st.status = torch.zeros(1, dtype=torch.int32)
    st.loss_params = types.SimpleNamespace(dtype=dtype, temperature=1.0)
    return st


def test_scores_into_earlier_outputs(calls):
    st = make(6, 16)
    z, y = torch.zeros(6, 16), torch.zeros(6, dtype=torch.int32)
    out = st.score(z, y, top_k=3)
    assert st.score(z, y, top_k=3, out=out) is out
    assert [c[1][7].data_ptr() for c in calls] == [out["top_ids"].data_ptr()] * 2
    plain = st.score(z, y)
    assert st.score(z, None, out=plain) is plain
    longer = {n: torch.zeros(9, *v.shape[1:], dtype=v.dtype) for n, v in out.items()}      # more rows than T_max
    assert st.score(z, y, top_k=3, out=longer) is longer
    n = len(calls)
    for k in (0, 2, 4, 8):                                           # ids of another pitch would come out scrambled, of 0 stale
        with pytest.raises(ValueError):
            st.score(z, y, top_k=k, out=out)
    for name in ("logp", "entropy", "lse", "stats", "top_ids", "top_logp"):
        with pytest.raises(ValueError):
            st.score(z, y, top_k=3, out=dict(out, **{name: out[name][:5]}))
    with pytest.raises(ValueError):
        st.score(z, y, top_k=3, out=dict(out, top_logp=torch.zeros(18)))
    assert len(calls) == n


def frozen_head(V, H):
    W_q = torch.zeros(V, (H + 127) // 128 * 128, dtype=torch.int8)[:, :H]
    return W_q, torch.ones(V)


def test_weights_of_another_width_are_refused(calls):
    st = make(6, 40)
    hidden = torch.zeros(6, 128)
    st.score_hidden_i8(hidden, *frozen_head(40, 128))
    assert [c[0] for c in calls] == ["quantize_rows_i8", "linear_i8", "token_logprobs"]
    W_q, W_scale = frozen_head(40, 100)                              # padded to 128 columns: the codes of 100 pass as 128
    for args in ((hidden, W_q, W_scale), (hidden, *frozen_head(40, 256)), (hidden, frozen_head(41, 128)[0], torch.ones(40)),
                 (hidden, frozen_head(39, 128)[0], torch.ones(40)), (hidden, torch.zeros(40 * 128, dtype=torch.int8), torch.ones(40))):
        with pytest.raises(ValueError):
            st.score_hidden_i8(*args)
    assert len(calls) == 3


def test_calls_share_no_scratch(calls):
    """Two calls may be under way at once (two streams), or be replayed later (captured): each has codes, scales and logits of
    its own."""
    st = make(6, 40)
    hidden = torch.zeros(6, 128)
    st.score_hidden_i8(hidden, *frozen_head(40, 128), chunk_tokens=4)
    first = [a for _, a in calls]                                    # the recorder keeps the tensors: their memory is not free
    del calls[:]
    st.score_hidden_i8(hidden, *frozen_head(40, 128), chunk_tokens=4)
    second = [a for _, a in calls]
    assert len(first) == len(second) == 6
    for i, names in ((0, (2, 3)), (1, (1, 2, 5)), (2, (1,))):        # codes and scales; codes, scales and logits; logits
        for j in names:
            assert first[i][j].data_ptr() != second[i][j].data_ptr()
            assert first[i][j].data_ptr() == first[i + 3][j].data_ptr()          # the chunks of a call follow each other


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_is_laid_out_as_the_logits_are(calls, dtype):
    """score_backward without dlogits: a result with the logits' shape and row pitch, also of rows that are padded."""
    T, V, ld = 6, 1003, 1008
    st = make(T, V, B.BF16 if dtype is torch.bfloat16 else B.F32)
    buf, y, one = torch.zeros(T, ld, dtype=dtype), torch.zeros(T, dtype=torch.int32), torch.ones(T)
    scored = dict(stats=torch.zeros(T, 4))
    more = torch.zeros(T + 3, ld, dtype=dtype)
    for logits in (buf[:, :V], buf, buf.view(2, 3, ld), buf.view(2, 3, ld)[:, :, :V], buf.view(-1), more[:, :V], more[2:-1, :V]):
        got = st.score_backward(logits, y, scored, dlogp=one, row_stride=ld)
        assert got.shape == logits.shape and got.dtype is dtype and not bool(got.any())
        assert calls[-1][0] == "token_logprobs_backward" and calls[-1][1][7] is got
        for x in (logits, got):                                      # what the binding then asks of both
            assert B._mat(x, "x", x.get_device(), dtype, T, V, ld) == x.data_ptr()
        if logits.dim() > 1:
            assert got.stride() == logits.stride()
    st1 = make(1, V)
    row = torch.zeros(1, ld)[:, :V]
    assert st1.score_backward(row, y[:1], scored, dlogp=one[:1], row_stride=ld).shape == row.shape
    mine = torch.zeros(T, ld, dtype=dtype)
    assert st.score_backward(buf, y, scored, dlogp=one, dlogits=mine, row_stride=ld) is mine
