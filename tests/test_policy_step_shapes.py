"""What DppoStep's distillation, verification and block-scaled scoring methods refuse or lay out by the shapes they are given, with the
library's calls replaced by recorders (CPU)."""
import pytest
import torch

from paper_2603_04135_b200 import binding as B
from paper_2603_04135_b200 import step as S
from test_policy_step import calls, make  # noqa: F401  (a fixture)


def test_distill_wants_one_log_prob_for_each_id(calls):  # noqa: F811
    """Log-probs of another width would be read with the ids' pitch."""
    st = make(6, 16)
    z, ids = torch.zeros(6, 16), torch.zeros(6, 5, dtype=torch.int32)
    out = st.distill(z, ids, torch.zeros(6, 5))
    n = len(calls)
    for lp in (torch.zeros(6, 8), torch.zeros(6, 4), torch.zeros(5, 5), torch.zeros(30), torch.zeros(6, 5, 1), torch.zeros(8, 5)[:5]):
        with pytest.raises(ValueError):
            st.distill(z, ids, lp)
        with pytest.raises(ValueError):
            st.distill_backward(z, ids, lp, out)
    assert len(calls) == n
    more = torch.zeros(8, 5)                                         # what an earlier call for more tokens left
    st.distill(z, more.int(), more)
    st.distill_backward(z, ids, more, out)
    assert len(calls) == n + 2


@pytest.mark.parametrize("dtype,per", [(torch.bfloat16, 8), (torch.float32, 4)])
def test_a_single_row_has_no_pitch_to_be_aligned(monkeypatch, dtype, per):
    """Rows on 16 bytes: of one row that says nothing about its length."""
    seen = []
    for name in ("quantize_f8", "quantize_rows_i8"):
        monkeypatch.setattr(B, name, lambda prm, *a, **k: seen.append(prm.x_stride))
    for n in ("linear_f8", "linear_i8", "token_logprobs"):
        monkeypatch.setattr(B, n, lambda *a, **k: None)
    K = 2501
    pitch = -(-K // per) * per
    S.quantize_f8(torch.zeros(1, K, dtype=dtype))
    S.quantize_f8(torch.zeros(1, K, dtype=dtype), block_rows=1)
    S.quantize_rows_i8(torch.zeros(1, K, dtype=dtype))
    st = make(1, 40)
    st.score_hidden_f8(torch.zeros(1, K, dtype=dtype), torch.zeros(40, 2512, dtype=torch.float8_e4m3fn)[:, :K], torch.zeros(1, 20))
    st.score_hidden_i8(torch.zeros(1, K, dtype=dtype), torch.zeros(40, 2512, dtype=torch.int8)[:, :K], torch.zeros(40))
    assert seen == [pitch] * 5
    S.quantize_f8(torch.zeros(3, 2600, dtype=dtype)[:, :K])          # several rows: as they lie
    S.quantize_f8(torch.zeros(3, 2600, dtype=dtype)[:1, :K])
    assert seen[5:] == [2600, 2600]
