"""What DppoStep's distillation, verification and block-scaled scoring methods refuse or lay out by the shapes they are given, with the
library's calls replaced by recorders (CPU)."""
import pytest
import torch

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
