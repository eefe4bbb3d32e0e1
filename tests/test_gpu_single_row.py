"""One row of any length through the quantisations and the scores from hidden states, against the same row of a padded matrix, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", [1, 5, 127, 129, 2501])
def test_single_row(dtype, K):
    from paper_2603_04135_b200 import step as S
    g = torch.Generator(device="cuda").manual_seed(K)
    one = torch.empty(1, K, device="cuda").normal_(0.0, 1.0, generator=g).to(dtype)
    two = torch.zeros(2, (K + 15) // 16 * 16, dtype=dtype, device="cuda")[:, :K]
    two[0] = one[0]
    u8 = lambda t: t.contiguous().view(torch.uint8)
    for rows in (1, 128):
        (q1, s1), (q2, s2) = S.quantize_f8(one, rows), S.quantize_f8(two, rows)
        assert torch.equal(u8(q1), u8(q2[:1])) and torch.equal(s1, s2[:, :1] if rows == 1 else s2)
    (q1, s1), (q2, s2) = S.quantize_rows_i8(one), S.quantize_rows_i8(two)
    assert torch.equal(q1, q2[:1]) and torch.equal(s1, s2[:1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_score_of_a_single_token(dtype):
    from paper_2603_04135_b200 import step as S
    H, V = 301, 700
    g = torch.Generator(device="cuda").manual_seed(3)
    W = torch.empty(V, 304, device="cuda").normal_(0.0, 0.1, generator=g)[:, :H]
    h = torch.empty(1, H, device="cuda").normal_(0.0, 1.0, generator=g).to(dtype)
    padded = torch.zeros(1, 304, dtype=dtype, device="cuda")[:, :H]
    padded.copy_(h)
    st = S.DppoStep(1, 1, 8, 1, 1.0, 1.0, V, "f32", 1)
    st.counts[3] = 1
    for quantize, score in ((S.quantize_f8, st.score_hidden_f8), (S.quantize_rows_i8, st.score_hidden_i8)):
        w, s = quantize(W)
        a, b = score(h, w, s, top_k=3), score(padded, w, s, top_k=3)
        assert torch.equal(a["top_ids"], b["top_ids"]) and torch.equal(a["lse"], b["lse"]) and int(st.status.item()) == 0
