"""Sizes that the wrappers of attention and head norm hand on to the library: none at all, and ones beyond a C int."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [2, 1])
def test_heads_of_no_elements_are_refused(heads):
    """By the wrapper (as tensors whose heads are not dense) or by the library."""
    import torch
    from paper_1810_08313_b200 import binding as b
    q, lse = torch.zeros(1, 4, heads, 0, device="cuda"), torch.zeros(1, heads, 4, device="cuda")
    w, pos, f = torch.ones(1, 0, device="cuda"), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), b.rope_frequencies(0)
    for call in (lambda: b.attention(q, q, q), lambda: b.attention(q, q, q, scale=1.0), lambda: b.attention_grad(q, q, q, q, q, lse),
                 lambda: b.qk_norm_rope(q, q, w, w, pos, f), lambda: b.qk_norm_rope_grad(q, q, q, q, w, w, pos, f)):
        with pytest.raises((ValueError, b.LsError)):
            call()


def test_counts_beyond_a_c_int_are_refused():
    """2^32 + 1 sequences are not one, nor 2^31 + 4 frequencies four.  (Tables that nothing reads: their sizes count.)"""
    import torch
    from paper_1810_08313_b200 import binding as b
    q, lse = torch.zeros(1, 4, 2, 8, device="cuda"), torch.zeros(1, 2, 4, device="cuda")
    seq = torch.empty(1, 2 ** 32 + 2, dtype=torch.int32, device="cuda")
    for call in (lambda: b.attention(q, q, q, seq), lambda: b.attention_grad(q, q, q, q, q, lse, seq)):
        with pytest.raises(b.LsError) as e:
            call()
        assert e.value.code == b.LS_ERR_TOO_LARGE
    del seq
    w, pos = torch.ones(1, 8, device="cuda"), torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    f = torch.empty(2 ** 31 + 4, dtype=torch.float64, device="cuda")
    for call in (lambda: b.qk_norm_rope(q, q, w, w, pos, f), lambda: b.qk_norm_rope_grad(q, q, q, q, w, w, pos, f)):
        with pytest.raises(b.LsError) as e:
            call()
        assert e.value.code == b.LS_ERR_TOO_LARGE
