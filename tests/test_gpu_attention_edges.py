"""Attention where calls that the documentation allows go wrong most easily: boundaries without sense, values that are not finite."""
import pytest

pytestmark = pytest.mark.gpu


def _randn(seed, *shape, dtype="bfloat16"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(getattr(torch, dtype))


# ---- boundaries that do not ascend -----------------------------------------------------------------------------------

def _first_block(cuts, row):
    """The block of 128 keys at which a tile of rows from `row` on starts: its sequence is the one behind the last of as many
    boundaries as are not above the row."""
    s = sum(c <= row for c in cuts) - 1
    return max(cuts[max(s, 0)], 0) // 128


# descending at places where the second tile of a pair of 128 rows starts at an earlier key than the first
DESCENDING = [([0, 300, 10, 600], 256), ([0, 250, 300, 20, 1000], 256), ([300, 0, 10, 200, 20, 900], 256)]


@pytest.mark.parametrize("dtype,hd", [("bfloat16", 128), ("bfloat16", 72), ("bfloat16", 64), ("float32", 128), ("bfloat16", 136)])
@pytest.mark.parametrize("cuts,row", DESCENDING)
def test_descending_boundaries_end_every_wait(cuts, row, dtype, hd):
    """Some result in every row of its own, and no wait that runs out."""
    import torch
    from paper_1810_08313_b200 import binding as b
    assert _first_block(cuts, row + 128) < _first_block(cuts, row) <= row // 128
    tokens = cuts[-1]
    q, k, v = _randn(1, 1, tokens, 4, hd, dtype=dtype), _randn(2, 1, tokens, 2, hd, dtype=dtype), _randn(3, 1, tokens, 2, hd, dtype=dtype)
    seq = torch.tensor([cuts], dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 77.0), torch.full((1, 4, tokens), 77.0, device="cuda")
    b.attention(q, k, v, seq, out=out, lse=lse)
    b.device_status()
    assert not bool((out == 77.0).all(-1).any()) and not bool((lse == 77.0).any())
    # (a negative mark: dv of dout = 1 is a sum of probabilities, the same in every column, and may be 77)
    grads = [torch.full_like(t, -55.0) for t in (q, k, v)]
    b.attention_grad(torch.ones_like(q), q, k, v, out, lse, seq, dq=grads[0], dk=grads[1], dv=grads[2])
    b.device_status()
    assert not any(bool((t == -55.0).all(-1).any()) for t in grads)
