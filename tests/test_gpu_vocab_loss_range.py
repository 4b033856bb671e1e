"""The cross entropy where probabilities span many orders of magnitude, against 64 bits.

Rows of h are unit vectors and entries of W multiples of 1/4 below 64 in size, so that every logit is an entry of W,
exact in bf16, and an entry of dW is one entry of dz, rounded."""
import pytest

pytestmark = pytest.mark.gpu


def _case(z, labels, dtype, d):
    """h, W, labels whose logits are z [rows][V], and dz in 64 bits (not divided by the number of rows)."""
    import torch
    rows, V = z.shape
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    h = torch.zeros(1, rows, d, device="cuda", dtype=dt)
    h[0, torch.arange(rows), torch.arange(rows)] = 1.0
    W = torch.zeros(1, V, d, device="cuda", dtype=dt)
    W[0, :, :rows] = z.T.to(dt)
    assert torch.equal(W[0, :, :rows].double(), z.T)
    at = labels.long()[:, None]
    e = (z - z.max(1, keepdim=True).values).exp()
    others = e.clone().scatter_(1, at, 0.0).sum(1, keepdim=True)
    total = others + e.gather(1, at)
    dz = (e / total).scatter_(1, at, -others / total)              # (1 - p of the label without a difference)
    return h, W, labels.int()[None], dz, others[:, 0], total[:, 0]


def _quarters(g, lo, hi, *shape):
    import torch
    return torch.randint(4 * lo, 4 * hi + 1, shape, generator=g, device="cuda").double() / 4


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,V,d", [(8, 100, 64), (8, 700, 72), (60, 128, 64), (60, 700, 65), (60, 3001, 64), (3, 300, 64)])
def test_gradient_of_unlikely_columns(rows, V, d, dtype):
    """Logits up to 40 below the largest.  dz carries one rounding of the exponential (2^-11), one of itself (2^-8) and dW one more,
    relative to its size however small; exponentials and normalisers are below 2^-16 (the argument, up to 58, is rounded
    once: 2^-19).  1 / rows and its product with the scale: 2^-23.  In fp32: the argument's rounding, at most 2^-18."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(rows + V)
    z = _quarters(g, -40, 0, rows, V)
    z[:, torch.randint(0, V, (rows,), generator=g, device="cuda")] = 0.0
    z[:, V - 1] = -40.0
    labels = torch.randint(0, V - 1, (rows,), generator=g, device="cuda")
    h, W, y, dz, _, _ = _case(z, labels, dtype, d)
    got = b.vocab_loss_grad(h, W, y, scale=float(rows))[4][0, :, :rows].T.double()
    tol = (2.0 ** -11 + 2 * 2.0 ** -8 + 2.0 ** -14 if dtype == "bf16" else 2.0 ** -17) * dz.abs()
    # (a label's own entry, 1 - p, is a difference here: an absolute 2^-18)
    tol.scatter_add_(1, labels[:, None], torch.full((rows, 1), 2.0 ** -18, device="cuda", dtype=torch.float64))
    err = (got - dz).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    assert float(got[:, V - 1].abs().min()) > 0.0
