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


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,V,d", [(1, 100, 64), (4, 700, 64), (8, 100, 64), (12, 700, 72), (40, 128, 65), (60, 3001, 64)])
def test_certain_rows(rows, V, d, dtype):
    """Labels 8 to 25 above every other logit, which are within 3 of one another: loss, dz at the label and dh are sums of the other
    columns' small terms and keep their relative accuracy.  Terms and their sums: below 2^-16 (the argument, up to 41, is rounded
    once, the constant is off by 2^-25 of it, the exponential by 2^-22).  bf16: roundings as in
    test_gradient_of_unlikely_columns; dh adds them up."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(rows + V + 1)
    margin = (32 + (torch.arange(rows, device="cuda") * 68) // max(1, rows - 1)).double()[:, None] / 4
    z = -margin - _quarters(g, 0, 3, rows, V)
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda")
    z.scatter_(1, labels[:, None], 0.0)
    z += _quarters(g, 0, 16, rows, 1)                              # log-sum-exps away from zero
    h, W, y, dz, others, total = _case(z, labels, dtype, d)
    want = torch.log1p(others / (total - others))
    for out in (b.vocab_loss(h, W, y), b.vocab_loss_grad(h, W, y, scale=float(rows))):
        assert bool(((out[1][0].double() - want).abs() <= 2.0 ** -16 * want).all()), (out[1][0], want)
        assert abs(float(out[0]) - float(want.mean())) <= 2.0 ** -15 * float(want.mean())
    one = 2.0 ** -11 + 2.0 ** -8 + 2.0 ** -14 if dtype == "bf16" else 2.0 ** -15
    end = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    got = out[4][0, :, :rows].T.double()
    assert bool(((got - dz).abs() <= (one * 1.01 + end) * dz.abs()).all()), float(((got - dz) / dz).abs().max())
    w64 = W[0].double()
    ref, size = dz @ w64, dz.abs() @ w64.abs()
    assert bool(((out[3][0].double() - ref).abs() <= (one + 2.0 ** -14) * size + end * ref.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 20])
def test_labels_of_infinite_logits(rows, dtype):
    """A label with a logit of -inf has an infinite loss and dz -1; beside columns of -inf a label alone has loss 0.  (fp32 counts
    infinities as 3.39e38.)"""
    import torch
    from paper_1810_08313_b200 import binding as b
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    h = torch.ones(1, rows, 64, device="cuda", dtype=dt)
    h[..., 1:] = 0.0
    W = torch.zeros(1, 300, 64, device="cuda", dtype=dt)
    W[0, 7, 0] = float("-inf")
    y = torch.full((1, rows), 7, device="cuda", dtype=torch.int32)
    y[0, 0] = 9
    loss, rl, lse, _, _ = b.vocab_loss_grad(h, W, y)
    assert bool((rl[0, 1:] > 3e38).all()) and abs(float(rl[0, 0]) - 5.7004436) < 1e-5       # log 299
    assert bool(((lse - 5.7004436).abs() < 1e-5).all())
    W[0, :, 0] = float("-inf")
    W[0, 9, 0] = 2.0
    y.fill_(9)
    loss, rl, lse, _, dW = b.vocab_loss_grad(h, W, y)
    assert float(loss) == 0.0 and float(rl.abs().max()) == 0.0 and bool((lse == 2.0).all())
    assert float(dW[0, 9].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 12, 70])
def test_rows_of_nan_keep_to_themselves(rows, dtype):
    """A labelled row that is NaN makes its own losses, dh and the mean NaN; the other rows keep their bits.  dW, a sum over the
    rows, is NaN where that row enters."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(rows)
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    h = torch.randn(1, rows, 64, generator=g, device="cuda").to(dt)
    W = (torch.randn(1, 400, 64, generator=g, device="cuda") / 8).to(dt)
    y = torch.randint(0, 400, (1, rows), generator=g, device="cuda").int()
    ref = b.vocab_loss_grad(h, W, y)
    bad = h.clone()
    bad[0, 1, 5] = float("nan")
    got = b.vocab_loss_grad(bad, W, y)
    keep = [i for i in range(rows) if i != 1]
    for k in (1, 2, 3):
        assert torch.equal(got[k][0, keep], ref[k][0, keep]) and bool(got[k][0, 1].isnan().all())
    assert bool(got[0].isnan().all()) and bool(got[4].isnan().all())


@pytest.mark.parametrize("rows", [1, 2, 4])
@pytest.mark.parametrize("d", [4096, 2000, 385])
def test_label_logits_of_few_rows(rows, d):
    """Long sums of equal signs at the label, zeros elsewhere: with a handful of bf16 rows nothing averages the losses, so the
    label's logit must not carry the truncation of the tensor core.  The other columns' sum is exact but for one exponential
    (2^-22); the label's argument is rounded near zero; a logarithm and the result: 2^-20 of the loss in all."""
    import torch
    from paper_1810_08313_b200 import binding as b
    V, m = 20001, 2
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    h = torch.randn(m, rows, d, generator=g, device="cuda").abs().bfloat16()
    W = torch.zeros(m, V, d, device="cuda", dtype=torch.bfloat16)
    y = torch.stack([torch.randperm(V, generator=g, device="cuda")[:rows] for _ in range(m)])
    own = torch.rand(m, rows, d, generator=g, device="cuda") + 0.2
    own = (own / (own * h.float()).sum(-1, keepdim=True) * (9.5 + torch.rand(m, rows, 1, generator=g, device="cuda"))).bfloat16()
    for i in range(m):
        W[i, y[i]] = own[i]
    z = torch.einsum("mrd,mvd->mrv", h.double(), own.double())      # the rows' labels among one another
    zy = z.diagonal(dim1=1, dim2=2)
    top = z.max(-1).values
    # (a row's other columns: zeros, and the logits of the other rows' labels)
    others = (z - zy[..., None]).exp().sum(-1) - 1.0 + (V - rows) * torch.exp(-zy)
    want = torch.log1p(others)
    for out in (b.vocab_loss(h, W, y.int()), b.vocab_loss_grad(h, W, y.int())):
        if rows == 1:
            assert bool(((out[1].double() - want).abs() <= 2.0 ** -20 * want).all()), (out[1].double() - want) / want
        else:
            # (those logits are products of the tensor core: 2^-22 of them for each of its chunks' 16 MMAs, in their share)
            share = 1.0 - (V - rows) * torch.exp(-zy) / others
            tol = 2.0 ** -20 * want + 2.0 ** -18 * top * share
            assert bool(((out[1].double() - want).abs() <= tol).all()), (out[1].double() - want) / want
