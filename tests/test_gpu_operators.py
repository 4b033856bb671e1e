"""Layer norm, the large-vocabulary cross entropy and the orthogonalised momentum step against 64-bit definitions.

Tolerances are elementwise bounds computed beside the reference from the roundings the kernels make (u = 2^-24, half a
step of fp32; 2^-8 relative for bf16 outputs; a tensor-core chunk of at most 64 MMAs whose accumulator truncates, at
most 2^-22 of the absolute sum each, counted below as MMA)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MMA = 2.0 ** -22
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _t(dtype):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _within(got, want, tol, what=""):
    import torch
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    if bool(bad.any()):
        i = int(torch.argmax((err / tol.clamp(min=1e-300)).nan_to_num(float("inf")).flatten()))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst at {i}: got "
                             f"{float(got.flatten()[i])}, want {float(want.flatten()[i])}, tolerance {float(tol.flatten()[i])}")


# ---- layer norm ----------------------------------------------------------------------------------------------------

def _ln_case(m, rows, d, dtype, seed=0, offset=0.3):
    g = _gen(seed)
    x = (_randn(g, m, rows, d) * (0.5 + _randn(g, m, 1, d).abs()) + offset).to(_t(dtype))
    w, bias = 1.0 + 0.2 * _randn(g, m, d), 0.3 * _randn(g, m, d)
    dy = _randn(g, m, rows, d).to(_t(dtype))
    return x, w, bias, dy


def _ln_stats(x, eps):
    x = x.double()
    mean = x.mean(-1)
    return mean, 1.0 / ((x - mean[..., None]).square().mean(-1) + eps).sqrt()


# A sum over a row is at most 32 additions in a thread, five over a warp and 32 over warps: 69 roundings of the absolute sum.
SUM = 72 * U


def _ln_check(x, w, bias, out, eps, dtype):
    y, mean, rstd = out
    m64, r64 = _ln_stats(x, eps)
    x64 = x.double()
    big = x64.abs().mean(-1)                                          # the mean's absolute sum
    tol_mean = SUM * big + U * m64.abs()
    _within(mean, m64, tol_mean + 1e-300, "mean")
    # var = mean square of c = x - mean: c is off by tol_mean + U |c|, its square and their sum round as well
    c = (x64 - m64[..., None]).abs()
    var = 1.0 / (r64 * r64)
    dvar = (2 * c * (tol_mean[..., None] + U * c) + tol_mean[..., None] ** 2).mean(-1) + (SUM + 4 * U) * var
    tol_r = r64 * (0.5 * dvar / var * 1.01 + 4 * U)
    _within(rstd, r64, tol_r, "rstd")
    xhat = c * r64[..., None]
    tol = (w.double()[:, None].abs() * (r64[..., None] * (tol_mean[..., None] + U * c) + c * tol_r[..., None] + 4 * U * xhat))
    y64 = (x64 - m64[..., None]) * r64[..., None] * w.double()[:, None]
    if bias is not None:
        y64 = y64 + bias.double()[:, None]
    _within(y, y64, tol * 1.02 + (2 * U + HALF[dtype]) * y64.abs() + 1e-300, "y")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,rows,d", [(1, 1, 1), (2, 3, 7), (3, 5, 8), (1, 16, 512), (2, 33, 513), (1, 70, 1024), (3, 9, 1001),
                                      (1, 17, 2048), (2, 5, 2056), (1, 6, 4096), (1, 5, 8192), (1, 3, 8200), (1, 4, 16384)])
def test_layer_norm(m, rows, d, dtype):
    from paper_1810_08313_b200 import binding as b
    x, w, bias, _ = _ln_case(m, rows, d, dtype, seed=rows * d)
    out = b.layer_norm(x, w, bias, eps=1e-5)
    _ln_check(x, w, bias, out, 1e-5, dtype)
    _ln_check(x, w, None, b.layer_norm(x, w, eps=1e-3), 1e-3, dtype)


def _ln_grad_check(x, w, dy, mean, rstd, got, dtype):
    dx, dw, db = got
    x64, d64, w64 = x.double(), dy.double(), w.double()[:, None]
    m64, r64 = mean.double()[..., None], rstd.double()[..., None]     # as given: the gradient of the kernel's own inputs
    xhat = (x64 - m64) * r64
    tx = 3 * U * xhat.abs()                                            # of xhat: a difference and a product
    t = d64 * w64
    a, bm = t.mean(-1, keepdim=True), (t * xhat).mean(-1, keepdim=True)
    ta = (SUM + 2 * U) * t.abs().mean(-1, keepdim=True)
    tb = (SUM + 4 * U) * (t * xhat).abs().mean(-1, keepdim=True) + (t.abs() * tx).mean(-1, keepdim=True)
    dx64 = r64 * (t - a - xhat * bm)
    terms = t.abs() + a.abs() + (xhat * bm).abs()
    tol = r64 * (ta + xhat.abs() * tb + tx * bm.abs() + 5 * U * terms)
    _within(dx, dx64, tol * 1.02 + HALF[dtype] * dx64.abs() + 1e-300, "dx")
    # sums over rows: at most rows additions in a thread, then parts and slices
    k = (min(x.shape[1], 400) + 64) * U
    if x.shape[1] > 400:
        k = (x.shape[1] / 100 + 400) * U                               # a CTA of the grid takes every gridDim-th row
    dw64, db64 = (d64 * xhat).sum(1), d64.sum(1)
    _within(dw, dw64, k * (d64 * xhat).abs().sum(1) + (d64.abs() * tx).sum(1) + 1e-300, "dweight")
    _within(db, db64, k * d64.abs().sum(1) + 1e-300, "dbias")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,rows,d", [(1, 1, 1), (2, 3, 7), (1, 1, 16), (3, 50, 512), (2, 33, 513), (1, 700, 1024), (3, 9, 1001),
                                      (1, 1300, 2048), (2, 5, 2056), (1, 40, 4096), (1, 5, 8192), (1, 3, 8200), (1, 4, 16384)])
def test_layer_norm_grad(m, rows, d, dtype):
    from paper_1810_08313_b200 import binding as b
    x, w, _, dy = _ln_case(m, rows, d, dtype, seed=rows + d)
    _, mean, rstd = b.layer_norm(x, w)
    _ln_grad_check(x, w, dy, mean, rstd, b.layer_norm_grad(dy, x, w, mean, rstd), dtype)


def test_layer_norm_gradient_against_differences():
    """Directional central differences of the 64-bit loss sum(dy * layer_norm(x)).  Truncation: h^2 / 6 times a third
    derivative; with rows of unit variance and a direction of unit entries that stays below 100 h^2 sum|dy| = 1e-8 sum|dy|
    at h = 1e-5; the kernel's own roundings are below 1e-4 of the absolute terms (test_layer_norm_grad bounds them)."""
    import torch
    from paper_1810_08313_b200 import binding as b
    x, w, bias, dy = _ln_case(2, 11, 96, "fp32", seed=3)
    _, mean, rstd = b.layer_norm(x, w, bias)
    dx, dw, db = b.layer_norm_grad(dy, x, w, mean, rstd)
    g = _gen(9)

    def loss(x64, w64, b64):
        m64, r64 = _ln_stats(x64, 1e-5)
        return float((dy.double() * ((x64 - m64[..., None]) * r64[..., None] * w64[:, None] + b64[:, None])).sum())

    X, W, B = x.double(), w.double(), bias.double()
    h = 1e-5
    for grad, base, put in ((dx, X, lambda v: (v, W, B)), (dw, W, lambda v: (X, v, B)), (db, B, lambda v: (X, W, v))):
        dirn = torch.sign(_randn(g, *base.shape)).double()
        num = (loss(*put(base + h * dirn)) - loss(*put(base - h * dirn))) / (2 * h)
        ana = float((grad.double() * dirn).sum())
        scale = float(grad.double().abs().sum()) + float(dy.double().abs().sum())
        assert abs(num - ana) <= 1e-5 * scale, (num, ana, scale)


def test_layer_norm_without_rows():
    import torch
    from paper_1810_08313_b200 import binding as b
    x = torch.empty(2, 0, 24, device="cuda")
    w = torch.ones(2, 24, device="cuda")
    y, mean, rstd = b.layer_norm(x, w)
    assert y.shape == (2, 0, 24) and mean.shape == (2, 0)
    dw = torch.full((2, 24), 7.0, device="cuda")
    db = torch.full((2, 24), 7.0, device="cuda")
    b.layer_norm_grad(x, x, w, mean, rstd, dweight=dw, dbias=db)
    assert float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_layer_norm_special_rows(dtype):
    """A constant row has no variance: y is the bias (eps > 0).  NaN and infinite rows stay their own: the others are
    the bits they are without them."""
    import torch
    from paper_1810_08313_b200 import binding as b
    x, w, bias, dy = _ln_case(1, 6, 264, dtype, seed=5)
    x[0, 2] = 1.5
    y, mean, rstd = b.layer_norm(x, w, bias)
    assert torch.equal(y[0, 2], bias[0].to(y.dtype)) and float(mean[0, 2]) == 1.5
    assert abs(float(rstd[0, 2]) - 1e-5 ** -0.5) < 1e-4 * 1e-5 ** -0.5
    z = x.clone()
    z[0, 1, 7], z[0, 4, 3] = float("nan"), float("inf")
    y2, _, _ = b.layer_norm(z, w, bias)
    keep = [0, 2, 3, 5]
    assert torch.equal(y2[0, keep], y[0, keep])
    assert bool(y2[0, 1].isnan().all()) and bool(y2[0, 4].isnan().any())


def test_layer_norm_strides_alignment_and_padding():
    """Parameters that are views into packed replica vectors, activations with a gap between replicas and an odd start;
    what lies between the replicas is left alone."""
    import torch
    from paper_1810_08313_b200 import binding as b
    for dtype, off in (("fp32", 0), ("fp32", 1), ("bf16", 1), ("bf16", 8)):
        m, rows, d = 3, 10, 264
        x, w, bias, dy = _ln_case(m, rows, d, dtype, seed=6)
        pack = torch.zeros(m, 4096, device="cuda")
        pack[:, 100:100 + d], pack[:, 1000:1000 + d] = w, bias
        gap = rows * d + 24
        buf = torch.full((m * gap + 16,), 3.0, device="cuda", dtype=_t(dtype))
        xs = torch.as_strided(buf, (m, rows, d), (gap, d, 1), off)
        xs.copy_(x)
        before = buf.clone()
        wv, bv = pack[:, 100:100 + d], pack[:, 1000:1000 + d]
        _ln_check(x, w, bias, b.layer_norm(xs, wv, bv), 1e-5, dtype)
        out = torch.full((m * gap + 16,), 5.0, device="cuda", dtype=_t(dtype))
        ov = torch.as_strided(out, (m, rows, d), (gap, d, 1), off)
        _, mean, rstd = b.layer_norm(xs, wv, bv, out=ov)
        assert torch.equal(buf, before)
        gpack = torch.full((m, 4096), 9.0, device="cuda")
        dxb = torch.full_like(out, 5.0)
        dxv = torch.as_strided(dxb, (m, rows, d), (gap, d, 1), off)
        dwv, dbv = gpack[:, 100:100 + d], gpack[:, 1000:1000 + d]
        b.layer_norm_grad(dy, xs, wv, mean, rstd, dx=dxv, dweight=dwv, dbias=dbv)
        _ln_grad_check(x, w, dy, mean, rstd, (dxv, dwv, dbv), dtype)
        for t in (out, dxb):
            flat = torch.ones_like(t, dtype=torch.bool)
            torch.as_strided(flat, (m, rows, d), (gap, d, 1), off).fill_(False)
            assert bool((t[flat] == 5.0).all())
        gpack[:, 100:100 + d] = 9.0
        gpack[:, 1000:1000 + d] = 9.0
        assert bool((gpack == 9.0).all())


def test_layer_norm_offsets_beyond_32_bits():
    """More than 2^31 elements: the last rows are those of a call of their own."""
    import torch
    from paper_1810_08313_b200 import binding as b
    d, rows = 4096, 2 ** 19 + 37
    x = torch.zeros(rows, d, device="cuda", dtype=torch.bfloat16)
    g = _gen(8)
    tail = _randn(g, 40, d).to(torch.bfloat16)
    x[-40:] = tail
    w = 1.0 + 0.1 * _randn(g, d)
    y, mean, rstd = b.layer_norm(x, w)
    y2, mean2, rstd2 = b.layer_norm(tail, w)
    assert torch.equal(y[-40:], y2) and torch.equal(mean[-40:], mean2) and torch.equal(rstd[-40:], rstd2)
    dx, dw, db = b.layer_norm_grad(x, x, w, mean, rstd)
    dx2, _, _ = b.layer_norm_grad(tail, tail, w, mean2, rstd2)
    assert torch.equal(dx[-40:], dx2)
    del x, y, dx


# ---- cross entropy -------------------------------------------------------------------------------------------------

def _ce_case(m, rows, d, V, dtype, seed=0, sure=8.0, ignored=0.1):
    import torch
    g = _gen(seed)
    W = (_randn(g, m, V, d) / math.sqrt(d)).to(_t(dtype))
    y = torch.randint(0, V, (m, rows), generator=g, device="cuda")
    own = torch.stack([W[i][y[i]] for i in range(m)]).float()
    h = (_randn(g, m, rows, d) + sure * torch.rand((m, rows, 1), generator=g, device="cuda") * own).to(_t(dtype))
    drop = torch.rand((m, rows), generator=g, device="cuda") < ignored
    return h, W, torch.where(drop, -1, y).int()


def _ce_check(h, W, labels, out, dtype, scale=1.0, grad=True):
    """Elementwise bounds: dz of the logits from their absolute sums; lse is at most that plus the exponentials' 2^-21;
    the probabilities are rounded to fp16 (2^-11 relative, 2^-25 of the slice's largest absolute) and bf16 (2^-8); sums as
    for the logits; one rounding of the output."""
    import torch
    for i in range(h.shape[0]):
        h64, W64, y = h[i].double(), W[i].double(), labels[i].long()
        V, d = W64.shape
        keep = (y >= 0) & (y < V)
        n = max(1, int(keep.sum()))
        z = h64 @ W64.T
        tz = MMA * (64 + d / 64) * (h64.abs() @ W64.abs().T)
        top = tz.max(1).values
        lse = torch.logsumexp(z, 1)
        tl = top + 2.0 ** -20 * (2 + lse.abs())
        _within(out[2][i], lse, tl, "lse")
        idx = y.clamp(0, V - 1)[:, None]
        rl = torch.where(keep, lse - z.gather(1, idx)[:, 0], 0.0)
        trl = torch.where(keep, tl + top + 2 * U * rl.abs(), 0.0)
        _within(out[1][i], rl, trl + 1e-300, "row_loss")
        want = rl.sum() / n
        _within(out[0][i], want, trl.sum() / n + 2 * U * want.abs() + 1e-300, "loss")
        if not grad:
            continue
        p = torch.exp(z - lse[:, None])
        dz = p.clone()
        dz.scatter_add_(1, idx, torch.full_like(lse, -1.0)[:, None])
        dz[~keep] = 0.0
        rel = (top + tl)[:, None] + 2.0 ** -20
        tdz = p * (rel * 1.1 + (2.0 ** -11 if dtype == "bf16" else 0.0)) + (2.0 ** -25 if dtype == "bf16" else 0.0)
        # the label's entry comes from expm1: off by p times the logits' error
        tdz = tdz + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * dz.abs()
        tdz[~keep] = 0.0
        for got, a, ta, o in ((out[3][i], dz, tdz, W64), (out[4][i], dz.T, tdz.T, h64 * keep[:, None])):
            k = a.shape[1]
            want = scale / n * (a @ o)
            tol = abs(scale) / n * (ta @ o.abs() + MMA * (64 + k / 64) * (a.abs() @ o.abs()))
            _within(got, want, tol * 1.02 + (HALF[dtype] + 4 * U) * want.abs() + 1e-38, "gradient")


SHAPES = [(1, 1, 8, 3), (1, 1, 1, 1), (2, 3, 5, 7), (1, 256, 64, 256), (1, 257, 72, 259), (2, 65, 200, 777), (1, 40, 129, 1000),
          (1, 300, 130, 515), (1, 33, 1024, 2049), (1, 700, 512, 3000), (3, 20, 96, 130)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,rows,d,V", SHAPES)
def test_vocab_loss_and_gradient(m, rows, d, V, dtype):
    from paper_1810_08313_b200 import binding as b
    h, W, y = _ce_case(m, rows, d, V, dtype, seed=rows + V)
    _ce_check(h, W, y, b.vocab_loss(h, W, y), dtype, grad=False)
    _ce_check(h, W, y, b.vocab_loss_grad(h, W, y, scale=1.7), dtype, scale=1.7)


@pytest.mark.parametrize("rows", [7, 16, 17, 31, 33, 64, 65, 127, 129, 191, 193, 255])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_vocab_loss_every_count_of_boxes(rows, dtype):
    """Row counts whose tiles are filled by one to four boxes, whole and partial, and label-less rows at the end of each."""
    from paper_1810_08313_b200 import binding as b
    h, W, y = _ce_case(1, rows, 72, 300, dtype, seed=rows)
    y[:, -1] = -1
    _ce_check(h, W, y, b.vocab_loss(h, W, y), dtype, grad=False)
    _ce_check(h, W, y, b.vocab_loss_grad(h, W, y), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,rows,d,V", [(1, 1, 8, 130), (2, 4, 136, 1000), (3, 4, 264, 257), (2, 5, 520, 700), (2, 9, 132, 385),
                                        (1, 16, 1000, 129), (2, 17, 260, 500), (1, 32, 77, 1025)])
def test_vocab_loss_few_rows(m, rows, d, V, dtype):
    """Row counts on both sides of every limit for few rows, several replicas; a row without a label may hold anything."""
    import torch
    from paper_1810_08313_b200 import binding as b
    h, W, y = _ce_case(m, rows, d, V, dtype, seed=rows + d)
    _ce_check(h, W, y, b.vocab_loss(h, W, y), dtype, grad=False)
    _ce_check(h, W, y, b.vocab_loss_grad(h, W, y, scale=0.7), dtype, scale=0.7)
    y2 = y.clone()
    y2[:, -1] = V
    clean = b.vocab_loss_grad(h, W, y2)
    h2 = h.clone()
    h2[:, -1] = float("nan")
    for i, (got, want) in enumerate(zip(b.vocab_loss_grad(h2, W, y2), clean)):
        if i == 2:
            got, want = got[:, :-1], want[:, :-1]          # lse of the row itself is NaN
        assert torch.equal(got, want)
    assert float(clean[3][:, -1].abs().max()) == 0.0
    b.device_status()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_vocab_loss_labels_that_do_not_count(dtype):
    """Rows without a label (negative or beyond the vocabulary) have no loss and no gradient, and whatever their h holds
    stays out of dW; a call without any label has loss 0 and zero gradients."""
    import torch
    from paper_1810_08313_b200 import binding as b
    h, W, y = _ce_case(1, 50, 64, 300, dtype, seed=4, ignored=0.0)
    y[0, 7], y[0, 20], y[0, 49] = -100, 300, 2 ** 31 - 1
    ref = b.vocab_loss_grad(h, W, y)
    _ce_check(h, W, y, ref, dtype)
    bad = h.clone()
    bad[0, 7], bad[0, 20], bad[0, 49] = float("nan"), float("inf"), -3e38
    got = b.vocab_loss_grad(bad, W, y)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert torch.equal(got[3], ref[3]) and torch.equal(got[4], ref[4])
    assert float(got[3][0, [7, 20, 49]].abs().max()) == 0.0
    y.fill_(-1)
    got = b.vocab_loss_grad(h, W, y)
    assert float(got[0]) == 0.0 and float(got[1].abs().max()) == 0.0
    assert float(got[3].abs().max()) == 0.0 and float(got[4].abs().max()) == 0.0


def test_vocab_loss_without_rows():
    import torch
    from paper_1810_08313_b200 import binding as b
    h = torch.empty(2, 0, 16, device="cuda", dtype=torch.bfloat16)
    W = torch.ones(2, 9, 16, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(2, 0, device="cuda", dtype=torch.int32)
    dW = torch.full_like(W, 3.0)
    loss, rl, lse, dh, _ = b.vocab_loss_grad(h, W, y, dW=dW)
    assert loss.tolist() == [0.0, 0.0] and rl.shape == (2, 0) and dh.shape == h.shape and float(dW.abs().max()) == 0.0
    assert b.vocab_loss(h, W, y)[0].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_vocab_loss_extreme_logits(dtype):
    """Logits of hundreds and logits of -inf: the maximum carries the sum.  Rows are one-hot so that logits are entries
    of W exactly."""
    import torch
    from paper_1810_08313_b200 import binding as b
    d, V = 16, 700
    W = torch.zeros(1, V, d, device="cuda")
    W[0, :, 0] = torch.linspace(-500, 500, V, device="cuda").round()
    W[0, :, 1] = -3.0e4
    W[0, 5, 1] = 2.0
    W[0, 300:, 2] = float("-inf")            # whole slices of -inf, and the ragged end
    W[0, 3, 2] = 1.0
    h = torch.zeros(1, 4, d, device="cuda")
    h[0, 0, 0] = 1.0
    h[0, 1, 1] = 1.0
    h[0, 2, 0] = 0.25
    h, W = h.to(_t(dtype)), W.to(_t(dtype))
    # row 2 multiplies column 2 (with its infinities) by zero, which is NaN in every form; only rows 0, 1 without column 2
    Wf = W.clone()
    Wf[0, :, 2] = 0.0
    y = torch.tensor([[V - 1, 5, 0, -1]], device="cuda", dtype=torch.int32)
    _ce_check(h, Wf, y, b.vocab_loss_grad(h, Wf, y), dtype)
    one = torch.ones(1, 1, 8, device="cuda").to(_t(dtype))
    Wi = torch.zeros(1, 400, 8, device="cuda").to(_t(dtype))
    Wi[0, 128:, 0] = float("-inf")
    loss, rl, lse = b.vocab_loss(one, Wi, torch.zeros(1, 1, device="cuda", dtype=torch.int32))
    assert abs(float(lse) - math.log(128.0)) < 1e-5 and abs(float(loss) - math.log(128.0)) < 1e-5


@pytest.mark.parametrize("rows", [8, 200])
def test_vocab_loss_fp32_probabilities_of_large_logits(rows):
    """Exact logits around a log-sum-exp of 100: the probabilities must not carry the rounding of that number (2^-18), only
    that of differences.  p = 2^t / S, t = (z - max) log2(e): t is off by 2^-24 |t| and by the constant's 2^-26 |t|, which
    p turns into ln 2 of that; exp2 of p and of the terms of S, the division, the sums and the products with h = 1 are below
    2^-20 together."""
    import torch
    from paper_1810_08313_b200 import binding as b
    d, V = 256, 700
    g = _gen(rows)
    h = torch.zeros(1, rows, d, device="cuda")
    h[0, torch.arange(rows), torch.arange(rows)] = 1.0
    W = (torch.randint(60 * 64, 100 * 64, (1, V, d), generator=g, device="cuda") / 64).float()
    labels = torch.randint(0, V, (1, rows), generator=g, device="cuda", dtype=torch.int32)
    _, _, _, dh, dW = b.vocab_loss_grad(h, W, labels, scale=float(rows))
    z = W[0, :, :rows].double().T
    p = torch.softmax(z, -1)
    t = z.max(-1, keepdim=True)[0] - z
    want = p - torch.nn.functional.one_hot(labels[0].long(), V).double()
    # 1 / rows is rounded, too, and its product with the scale
    _within(dW[0, :, :rows].T, want, (2.0 ** -20 + 2.0 ** -23 * t) * p + 4 * U * want.abs() + 1e-37, "dW")
    assert float(dW[0, :, rows:].abs().max()) == 0.0


def test_vocab_loss_gradient_against_differences():
    """Central differences of the 64-bit mean loss.  h = 1e-4 along directions of unit entries: truncation below
    h^2 (sum|dir W|)^3-scaled third derivatives of a softmax, under 1e-6 of the loss scale here; the kernel's fp32 gradient is
    bounded elementwise in test_vocab_loss_and_gradient."""
    import torch
    from paper_1810_08313_b200 import binding as b
    h, W, y = _ce_case(1, 24, 40, 90, "fp32", seed=2, ignored=0.2)
    _, _, _, dh, dW = b.vocab_loss_grad(h, W, y)
    keep = y[0] >= 0

    def loss(h64, W64):
        z = h64 @ W64.T
        return float((torch.logsumexp(z, 1) - z.gather(1, y[0].long().clamp(min=0)[:, None])[:, 0])[keep].mean())

    H, Wd = h[0].double(), W[0].double()
    g = _gen(3)
    for grad, base, put in ((dh[0], H, lambda v: (v, Wd)), (dW[0], Wd, lambda v: (H, v))):
        dirn = _randn(g, *base.shape).double() / math.sqrt(base.shape[1])
        num = (loss(*put(base + 1e-4 * dirn)) - loss(*put(base - 1e-4 * dirn))) / 2e-4
        ana = float((grad.double() * dirn).sum())
        assert abs(num - ana) <= 1e-5 * (1.0 + float((grad.double() * dirn).abs().sum())), (num, ana)


@pytest.mark.parametrize("dtype,d", [("bf16", 96), ("bf16", 97), ("fp32", 96), ("fp32", 33)])
def test_vocab_loss_strides_and_padding(dtype, d):
    """Replicas apart from each other; what lies between them is left alone."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, rows, V = 2, 37, 301
    h, W, y = _ce_case(m, rows, d, V, dtype, seed=11)
    gh, gw = rows * d + 64, V * d + 128
    if d % 8:
        gh, gw = gh + 3, gw + 5

    def spread(t, gap, fill):
        buf = torch.full((m * gap,), fill, device="cuda", dtype=_t(dtype))
        v = torch.as_strided(buf, (m,) + tuple(t), (gap, t[1], 1))
        return buf, v

    bh, hv = spread((rows, d), gh, 2.0)
    bw, wv = spread((V, d), gw, 2.0)
    hv.copy_(h)
    wv.copy_(W)
    bdh, dhv = spread((rows, d), gh, 5.0)
    bdw, dwv = spread((V, d), gw, 5.0)
    keep = bh.clone(), bw.clone()
    out = b.vocab_loss_grad(hv, wv, y, dh=dhv, dW=dwv)
    assert torch.equal(bh, keep[0]) and torch.equal(bw, keep[1])
    _ce_check(h, W, y, out, dtype)
    for buf, t, gap in ((bdh, (rows, d), gh), (bdw, (V, d), gw)):
        flat = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(flat, (m,) + t, (gap, t[1], 1)).fill_(False)
        assert bool((buf[flat] == 5.0).all())


@pytest.mark.parametrize("dtype,d,V", [("bf16", 64, 131072), ("fp32", 16, 131072), ("bf16", 65, 131072)])
def test_vocab_loss_rows_in_several_pieces(dtype, d, V):
    """So many rows that the probabilities are taken in pieces: the same losses and dh as calls of fewer rows (their sums
    over the vocabulary are the same), and dW within its bound, checked on sampled rows of the matrix."""
    import torch
    from paper_1810_08313_b200 import binding as b
    rows = 2 ** 29 // V + 300 if dtype == "bf16" else 2 ** 27 // V + 300
    h, W, y = _ce_case(1, rows, d, V, dtype, seed=12)
    loss, rl, lse, dh, dW = b.vocab_loss_grad(h, W, y)
    n = int((y >= 0).sum())
    at = torch.randint(0, V, (64,), generator=_gen(1), device="cuda")
    at[0], at[1] = V - 1, int(y[0, rows - 1].clamp(min=0))
    h64, W64 = h[0].double(), W[0].double()
    want, bound = torch.zeros(64, d, device="cuda", dtype=torch.float64), torch.zeros(64, d, device="cuda", dtype=torch.float64)
    for r in range(0, rows, 512):
        hh, yy = h64[r:r + 512], y[0, r:r + 512]
        l64 = torch.logsumexp(hh @ W64.T, 1)
        tl = MMA * 80 * float((hh.abs() @ W64[:2048].abs().T).max()) + 2.0 ** -20 * (2 + l64.abs())
        _within(lse[0, r:r + 512], l64, 4 * tl, "lse")
        p = torch.exp(hh @ W64[at].T - l64[:, None])
        dz = p - (at[None] == yy[:, None]).double()
        dz[yy < 0] = 0.0
        rel = 2.2 * tl[:, None]                          # of p: its logit and the log-sum-exp
        t = p * (2.0 ** -11 + rel) + 2.0 ** -25 + 2.0 ** -8 * dz.abs() if dtype == "bf16" else p * rel + 2.0 ** -22 * dz.abs()
        t[yy < 0] = 0.0
        hz = hh * (yy >= 0)[:, None]
        want += dz.T @ hz
        bound += t.T @ hz.abs() + MMA * 200 * (dz.abs().T @ hz.abs())
    _within(dW[0, at], want / n, bound / n * 1.02 + HALF[dtype] * want.abs() / n + 1e-38, "dW")
    few = b.vocab_loss_grad(h[:, -256:].contiguous(), W, y[:, -256:].contiguous())
    assert torch.equal(few[1], rl[:, -256:]) and torch.equal(few[2], lse[:, -256:])


def test_vocab_loss_matrix_beyond_32_bits():
    """W of more than 2^31 elements: the losses of a few rows, against 64-bit sums taken in parts."""
    import torch
    from paper_1810_08313_b200 import binding as b
    V, d = 2 ** 20 + 11, 2056
    W = torch.empty(V, d, device="cuda", dtype=torch.bfloat16)
    g = _gen(2)
    for v in range(0, V, 1 << 17):
        W[v:v + (1 << 17)] = (_randn(g, min(1 << 17, V - v), d) / math.sqrt(d)).to(torch.bfloat16)
    h = _randn(g, 5, d).to(torch.bfloat16)
    y = torch.tensor([0, V - 1, V // 2, -1, V - 1], device="cuda", dtype=torch.int32)
    loss, rl, lse = b.vocab_loss(h, W, y)
    z = torch.cat([h.double() @ W[v:v + (1 << 16)].double().T for v in range(0, V, 1 << 16)], 1)
    want = torch.logsumexp(z, 1)
    tol = MMA * (64 + d / 64) * float((h.double().abs() @ W[:4096].double().abs().T).max()) * 2 + 2.0 ** -20 * 20
    _within(lse, want, torch.full_like(want, tol), "lse")
    rows = [0, 1, 2, 4]
    _within(rl[rows], want[rows] - z[rows, y[rows].long()], torch.full((4,), 2 * tol, device="cuda", dtype=torch.float64), "row loss")
    assert float(rl[3]) == 0.0
    del W


# ---- orthogonalisation ---------------------------------------------------------------------------------------------

A, B, CC = 3.4445, -4.7750, 2.0315


def _ns_step64(x):
    """One Newton-Schulz step of x [n][k], n <= k, in 64 bits, and an elementwise bound of a kernel step's error:
    a product is off by K = 2^-22 (a chunk of 24 MMAs, the chunks' sums, and 2^-22 for each operand's pieces), a
    stored matrix by 2^-22 of its entries and 2^-25 over its scale."""
    import torch
    n, k = x.shape
    K = lambda length: MMA * (28 + length / 128)      # noqa: E731
    a = x @ x.T
    eye = torch.eye(n, device=x.device, dtype=torch.float64)
    c = B * eye + CC * a
    p = A * eye + a @ c
    ta = K(k) * (x.abs() @ x.abs().T) + MMA * a.abs() + 2.0 ** -25 / 8192
    tc = CC * ta + MMA * c.abs() + 2.0 ** -25 / 4096
    tp = ta @ c.abs() + a.abs() @ tc + K(n) * (a.abs() @ c.abs()) + MMA * p.abs() + 2.0 ** -25 / 8192
    out = p @ x
    scale = min(16384.0, 2.0 ** math.floor(0.5 * math.log2(n * k)))
    tol = tp @ x.abs() + K(n) * (p.abs() @ x.abs()) + MMA * out.abs() + 2.0 ** -25 / scale
    return out, tol


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 5), (16, 16), (40, 100), (256, 256), (300, 200), (130, 515), (257, 64)])
def test_orthogonalize_step_by_step(rows, cols):
    """Each step against a 64-bit step from the kernel's own previous result, elementwise."""
    import torch
    from paper_1810_08313_b200 import binding as b
    u = _randn(_gen(rows + cols), 1, rows, cols) * 1e-3
    flip = (lambda t: t.T) if rows > cols else (lambda t: t)
    u64 = flip(u[0].double())
    x = u64 / (torch.linalg.norm(u64) + 1e-7)
    start = 2 * MMA * x.abs()
    for s in range(1, 6):
        want, tol = _ns_step64(x)
        if s == 1:
            # the kernel's X_0 is rounded once more: an error e of X changes A by |e||X|^T twice and the product once
            n = x.shape[0]
            ea = start @ x.abs().T + x.abs() @ start.T
            tol = tol + ((ea @ (abs(B) + 2 * CC * (x.abs() @ x.abs().T))) @ x.abs()) + (A + abs(B) + CC) * start \
                + ((x.abs() @ x.abs().T) @ (abs(B) + CC * (x.abs() @ x.abs().T))) @ start
        got = flip(b.orthogonalize(u, steps=s)[0])
        # (the next step starts from pieces of 22 bits, of which the fp32 result is the sum)
        _within(got, want, tol * 1.05 + 2 * U * want.abs() + 1e-30, f"step {s}")
        x = got.double()
    sv = torch.linalg.svdvals(x)
    if min(rows, cols) <= 40:
        assert float(sv.max()) < 1.25


def _ns_group64(x, steps, start=None):
    """`steps` Newton-Schulz steps of x [n][k] in 64 bits, and an elementwise bound of the error of a kernel that forms
    their product Q from A = X X^T alone, A' = A P P, with the errors of _ns_step64.  start: the error of x."""
    import torch
    n, k = x.shape
    K = lambda length: MMA * (28 + length / 128)      # noqa: E731
    both = lambda t: torch.maximum(t, t.T)            # noqa: E731  (an element is computed on one side of the diagonal)

    def prod(l, tl, r, tr, scale):
        out = l @ r
        return out, both(tl @ r.abs() + l.abs() @ tr + K(n) * (l.abs() @ r.abs())) + MMA * out.abs() + 2.0 ** -25 / scale

    eye = torch.eye(n, device=x.device, dtype=torch.float64)
    a = x @ x.T
    ta = K(k) * (x.abs() @ x.abs().T) + MMA * a.abs() + 2.0 ** -25 / 8192
    if start is not None:
        ta = ta + start @ x.abs().T + x.abs() @ start.T
    q = tq = None
    for s in range(steps):
        c = B * eye + CC * a
        tc = CC * ta + MMA * c.abs() + 2.0 ** -25 / 4096
        p, tp = prod(a, ta, c, tc, 8192)
        p = p + A * eye
        tp = tp + MMA * A * eye
        if q is None:
            q, tq = p, tp
        else:
            q, tq = prod(p, tp, q, tq, 4096 if s == 1 else 1024)
        if s + 1 < steps:
            bb, tb = prod(a, ta, p, tp, 8192)
            a, ta = prod(bb, tb, p, tp, 8192)
    out = q @ x
    scale = min(16384.0, 2.0 ** math.floor(0.5 * math.log2(n * k)))
    tol = tq @ x.abs() + K(n) * (q.abs() @ x.abs()) + MMA * out.abs() + 2.0 ** -25 / scale
    if start is not None:
        tol = tol + q.abs() @ start
    return out, tol


@pytest.mark.parametrize("m,rows,cols", [(30, 257, 1000), (40, 900, 257), (2, 1000, 2501)])
def test_steps_from_bf16_taken_together(m, rows, cols):
    """Sizes at which steps from bf16 gradients are taken in groups (three first when their number is odd, else two): each group
    against 64 bits from the kernel's own result before it, elementwise.  W = 0, lr = 1 and no momentum give -O in fp32."""
    import torch
    from paper_1810_08313_b200 import binding as b
    u = (_randn(_gen(rows + cols), m, rows, cols) * 1e-3).to(torch.bfloat16)
    flip = (lambda t: t.T) if rows > cols else (lambda t: t)
    z = m - 1
    u64 = flip(u[z].double())
    factor = math.sqrt(max(1.0, rows / cols))
    got = {0: u64 / (torch.linalg.norm(u64) + 1e-7)}
    for before, steps in ((0, 1), (0, 2), (0, 3), (2, 4), (3, 5), (5, 7)):
        w, v = torch.zeros(m, rows, cols, device="cuda"), torch.zeros(m, rows, cols, device="cuda")
        b.muon_step(w, v, u, 1.0, momentum=0.0, nesterov=False, steps=steps)
        x = got[before]
        want, tol = _ns_group64(x, steps - before, 2 * MMA * x.abs() if before == 0 else None)
        # (the factor and its product with O are rounded, and the earlier result carries the same: three roundings more)
        got[steps] = flip(-w[z].double()) / factor
        _within(got[steps], want, tol * 1.05 + 8 * U * want.abs() + 1e-30, f"{before} to {steps} steps")
    # in bf16 the same result, rounded
    out = b.orthogonalize(u, steps=5)
    assert torch.equal(out, b.orthogonalize(u, steps=5))
    _within(flip(out[z].double()), got[5], 2.0 ** -8 * got[5].abs() + 1e-30, "bf16")
    b.device_status()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,rows,cols", [(3, 96, 160), (2, 513, 300), (1, 64, 1000)])
def test_orthogonalize_replicas_and_types(m, rows, cols, dtype):
    """Replicas of different magnitude are independent: each is the bits of a call of its own; bf16 input gives the rounding of the
    fp32 result of the same values."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = _gen(m * rows)
    u = (_randn(g, m, rows, cols) * torch.tensor([1.0, 1e-6, 1e4], device="cuda")[:m, None, None]).to(_t(dtype))
    out = b.orthogonalize(u)
    assert out.dtype == u.dtype
    full = b.orthogonalize(u.float())
    assert torch.equal(out, full.to(out.dtype))
    for i in range(m):
        # (one replica: a grid of its own, the partial sums of squares differ in the last bit of a double)
        one = b.orthogonalize(u[i].float())
        assert float((one - full[i]).abs().max()) <= 1e-5 * float(full[i].abs().max())
    o64 = full[0].double()
    gram = o64 @ o64.T if rows <= cols else o64.T @ o64
    ev = torch.linalg.eigvalsh(gram)
    assert 0.2 < float(ev.min()) and float(ev.max()) < 1.5


def test_orthogonalize_special_matrices():
    """A zero matrix stays zero; rank one is scaled to singular value about 1; a NaN fills its replica and leaves the others."""
    import torch
    from paper_1810_08313_b200 import binding as b
    u = torch.zeros(3, 48, 80, device="cuda")
    u[1] = torch.outer(torch.arange(1.0, 49.0, device="cuda"), torch.ones(80, device="cuda"))
    u[2] = _randn(_gen(1), 48, 80)
    ref = b.orthogonalize(u)
    assert float(ref[0].abs().max()) == 0.0
    s = torch.linalg.svdvals(ref[1].double())
    assert 0.6 < float(s[0]) < 1.25 and float(s[1]) < 1e-3
    v = u.clone()
    v[1, 3, 4] = float("nan")
    got = b.orthogonalize(v)
    assert bool(got[1].isnan().all()) and torch.equal(got[0], ref[0]) and torch.equal(got[2], ref[2])


@pytest.mark.parametrize("gdtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("m,rows,cols", [(1, 40, 70), (2, 130, 64)])
def test_muon_step(m, rows, cols, nesterov, gdtype):
    """v and w against their formulas with the kernel's own orthogonalisation of the same direction."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g0 = _gen(rows)
    w, v = _randn(g0, m, rows, cols), 0.1 * _randn(g0, m, rows, cols)
    g = (0.1 * _randn(g0, m, rows, cols)).to(_t(gdtype))
    w0, v0 = w.clone(), v.clone()
    lr, mu = 0.02, 0.95
    b.muon_step(w, v, g, lr=lr, momentum=mu, nesterov=nesterov)
    m32 = float(np.float32(mu))
    v64 = m32 * v0.double() + g.double()
    _within(v, v64, 2 * U * v64.abs() + 1e-300, "v")
    u32 = torch.addcmul(g.float(), torch.full_like(v, m32), v) if nesterov else v
    o = b.orthogonalize(u32)
    step = float(np.float32(lr)) * math.sqrt(max(1.0, rows / cols))
    w64 = w0.double() - step * o.double()
    # O of a direction rounded differently (2 u relative) moves by at most 4^5 of that in norm; entries by their largest
    tol = 4 * U * w64.abs() + step * (4 * U * o.double().abs() + 1024 * 2 * U * float(torch.linalg.norm(o[0].double())))
    _within(w, w64, tol, "w")


def test_muon_step_on_views_of_packed_replicas():
    """Matrices inside the packed parameter and momentum vectors of a handle; everything around them stays."""
    import torch
    from paper_1810_08313_b200 import binding as b
    eng = b.LocalSGD(3, (24, 40, 10), lr=0.1, momentum=0.9, batch=8)
    p, v = eng.state_view()
    g = _gen(1)
    p.copy_(_randn(g, *p.shape))
    v.copy_(0.1 * _randn(g, *v.shape))
    p0, v0 = p.clone(), v.clone()
    wv, vv = p[:, :960].unflatten(1, (40, 24)), v[:, :960].unflatten(1, (40, 24))
    grad = _randn(g, 3, 40, 24)
    w2, v2 = wv.contiguous().clone(), vv.contiguous().clone()
    b.muon_step(wv, vv, grad, lr=0.05)
    b.muon_step(w2, v2, grad, lr=0.05)
    assert torch.equal(wv, w2) and torch.equal(vv, v2)
    assert torch.equal(p[:, 960:], p0[:, 960:]) and torch.equal(v[:, 960:], v0[:, 960:])
    assert not torch.equal(p[:, :960], p0[:, :960])
    eng.close()


# ---- streams, graphs, refusals, use together -----------------------------------------------------------------------

def _everything(b, s):
    y, mean, rstd = b.layer_norm(s["x"], s["w"], s["bias"])
    loss, rl, lse, dh, dW = b.vocab_loss_grad(y.to(s["W"].dtype), s["W"], s["labels"])
    dx, dw, db = b.layer_norm_grad(dh.to(s["x"].dtype), s["x"], s["w"], mean, rstd)
    o = b.orthogonalize(dW)
    return y, mean, rstd, loss, rl, lse, dh, dW, dx, dw, db, o


def _inputs(seed, dtype="bf16"):
    import torch
    x, w, bias, _ = _ln_case(2, 150, 72, dtype, seed=seed)
    _, W, labels = _ce_case(2, 150, 72, 333, dtype, seed=seed)
    return {"x": x, "w": w, "bias": bias, "W": W, "labels": labels}


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_results_are_reproducible_on_any_stream_and_in_graphs(dtype):
    import torch
    from paper_1810_08313_b200 import binding as b
    s1, s2 = _inputs(1, dtype), _inputs(2, dtype)
    ref1, ref2 = [t.clone() for t in _everything(b, s1)], [t.clone() for t in _everything(b, s2)]
    for t, r in zip(_everything(b, s1), ref1):
        assert torch.equal(t, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _everything(b, s2)
    side.synchronize()
    for t, r in zip(got, ref2):
        assert torch.equal(t, r)
    # a stream handed over while another is current: the outputs belong to that stream
    y, mean, rstd = b.layer_norm(s1["x"], s1["w"], s1["bias"], stream=side)
    loss = b.vocab_loss(y, s1["W"], s1["labels"], stream=side)[0]
    side.synchronize()
    assert torch.equal(y, ref1[0]) and torch.equal(loss, b.vocab_loss(ref1[0], s1["W"], s1["labels"])[0])
    # two graphs, replayed in turn with other inputs
    static = {k: v.clone() for k, v in s1.items()}
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _everything(b, static)
        graphs.append((g, out))
    for src, ref in ((s2, ref2), (s1, ref1), (s2, ref2)):
        for k in static:
            static[k].copy_(src[k])
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for t, r in zip(out, ref):
                assert torch.equal(t, r)
    b.device_status()


def test_two_calls_at_once_on_two_streams():
    import torch
    from paper_1810_08313_b200 import binding as b
    ins = [_inputs(5), _inputs(6)]
    refs = [[t.clone() for t in _everything(b, s)] for s in ins]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for rep in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i].append(_everything(b, ins[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out in outs[i]:
            for t, r in zip(out, refs[i]):
                assert torch.equal(t, r)
    b.device_status()


def test_new_tensors_on_another_stream_are_not_blocks_in_use():
    """A block that the current stream has given back while a read of it is still queued there must not become an output
    or a workspace of a call on another stream."""
    import torch
    from paper_1810_08313_b200 import binding as b
    s = _inputs(8, "fp32")
    side = torch.cuda.Stream()
    like = [(2, 150, 72), (2, 150), (2,), (2, 333, 72), (2, 72)]
    nbytes = [b.orthogonalize_workspace(2, 150, 72), b.vocab_loss_workspace(2, 150, 333, 72, "fp32", True),
              b.layer_norm_grad_workspace(2, 150, 72)]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    copies = []
    for n in [4 * math.prod(t) for t in like] * 3 + nbytes:
        block = torch.full((n,), 77, dtype=torch.uint8, device="cuda")
        copies.append(torch.empty_like(block))
        copies[-1].copy_(block)
        del block
    y, mean, rstd = b.layer_norm(s["x"], s["w"], s["bias"], stream=side)
    b.layer_norm_grad(y, s["x"], s["w"], mean, rstd, stream=side)
    b.vocab_loss(y, s["W"], s["labels"], stream=side)
    b.vocab_loss_grad(y, s["W"], s["labels"], stream=side)
    b.orthogonalize(s["x"], stream=side)
    torch.cuda.synchronize()
    for c in copies:
        assert bool((c == 77).all())
    assert torch.equal(y, b.layer_norm(s["x"], s["w"], s["bias"])[0])
    b.device_status()


def test_given_workspaces_and_outputs():
    import torch
    from paper_1810_08313_b200 import binding as b
    s = _inputs(7)
    ref = b.vocab_loss_grad(s["x"], s["W"], s["labels"])
    ws = torch.full((b.vocab_loss_workspace(2, 150, 333, 72, "bf16", True),), 255, device="cuda", dtype=torch.uint8)
    out = [torch.full_like(t, 7.0) for t in ref]
    got = b.vocab_loss_grad(s["x"], s["W"], s["labels"], loss=out[0], row_loss=out[1], lse=out[2], dh=out[3], dW=out[4], workspace=ws)
    for t, o, r in zip(got, out, ref):
        assert t is o and torch.equal(t, r)
    small = torch.empty(1024, device="cuda", dtype=torch.uint8)
    for call in (lambda: b.vocab_loss_grad(s["x"], s["W"], s["labels"], workspace=small),
                 lambda: b.vocab_loss(s["x"], s["W"], s["labels"], workspace=small[:256]),
                 lambda: b.orthogonalize(s["W"], workspace=small)):
        with pytest.raises(b.LsError) as e:
            call()
        assert e.value.code == b.LS_ERR_STATE_SIZE


def test_single_replica_without_the_axis():
    import torch
    from paper_1810_08313_b200 import binding as b
    s = _inputs(8)
    one = {k: v[:1].contiguous() for k, v in s.items()}
    flat = {k: v[0].contiguous() for k, v in s.items()}
    for t, r in zip(_everything(b, flat), _everything(b, one)):
        assert t.shape == (r.shape if r.dim() == 1 and t.dim() == 1 else r.shape[1:]) and torch.equal(t.flatten(), r.flatten())


def test_binding_refusals():
    import torch
    from paper_1810_08313_b200 import binding as b
    s = _inputs(9)
    x, w, W, y = s["x"], s["w"], s["W"], s["labels"]
    _, mean, rstd = b.layer_norm(x, w)
    bad = [lambda: b.layer_norm(x.half(), w), lambda: b.layer_norm(x, w.double()), lambda: b.layer_norm(x, w[:, :-1]),
           lambda: b.layer_norm(x.transpose(1, 2), w), lambda: b.layer_norm(x, w.cpu()), lambda: b.layer_norm(x[..., ::2], w[:, ::2]),
           lambda: b.layer_norm(x, w[:1].expand(2, -1)), lambda: b.layer_norm(x, w, out=torch.empty_like(x, dtype=torch.float32)),
           lambda: b.layer_norm_grad(x.float(), x, w, mean, rstd), lambda: b.layer_norm_grad(x, x, w, mean[:, :-1], rstd),
           lambda: b.vocab_loss(x, W.float(), y), lambda: b.vocab_loss(x, W, y.long()), lambda: b.vocab_loss(x, W[..., :-8], y),
           lambda: b.vocab_loss(x, W, y[:, :-1]), lambda: b.vocab_loss_grad(x, W, y, dW=torch.empty_like(W, dtype=torch.float32)),
           lambda: b.vocab_loss(x, W[:1], y), lambda: b.orthogonalize(W.half()), lambda: b.orthogonalize(W[0, 0]),
           lambda: b.muon_step(W, W, W, 0.1), lambda: b.muon_step(w, w.clone()[:, :-1], w, 0.1),
           lambda: b.vocab_loss(x, W, y, workspace=torch.empty(100, device="cuda"))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {i} was not refused")
    with pytest.raises(b.LsError):
        b.orthogonalize(W, steps=0)
    with pytest.raises(b.LsError):
        b.vocab_loss_grad(x, W, y, scale=float("inf"))
    with pytest.raises(b.LsError):
        b.layer_norm(x, w, eps=-1.0)


def test_a_training_run_of_all_operators_together():
    """Three replicas train x -> V x -> layer norm -> output matrix with cross entropy, by orthogonalised steps of V, plain
    steps of the rest, and averaging every second step, in fp32, beside the same run in 64 bits with torch's autograd.
    Tolerance: the bounds of the single operators give gradients within 1e-4 of their norm (dominated by the logits' 2^-22
    times about 100); an orthogonalised step turns a relative error e of its direction into at most 4^5 e of the
    update's norm, here 0.1 lr of the weights' norm or less a step, so four steps stay within 4 * 1024 * 1e-4 * lr of it."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, rows, d_in, d, V = 3, 96, 40, 64, 130
    g = _gen(42)
    nV, nW = d * d_in, V * d
    P = nV + 2 * d + nW
    flat = torch.empty(m, P, device="cuda")
    flat[:] = _randn(g, P)[None] * 0.2
    flat[:, nV:nV + d] = 1.0
    mom = torch.zeros(m, nV, device="cuda").unflatten(1, (d, d_in))
    hid, lw, lb = flat[:, :nV].unflatten(1, (d, d_in)), flat[:, nV:nV + d], flat[:, nV + d:nV + 2 * d]
    out = flat[:, nV + 2 * d:].unflatten(1, (V, d))
    ref = flat.double().clone()
    rmom = torch.zeros(m, d, d_in, device="cuda", dtype=torch.float64)
    lr, mu = 0.02, 0.9

    def newton(u):
        x = u / (torch.linalg.norm(u) + 1e-7)
        x = x.T if d > d_in else x
        for _ in range(5):
            a = x @ x.T
            x = A * x + (B * a + CC * a @ a) @ x
        return x.T if d > d_in else x

    for step in range(4):
        x = _randn(g, m, rows, d_in)
        y = torch.randint(-1, V, (m, rows), generator=g, device="cuda").int()
        # the operators
        z = torch.bmm(x, hid.transpose(1, 2))
        n, mean, rstd = b.layer_norm(z, lw, lb)
        loss, _, _, dn, dout = b.vocab_loss_grad(n, out, y)
        dz, dlw, dlb = b.layer_norm_grad(dn, z, lw, mean, rstd)
        dhid = torch.bmm(dz.transpose(1, 2), x)
        b.muon_step(hid, mom, dhid, lr=lr, momentum=mu)
        out -= 0.5 * dout
        lw -= 0.5 * dlw
        lb -= 0.5 * dlb
        # the same in 64 bits
        for i in range(m):
            q = ref[i].clone().requires_grad_(True)
            h64 = q[:nV].view(d, d_in)
            z64 = x[i].double() @ h64.T
            n64 = torch.nn.functional.layer_norm(z64, (d,), q[nV:nV + d], q[nV + d:nV + 2 * d], 1e-5)
            l64 = torch.nn.functional.cross_entropy(n64 @ q[nV + 2 * d:].view(V, d).T, y[i].long(), ignore_index=-1)
            (gr,) = torch.autograd.grad(l64, q)
            assert abs(float(loss[i]) - float(l64.detach())) <= 1e-4 * float(l64.detach())
            gh = gr[:nV].view(d, d_in)
            rel = float(torch.linalg.norm(dhid[i].double() - gh) / torch.linalg.norm(gh))
            assert rel < 1e-2 if step else rel < 1e-4, (step, rel)
            rmom[i] = mu * rmom[i] + gh
            new = ref[i] - 0.5 * gr
            new[:nV] = ref[i][:nV] - (lr * math.sqrt(max(1.0, d / d_in)) * newton(gh + mu * rmom[i])).reshape(-1)
            ref[i] = new
        if step % 2 == 1:
            b.average_flat(flat.view(-1), m, P)
            ref[:] = ref.mean(0, keepdim=True)
            assert torch.equal(flat[0], flat[1]) and torch.equal(flat[0], flat[2])
    err = float(torch.linalg.norm(flat.double() - ref) / torch.linalg.norm(ref))
    assert err <= 4 * 1024 * 1e-4 * lr, err
    b.device_status()
