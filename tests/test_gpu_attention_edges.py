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


# ---- values that are not finite ----------------------------------------------------------------------------------------

U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}
NAN, INF = float("nan"), float("inf")


def _reference(q, k, v, dout, out, lse, cuts, scale):
    """Results and absolute sums of one head of queries and keys in 64 bits, each sum over the visible pairs alone: what is masked
    is never multiplied.  (out, dq, dk, dv), the same of absolute values, and the largest |q| . |k| scale."""
    import torch
    tokens, hd = q.shape
    q, k, v, dout, out, lse = (t.double() for t in (q, k, v, dout, out, lse))
    res = [torch.zeros(tokens, hd, dtype=torch.float64, device="cuda") for _ in range(8)]
    most = 0.0
    for a, b in zip(cuts, cuts[1:]):
        qs, ks, vs, ds, os_, ls = q[a:b], k[a:b], v[a:b], dout[a:b], out[a:b], lse[a:b]
        see = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").tril_()[:, :, None]

        def pairs(x):                            # sums over keys of [query][key][column], of what is visible
            return torch.where(see, x, 0.0)

        s = (qs[:, None] * ks[None]).sum(-1) * scale
        clean = (qs.nan_to_num(0, 0, 0).abs() @ ks.nan_to_num(0, 0, 0).abs().T) * scale
        most = max(most, float(clean.max()))
        top = torch.where(see[..., 0], s, -INF).amax(1, keepdim=True)
        e = torch.where(see[..., 0], (s - top).exp(), 0.0)
        p = (e / e.sum(1, keepdim=True))[:, :, None]
        res[0][a:b] = pairs(p * vs[None]).sum(1)
        res[4][a:b] = pairs(p * vs[None].abs()).sum(1)
        p = (s - ls[:, None]).exp()[:, :, None]
        dot = (ds * os_).sum(-1)[:, None, None]
        dp = (ds[:, None] * vs[None]).sum(-1, keepdim=True)
        size = (ds[:, None] * vs[None]).abs().sum(-1, keepdim=True) + (ds * os_).abs().sum(-1)[:, None, None]
        dz = p * (dp - dot)
        res[1][a:b] = pairs(dz * ks[None]).sum(1) * scale
        res[5][a:b] = pairs(p * size * ks[None].abs()).sum(1) * scale
        res[2][a:b] = pairs(dz * qs[:, None]).sum(0) * scale
        res[6][a:b] = pairs(p * size * qs[:, None].abs()).sum(0) * scale
        res[3][a:b] = pairs(p * ds[:, None]).sum(0)
        res[7][a:b] = pairs(p * ds[:, None].abs()).sum(0)
    return res[:4], res[4:], most


def _poison(case, q, k, v, dout):
    """Rows 3 to 389 are in two sequences, cut at 150; tiles of 128 rows hold rows of both, and rows before and behind the poisoned ones."""
    if case == "v":
        v[:, 200] = NAN
    elif case == "v columns":
        v[:, 200, 0, 5], v[:, 60, 0, 0], v[:, 300, 0, 5] = NAN, INF, -INF
    elif case == "v infinities":
        v[:, 170, 0, 1], v[:, 260, 0, 1], v[:, 30, 0, 1], v[:, 260, 0, 2] = INF, -INF, -INF, -INF
    elif case == "dout":
        dout[:, 333] = NAN
    elif case == "dout columns":
        dout[:, 333, 0, 2], dout[:, 100, 1, 3], dout[:, 390:] = INF, NAN, NAN
    elif case == "token":
        for t in (q, k, v, dout):
            t[:, 201] = NAN
    elif case == "q":
        q[:, 140], q[:, 160, 1] = NAN, INF
    elif case == "outside":
        for t in (q, k, v, dout):
            t[:, :3], t[:, 390:] = INF, NAN
    elif case == "all":
        for t in (q, k, v, dout):
            t.fill_(NAN)


POISONS = ["v", "v columns", "v infinities", "dout", "dout columns", "token", "q", "outside", "all"]


@pytest.mark.parametrize("dtype,hd", [("float32", 24), ("float32", 64), ("float32", 100), ("bfloat16", 64), ("bfloat16", 128), ("bfloat16", 72),
                                      ("bfloat16", 136)])
@pytest.mark.parametrize("case", POISONS)
def test_values_that_are_not_finite(case, dtype, hd):
    """Elements are NaN, infinite or finite as the sums over the visible rows are, and finite ones are as near as others.

    Per term of the absolute sums: the probability's and dS' rounding, twice 2^-8 (in fp32 2^-24 each), the exponent (hd roundings of
    the product or 16 truncated MMAs of 2^-22 of its absolute sum, log-sum-exp and its reference at most 2^-20), the product dout . v
    the same, sums of at most 390 x 2 terms, and the result's rounding."""
    import torch
    from paper_1810_08313_b200 import binding as b
    tokens, cuts, heads, scale = 400, [3, 150, 390], 2, 0.5 / hd ** 0.5
    q, k, v, dout = (_randn(s, 1, tokens, n, hd, dtype=dtype) for s, n in ((1, heads), (2, 1), (3, 1), (4, heads)))
    _poison(case, q, k, v, dout)
    seq = torch.tensor([cuts], dtype=torch.int32, device="cuda")
    out, lse = b.attention(q, k, v, seq, scale=scale)
    got = b.attention_grad(dout, q, k, v, out, lse, seq, scale=scale)
    b.device_status()
    sums = [0.0] * 8
    dkv = [0.0] * 4
    for h in range(heads):
        want, size, most = _reference(q[0, :, h], k[0, :, 0], v[0, :, 0], dout[0, :, h], out[0, :, h], lse[0, h], cuts, scale)
        rel = 3 * HALF[dtype] + 2 * ((hd * U + 16 * 2.0 ** -22) * (most + 1) + 2.0 ** -20) + 800 * U + 60 * 2.0 ** -22
        for name, x, i in (("out", out[0, :, h], 0), ("dq", got[0][0, :, h], 1)):
            _agree(x, want[i], rel * size[i], f"{name} {h}", i == 0)
        for i in (2, 3):
            dkv[i - 2], dkv[i] = dkv[i - 2] + want[i], dkv[i] + rel * size[i]
    _agree(got[1][0, :, 0], dkv[0], dkv[2], "dk", False)
    _agree(got[2][0, :, 0], dkv[1], dkv[3], "dv", True)


def _agree(got, want, tol, what, kinds):
    """Finite where `want` is, within tol; else not, and (kinds) the same infinity or NaN."""
    import torch
    x, fine = got.double(), torch.isfinite(want)
    assert torch.equal(torch.isfinite(x), fine), what
    if kinds:
        assert torch.equal(x[~fine].nan_to_num(1, 2, 3), want[~fine].nan_to_num(1, 2, 3)), what
    assert bool(((x - want).abs()[fine] <= tol[fine] + 2.0 ** -126).all()), what


@pytest.mark.parametrize("case", ["v", "dout", "token", "all"])
def test_values_that_are_not_finite_take_bounded_time(case):
    """4096 rows of 8 heads of 128, with NaN where rows depend on many others: no row walks over all of its keys for nothing.

    A row formed by itself over 4096 keys takes a warp about a millisecond, and there are 8 x 4096 of them: 0.2 s and more before only
    those were formed that share a tile with what they do not see."""
    import torch
    from paper_1810_08313_b200 import binding as b
    tokens, heads, kv, hd = 4096, 8, 4, 128
    q, k, v, dout = (_randn(s, 1, tokens, n, hd) for s, n in ((1, heads), (2, kv), (3, kv), (4, heads)))
    _poison(case, q, k, v, dout)

    def once():
        out, lse = b.attention(q, k, v)
        return b.attention_grad(dout, q, k, v, out, lse)

    once()
    start, stop = torch.cuda.Event(True), torch.cuda.Event(True)
    start.record()
    once()
    stop.record()
    stop.synchronize()
    assert start.elapsed_time(stop) < 60.0


# ---- what keys have in common ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("hd", [64, 72, 128])
def test_gradient_of_queries_whose_keys_have_much_in_common(hd):
    """A row's dS add up to dout . (exact out - out), nearly zero, so that what the keys share (16 in column 0, where q is zero) must
    not come back from the roundings of dS: two bf16 pieces keep 2^-17 of a term, one would keep 2^-9.

    Bounds per term: the exponent (16 truncated MMAs of 2^-22 of the product's absolute sum, hd roundings, log-sum-exp), the
    product dout . v and D the same, 2^-16 of dS for its pieces, sums of n keys in MMAs of 16, the result's rounding."""
    import torch
    from paper_1810_08313_b200 import binding as b
    tokens, cuts, scale = 300, [0, 9, 30, 64, 130, 300], 1.0 / hd ** 0.5
    q, k, v, dout = (_randn(s, 1, tokens, 1, hd) for s in (1, 2, 3, 4))
    q[..., 0], k[..., 0] = 0.0, 16.0
    seq = torch.tensor([cuts], dtype=torch.int32, device="cuda")
    out, lse = b.attention(q, k, v, seq)
    dq = b.attention_grad(dout, q, k, v, out, lse, seq)[0][0, :, 0].double()
    q, k, v, dout, out = (t[0, :, 0].double() for t in (q, k, v, dout, out))
    lse = lse[0, 0].double()[:, None]
    i = torch.arange(tokens, device="cuda")
    of = torch.bucketize(i, torch.tensor(cuts, device="cuda"), right=True)
    see = (of[:, None] == of[None, :]) & (i[None, :] <= i[:, None])
    s = (q @ k.T) * scale
    p = torch.where(see, (s - lse).exp(), 0.0)
    dot = (dout * out).sum(1, keepdim=True)
    ds = p * (dout @ v.T - dot)
    mma, n = hd * U + 16 * 2.0 ** -22, see.sum(1, keepdim=True)
    d = mma * (q.abs() @ k.abs().T) * scale + 4 * U * (s.abs() + lse.abs()) + 2.0 ** -22
    term = d * ds.abs() + p * mma * (dout.abs() @ v.abs().T + (dout * out).abs().sum(1, keepdim=True)) + (2.0 ** -16 + 4 * U) * ds.abs()
    keys = (n + 64) * U + (n / 16 + 8) * 2.0 ** -22
    want = (ds @ k) * scale
    tol = 1.05 * scale * (term @ k.abs() + keys * (ds.abs() @ k.abs())) + (2.0 ** -8 + 2 * U) * want.abs() + 2.0 ** -126
    assert bool(((dq - want).abs() <= tol).all())
    # with one piece, column 0 of many rows would lie outside
    one = (ds.float().bfloat16().double() @ k) * scale
    assert int(((one - want).abs() > tol)[:, 0].sum()) > tokens // 4
