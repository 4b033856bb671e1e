"""Head norm with rotation, packed causal attention and gradient clipping against 64-bit definitions.

Tolerances are elementwise bounds computed beside the reference from the roundings the kernels make (U = 2^-24, half a step of
fp32; 2^-8 relative for a rounding to bf16; a tensor-core product of at most 16 MMAs whose accumulator truncates, at most 2^-22
of the absolute sum each)."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LEAST = 2.0 ** -126
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _t(dtype):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


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


# ---- head norm and rotation ----------------------------------------------------------------------------------------

def _rope_case(m, tokens, heads, kv, hd, rot, dtype, seed=0, far=200000):
    import torch
    from paper_1810_08313_b200 import binding as b
    g = _gen(seed)
    q = (_randn(g, m, tokens, heads, hd) * (0.3 + _randn(g, m, 1, heads, 1).abs())).to(_t(dtype))
    k = (2.0 * _randn(g, m, tokens, kv, hd)).to(_t(dtype))
    qw, kw = 1.0 + 0.3 * _randn(g, m, hd), 1.0 + 0.3 * _randn(g, m, hd)
    pos = torch.randint(0, far, (m, tokens), generator=g, device="cuda", dtype=torch.int32)
    return q, k, qw, kw, pos, b.rope_frequencies(rot, 10000.0)


def _pairs(hd, rot, interleaved):
    """Indices of the first and second elements of the turned pairs."""
    import torch
    p = torch.arange(rot // 2, device="cuda")
    return (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)


def _rotate(z, pos, freq, rot, interleaved, back=False):
    angle = pos.double()[..., None, None] * freq
    c, s = angle.cos(), angle.sin() * (-1.0 if back else 1.0)
    ia, ib = _pairs(z.shape[-1], rot, interleaved)
    y = z.clone()
    y[..., ia] = z[..., ia] * c - z[..., ib] * s
    y[..., ib] = z[..., ia] * s + z[..., ib] * c
    return y


def _mates(z, rot, interleaved):
    """|a| + |b| of the pair that an element belongs to (|a| alone outside)."""
    ia, ib = _pairs(z.shape[-1], rot, interleaved)
    y = z.abs()
    t = y[..., ia] + y[..., ib]
    y = y.clone()
    y[..., ia] = t
    y[..., ib] = t
    return y


# rstd: eight squares a lane and five shuffle steps (13 roundings, halved by the root), root and division: 9 U.  Times the
# weight 2 U, the turn 2 U, cosine and sine 8 U (the reduced angle rounded to fp32, and the functions).
ROPE = 21 * U


def _angle_tol(pos, freq):
    """What the double arithmetic leaves of an angle: two roundings of it."""
    return 2.0 ** -52 * float(pos.abs().max()) * float(freq.max() if freq.numel() else 0.0)


def _rope_check(q, k, qw, kw, pos, freq, eps, inter, got, dtype):
    rot = 2 * freq.numel()
    for x, w, y in ((q, qw, got[0]), (k, kw, got[1])):
        x64 = x.double()
        z = x64 / (x64.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()[:, None, None]
        want = _rotate(z, pos, freq, rot, inter)
        _within(y, want, (ROPE + _angle_tol(pos, freq)) * _mates(z, rot, inter) + HALF[dtype] * want.abs() + 1e-300, "y")


ROPE_SIZES = [(1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 2, 2), (2, 3, 4, 2, 8, 8), (1, 24, 8, 2, 64, 64), (3, 17, 6, 3, 80, 32),
              (1, 9, 5, 5, 96, 96), (2, 5, 32, 8, 128, 128), (1, 70, 3, 1, 128, 64), (1, 7, 2, 2, 256, 256), (1, 6, 2, 1, 33, 10),
              (2, 4, 3, 3, 255, 254), (1, 11, 7, 7, 24, 20), (1, 700, 4, 4, 16, 16), (1, 5, 40, 8, 72, 0), (1, 2500, 3, 1, 40, 40)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("m,tokens,heads,kv,hd,rot", ROPE_SIZES)
def test_qk_norm_rope(m, tokens, heads, kv, hd, rot, inter, dtype):
    from paper_1810_08313_b200 import binding as b
    q, k, qw, kw, pos, freq = _rope_case(m, tokens, heads, kv, hd, rot, dtype, seed=tokens + hd)
    got = b.qk_norm_rope(q, k, qw, kw, pos, freq, eps=1e-6, interleaved=inter)
    _rope_check(q, k, qw, kw, pos, freq, 1e-6, inter, got, dtype)


def _rope_grad_check(dy, x, w, pos, freq, eps, inter, dx, dw, dtype):
    rot = 2 * freq.numel()
    x64, w64 = x.double(), w.double()[:, None, None]
    r = 1.0 / (x64.square().mean(-1, keepdim=True) + eps).sqrt()
    xhat = x64 * r
    dz = _rotate(dy.double(), pos, freq, rot, inter, back=True)
    tz = (12 * U + _angle_tol(pos, freq)) * _mates(dy.double(), rot, inter)         # cosine, sine and the turn
    tx = 10 * U * xhat.abs()
    t = dz * w64
    tt = tz * w64.abs() + U * t.abs()
    along = (t * xhat).mean(-1, keepdim=True)
    ta = (16 * U * (t * xhat).abs() + tt * xhat.abs() + t.abs() * tx).mean(-1, keepdim=True)
    want = r * (t - xhat * along)
    tol = r * (tt + xhat.abs() * ta + tx * along.abs()) + 12 * U * r * (t.abs() + (xhat * along).abs())
    _within(dx, want, 1.02 * tol + HALF[dtype] * want.abs() + 1e-300, "dx")
    n = x.shape[1] * x.shape[2]                                  # additions in one lane at most, then lanes, warps and CTAs
    terms = (dz * xhat).abs()
    tol = (min(n, 4000) + 64) * U * terms.sum((1, 2)) + (tz * xhat.abs() + dz.abs() * tx).sum((1, 2))
    _within(dw, (dz * xhat).sum((1, 2)), 1.02 * tol + 1e-300, "dw")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("m,tokens,heads,kv,hd,rot", ROPE_SIZES)
def test_qk_norm_rope_grad(m, tokens, heads, kv, hd, rot, inter, dtype):
    from paper_1810_08313_b200 import binding as b
    q, k, qw, kw, pos, freq = _rope_case(m, tokens, heads, kv, hd, rot, dtype, seed=tokens + hd)
    g = _gen(5)
    dq, dk = _randn(g, *q.shape).to(q.dtype), _randn(g, *k.shape).to(q.dtype)
    got = b.qk_norm_rope_grad(dq, dk, q, k, qw, kw, pos, freq, eps=1e-6, interleaved=inter)
    _rope_grad_check(dq, q, qw, pos, freq, 1e-6, inter, got[0], got[2], dtype)
    _rope_grad_check(dk, k, kw, pos, freq, 1e-6, inter, got[1], got[3], dtype)


@pytest.mark.parametrize("inter", [False, True])
def test_qk_norm_rope_grad_against_differences(inter):
    """<gradient, direction> against a central difference of the 64-bit function (off by step^2 / 6 of its third derivative)."""
    import torch
    from paper_1810_08313_b200 import binding as b
    q, k, qw, kw, pos, freq = _rope_case(2, 13, 3, 1, 48, 32, "fp32", seed=3, far=100)
    g = _gen(9)
    gq, gk = _randn(g, *q.shape), _randn(g, *k.shape)

    def value(q, k, qw, kw):
        total = 0.0
        for x, w, d in ((q, qw, gq), (k, kw, gk)):
            z = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w[:, None, None]
            total += float((_rotate(z, pos, freq, 32, inter) * d.double()).sum())
        return total

    at = [t.double() for t in (q, k, qw, kw)]
    grads = b.qk_norm_rope_grad(gq, gk, q, k, qw, kw, pos, freq, interleaved=inter)
    for i in range(4):
        u = _randn(g, *at[i].shape).double()
        h = 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * u, at[i] - h * u
        want = (value(*up) - value(*down)) / (2 * h)
        got = float((grads[i].double() * u).sum())
        assert abs(got - want) <= 1e-5 * float((grads[i].double() * u).abs().sum()), (i, got, want)


def test_qk_norm_rope_far_positions_and_zero_rows():
    import torch
    from paper_1810_08313_b200 import binding as b
    q, k, qw, kw, pos, freq = _rope_case(1, 6, 2, 1, 64, 64, "fp32", seed=1)
    pos = torch.tensor([[0, -5, 2 ** 31 - 1, -2 ** 31, 10 ** 6, 131071]], dtype=torch.int32, device="cuda")
    _rope_check(q, k, qw, kw, pos, freq, 1e-6, False, b.qk_norm_rope(q, k, qw, kw, pos, freq), "fp32")
    z = torch.zeros_like(q)
    y, _ = b.qk_norm_rope(z, k, qw, kw, pos, freq)
    assert not bool(y.any())
    dq, dk, dqw, dkw = b.qk_norm_rope_grad(torch.ones_like(z), torch.zeros_like(k), z, k, qw, kw, pos, freq)
    assert bool(torch.isfinite(dq).all()) and not bool(dqw.any()) and not bool(dk.any()) and not bool(dkw.any())
    # a NaN stays in its head
    q[0, 2, 1, 5] = float("nan")
    y, yk = b.qk_norm_rope(q, k, qw, kw, pos, freq)
    bad = torch.isnan(y).any(-1)[0].nonzero().tolist()
    assert bad == [[2, 1]] and not bool(torch.isnan(yk).any())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("off", [0, 1])
def test_qk_norm_rope_of_a_projection(dtype, off):
    """q and k as parts of one projection's rows, read and written in place of their own rows; misaligned by one element."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, tokens, heads, kv, hd = 2, 37, 6, 2, 64
    width = (heads + 2 * kv) * hd + 8
    g = _gen(2)
    base = _randn(g, m, tokens * width + 16).to(_t(dtype))
    rows = base[:, off:off + tokens * width].unflatten(1, (tokens, width))
    q, k = rows[..., :heads * hd].unflatten(-1, (heads, hd)), rows[..., heads * hd:(heads + kv) * hd].unflatten(-1, (kv, hd))
    _, _, qw, kw, pos, freq = _rope_case(m, tokens, heads, kv, hd, hd, dtype)
    dst = torch.full_like(base, 7.0)
    drows = dst[:, off:off + tokens * width].unflatten(1, (tokens, width))
    qo, ko = drows[..., :heads * hd].unflatten(-1, (heads, hd)), drows[..., heads * hd:(heads + kv) * hd].unflatten(-1, (kv, hd))
    got = b.qk_norm_rope(q, k, qw, kw, pos, freq, q_out=qo, k_out=ko)
    _rope_check(q, k, qw, kw, pos, freq, 1e-6, False, got, dtype)
    assert bool((drows[..., (heads + kv) * hd:] == 7.0).all()) and bool((dst[:, off + tokens * width:] == 7.0).all())
    dst.fill_(7.0)
    gq, gk = _randn(g, *q.shape).to(q.dtype), _randn(g, *k.shape).to(q.dtype)
    out = b.qk_norm_rope_grad(gq, gk, q, k, qw, kw, pos, freq, dq=qo, dk=ko)
    _rope_grad_check(gq, q, qw, pos, freq, 1e-6, False, out[0], out[2], dtype)
    _rope_grad_check(gk, k, kw, pos, freq, 1e-6, False, out[1], out[3], dtype)
    assert bool((drows[..., (heads + kv) * hd:] == 7.0).all())


# ---- attention -----------------------------------------------------------------------------------------------------

def _mask(tokens, starts):
    """[tokens][tokens]: key j is seen by row i."""
    import torch
    seq = torch.full((tokens,), -1, dtype=torch.int64)
    for s, (a, b) in enumerate(zip(starts, starts[1:])):
        seq[a:b] = s
    seq = seq.cuda()
    i = torch.arange(tokens, device="cuda")
    return (seq[:, None] == seq[None, :]) & (seq >= 0)[:, None] & (i[None, :] <= i[:, None])


def _attn_case(m, tokens, heads, kv, hd, dtype, seed=0, sharp=1.5):
    g = _gen(seed)
    q = (sharp * _randn(g, m, tokens, heads, hd)).to(_t(dtype))
    k, v = _randn(g, m, tokens, kv, hd).to(_t(dtype)), _randn(g, m, tokens, kv, hd).to(_t(dtype))
    return q, k, v


def _score_tol(q, k, s, ref, scale, hd):
    """Error of an exponent: the product's (hd roundings, or truncated MMAs), the scaling and the difference from the reference,
    and 2^-22 for the exponential."""
    a = (q.abs() @ k.abs().T) * abs(scale)
    return (hd * U + 16 * 2.0 ** -22) * a + 4 * U * (s.abs() + ref.abs()) + 2.0 ** -22


def _attn_check(q, k, v, starts, scale, out, lse, dtype):
    import torch
    m, tokens, heads, hd = q.shape
    group = heads // k.shape[2]
    rp = HALF[dtype] if dtype == "bf16" else U
    for r in range(m):
        see = _mask(tokens, starts[r])
        some = see.any(1)
        for h in range(heads):
            qq, kk, vv = q[r, :, h].double(), k[r, :, h // group].double(), v[r, :, h // group].double()
            s = (qq @ kk.T) * scale
            sm = s.masked_fill(~see, -math.inf)
            l64 = torch.logsumexp(sm, 1)
            p = torch.where(see, (sm - l64[:, None]).exp(), 0.0)
            want = torch.where(some[:, None], p @ vv, 0.0)
            # (the running reference is at most 8 binary orders away from the maximum)
            d = torch.where(see, _score_tol(qq, kk, s, l64.nan_to_num(0, 0, 0)[:, None].abs() + 8, scale, hd), 0.0)
            n = see.sum(1, keepdim=True).double()
            keys = (n + 64) * U + (n / 16 + 8) * 2.0 ** -22
            a = p @ vv.abs()
            # numerator and sum: each term's exponent, roundings of the operands, additions
            tol = (p * d) @ vv.abs() + (rp + keys) * a + ((p * d).sum(1, keepdim=True) + keys + 4 * U) * want.abs()
            _within(out[r, :, h], want, torch.where(some[:, None], 1.05 * tol + HALF[dtype] * want.abs(), 0.0), f"out {r} {h}")
            wl = torch.where(some, l64, 0.0)
            tl = (p * d).sum(1) + keys[:, 0] + 8 * U * wl.abs() + 8 * U
            _within(lse[r, h], wl, torch.where(some, 1.05 * tl, 0.0), f"lse {r} {h}")


def _attn_grad_check(dout, q, k, v, o, lse, starts, scale, got, dtype):
    import torch
    m, tokens, heads, hd = q.shape
    kv = k.shape[2]
    group = heads // kv
    rp = HALF[dtype] if dtype == "bf16" else U
    dq, dk, dv = got
    mma = hd * U + 16 * 2.0 ** -22
    for r in range(m):
        see = _mask(tokens, starts[r])
        n = float(see.sum(1).max()) * group
        keys = (n + 64) * U + (n / 16 + 8) * 2.0 ** -22
        for hk in range(kv):
            wk, wv, tk, tv = 0.0, 0.0, 0.0, 0.0
            kk, vv = k[r, :, hk].double(), v[r, :, hk].double()
            for h in range(hk * group, (hk + 1) * group):
                qq, dd, oo, l = q[r, :, h].double(), dout[r, :, h].double(), o[r, :, h].double(), lse[r, h].double()[:, None]
                # (what rows in no sequence hold does not count)
                live = see.any(1)[:, None]
                qq, dd, oo = (torch.where(live, t, 0.0) for t in (qq, dd, oo))
                kc, vc = torch.where(live, kk, 0.0), torch.where(live, vv, 0.0)
                s = (qq @ kc.T) * scale
                p = torch.where(see, (s - l).exp(), 0.0)
                d = _score_tol(qq, kc, s, l, scale, hd)
                dot = (dd * oo).sum(1, keepdim=True)
                dp = dd @ vc.T
                ds = p * (dp - dot)
                # (an exponential or product below the smallest normal number, 2^-126, may come out as zero)
                tp = p * d + torch.where(see, LEAST, 0.0)
                tds = LEAST + tp * (dp - dot).abs() + p * (mma * (dd.abs() @ vc.abs().T) + mma * (dd * oo).abs().sum(1, keepdim=True)) + (rp + 4 * U) * ds.abs()
                tp = tp + (rp + U) * p
                wq = (ds @ kc) * scale
                tq = (tds @ kc.abs() + keys * (ds.abs() @ kc.abs())) * abs(scale)
                _within(dq[r, :, h], wq, 1.05 * tq + (HALF[dtype] + 2 * U) * wq.abs() + LEAST, f"dq {r} {h}")
                wk, tk = wk + (ds.T @ qq) * scale, tk + (tds.T @ qq.abs() + keys * (ds.abs().T @ qq.abs())) * abs(scale)
                wv, tv = wv + p.T @ dd, tv + tp.T @ dd.abs() + keys * (p.T @ dd.abs())
            _within(dk[r, :, hk], wk, 1.05 * tk + (HALF[dtype] + 2 * U) * wk.abs() + LEAST, f"dk {r} {hk}")
            _within(dv[r, :, hk], wv, 1.05 * tv + (HALF[dtype] + 2 * U) * wv.abs() + LEAST, f"dv {r} {hk}")


def _starts(starts, m):
    """The same boundaries for every replica, moved by one for the second where they allow it."""
    import torch
    rows = [list(starts) for _ in range(m)]
    if m > 1 and len(starts) > 2 and starts[1] + 1 <= starts[2]:
        rows[1][1] += 1
    return rows, torch.tensor(rows, dtype=torch.int32, device="cuda")


def _attn_run(m, tokens, starts, heads, kv, hd, dtype, grad=True, sharp=1.5):
    from paper_1810_08313_b200 import binding as b
    q, k, v = _attn_case(m, tokens, heads, kv, hd, dtype, seed=tokens + hd, sharp=sharp)
    rows, seq = _starts(starts, m)
    scale = 1.0 / math.sqrt(hd)
    out, lse = b.attention(q, k, v, seq)
    _attn_check(q, k, v, rows, scale, out, lse, dtype)
    if grad:
        dout = _randn(_gen(4), *q.shape).to(q.dtype)
        got = b.attention_grad(dout, q, k, v, out, lse, seq)
        _attn_grad_check(dout, q, k, v, out, lse, rows, scale, got, dtype)
    b.device_status()


# sequences of one token, empty ones, boundaries beside tile edges, rows before the first and behind the last sequence
ATTN_SEQS = [(1, [0, 1]), (2, [0, 1, 2]), (5, [0, 5]), (64, [0, 64]), (65, [0, 65]), (127, [0, 40, 40, 127]), (128, [0, 128]),
             (129, [0, 129]), (130, [3, 10, 100]), (200, list(range(0, 201))), (255, [0, 127, 128, 129, 255]), (256, [0, 256]),
             (257, [0, 1, 257]), (300, [150, 150, 299]), (384, [0, 384]), (385, [0, 128, 256, 384, 385]), (517, [5, 130, 390, 500]),
             (640, [0, 640]), (40, [40, 40])]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,starts", ATTN_SEQS)
def test_attention_sequences(tokens, starts, dtype):
    _attn_run(2 if tokens < 300 else 1, tokens, starts, 4, 2, 64, dtype)


@pytest.mark.parametrize("tokens,starts", ATTN_SEQS)
def test_attention_sequences_heads_of_128(tokens, starts):
    _attn_run(1, tokens, starts, 3, 1, 128, "bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attention_of_nothing(dtype):
    """No sequences, and no tokens."""
    import torch
    from paper_1810_08313_b200 import binding as b
    q, k, v = _attn_case(2, 200, 2, 1, 64, dtype)
    seq = torch.full((2, 1), 50, dtype=torch.int32, device="cuda")
    out, lse = b.attention(q, k, v, seq)
    assert not bool(out.any()) and not bool(lse.any())
    assert not any(bool(t.any()) for t in b.attention_grad(torch.ones_like(q), q, k, v, out, lse, seq))
    out, lse = b.attention(q[:, :0], k[:, :0], v[:, :0])
    assert out.shape == (2, 0, 2, 64) and lse.shape == (2, 2, 0)
    assert [t.numel() for t in b.attention_grad(out, q[:, :0], k[:, :0], v[:, :0], out, lse)] == [0, 0, 0]
    pos = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    w = torch.ones(2, 64, device="cuda")
    got = b.qk_norm_rope_grad(q[:, :0], k[:, :0], q[:, :0], k[:, :0], w, w, pos, b.rope_frequencies(64))
    assert not bool(got[2].any()) and not bool(got[3].any())


def test_attention_refusals():
    import torch
    from paper_1810_08313_b200 import binding as b
    q, k, v = _attn_case(2, 20, 4, 2, 16, "bf16")
    seq = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for call in (lambda: b.attention(q, k.float(), v), lambda: b.attention(q, k, v[:, :19]), lambda: b.attention(q, k[..., :8], v),
                 lambda: b.attention(q[0], k, v), lambda: b.attention(q, k, v, seq[:1]), lambda: b.attention(q, k, v, seq.long()),
                 lambda: b.attention(q, k, v.transpose(2, 3).contiguous().transpose(2, 3)), lambda: b.attention(q, k, v, out=q[:, :, :2]),
                 lambda: b.attention(q.half(), k.half(), v.half()), lambda: b.attention(q, k, v, lse=torch.zeros(2, 4, 19, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: b.attention(q[:, :, :3], k, v), lambda: b.attention(q, k, v, scale=math.inf),
                 lambda: b.attention(q, k[:, :1].expand(-1, 20, -1, -1), v)):
        with pytest.raises(b.LsError):
            call()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [1, 7, 8, 16, 24, 32, 33, 40, 48, 72, 80, 96, 104, 112, 120, 128, 130, 136, 200, 256])
def test_attention_head_sizes(hd, dtype):
    _attn_run(1, 275, [0, 100, 275], 4, 2, hd, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 1), (6, 3), (7, 7), (12, 4), (16, 2)])
def test_attention_groups(heads, kv, dtype):
    _attn_run(2, 190, [0, 61, 190], heads, kv, 64, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sharp", [0.01, 12.0, 60.0])
def test_attention_flat_and_sharp(sharp, dtype):
    """Nearly uniform rows, and rows whose maximum moves by many binary orders from tile to tile."""
    _attn_run(1, 700, [0, 700], 2, 1, 64, dtype, sharp=sharp)


@pytest.mark.parametrize("dtype,hd", [("fp32", 64), ("bf16", 64), ("bf16", 128)])
def test_attention_many_tiles(hd, dtype):
    """Enough tiles of keys for all SMs: no cluster shares one."""
    _attn_run(3, 1100, [0, 500, 1093], 4, 4, hd, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("count", [31, 32, 40, 1400])
def test_attention_many_sequences(count, dtype):
    """More boundaries than a warp holds, in one and two levels of the search; some sequences are empty."""
    import random
    cuts = sorted(random.Random(count).choices(range(0, 1500), k=count + 1))
    _attn_run(1, 1500, cuts, 2, 1, 64, dtype)


def test_attention_rising_scores():
    """Keys that grow along the sequence: every tile has a new maximum."""
    import torch
    from paper_1810_08313_b200 import binding as b
    for dtype in ("fp32", "bf16"):
        for hd in (64, 128):
            q, k, v = _attn_case(1, 900, 2, 1, hd, dtype, seed=11)
            q[..., 0], k[..., 0] = 4.0, (torch.arange(900, device="cuda")[None, :, None] / 30.0).to(k.dtype)
            out, lse = b.attention(q, k, v)
            _attn_check(q, k, v, [[0, 900]], 1.0 / math.sqrt(hd), out, lse, dtype)
            dout = _randn(_gen(4), *q.shape).to(q.dtype)
            _attn_grad_check(dout, q, k, v, out, lse, [[0, 900]], 1.0 / math.sqrt(hd),
                             b.attention_grad(dout, q, k, v, out, lse), dtype)


@pytest.mark.parametrize("scale", [0.0, -0.7, 0.3])
def test_attention_scale(scale):
    from paper_1810_08313_b200 import binding as b
    for dtype in ("fp32", "bf16"):
        q, k, v = _attn_case(1, 150, 2, 2, 64, dtype, seed=2, sharp=0.5)
        out, lse = b.attention(q, k, v, scale=scale)
        _attn_check(q, k, v, [[0, 150]], scale, out, lse, dtype)
        dout = _randn(_gen(4), *q.shape).to(q.dtype)
        _attn_grad_check(dout, q, k, v, out, lse, [[0, 150]], scale,
                         b.attention_grad(dout, q, k, v, out, lse, scale=scale), dtype)


@pytest.mark.parametrize("dtype,hd", [("fp32", 64), ("bf16", 64), ("bf16", 128), ("bf16", 136)])
def test_attention_keeps_nan_to_itself(dtype, hd):
    """NaN and infinities in one sequence, and in the rows outside all, reach no other sequence and no earlier row."""
    import torch
    from paper_1810_08313_b200 import binding as b
    tokens, starts = 330, [10, 90, 200, 300]
    seq = torch.tensor([starts], dtype=torch.int32, device="cuda")
    q, k, v = _attn_case(1, tokens, 2, 1, hd, dtype, seed=7)
    dout = _randn(_gen(4), *q.shape).to(q.dtype)
    clean_out, clean_lse = b.attention(q, k, v, seq)
    clean = b.attention_grad(dout, q, k, v, clean_out, clean_lse, seq)
    nan, inf = float("nan"), float("inf")
    for t in (q, k, v, dout):
        t[:, :10] = nan
        t[:, 300:] = inf
    k[0, 140], v[0, 140] = nan, nan                       # from row 140 of the second sequence on
    out, lse = b.attention(q, k, v, seq)
    keep = [i for i in range(tokens) if not 140 <= i < 200]
    _attn_check(q[:, keep].nan_to_num(0, 0, 0), k[:, keep].nan_to_num(0, 0, 0), v[:, keep].nan_to_num(0, 0, 0),
                [[10, 90, 140, 240]], 1.0 / math.sqrt(hd), out[:, keep], lse[:, :, keep], dtype)
    assert bool(torch.isnan(out[:, 140:200]).all()) and bool(torch.isnan(lse[:, :, 140:200]).all())
    out[:, :10], out[:, 300:] = nan, inf
    lse[..., :10], lse[..., 300:] = nan, -inf
    dq, dk, dv = b.attention_grad(dout, q, k, v, out, lse, seq)
    for got, want in zip((dq, dk, dv), clean):
        other = torch.cat((got[:, :90], got[:, 200:]), 1).double()
        ref = torch.cat((want[:, :90], want[:, 200:]), 1).double()
        assert bool(torch.isfinite(other).all())
        assert float((other - ref).abs().max()) <= 0.05 * float(ref.abs().max())
        assert not bool(got[:, :10].any()) and not bool(got[:, 300:].any())
    # the queries before row 140 do not see it
    assert bool(torch.isfinite(dq[:, 90:140]).all()) and bool(torch.isnan(dq[:, 140:200]).all())
    assert bool(torch.isnan(dk[:, 90:200]).all()) and bool(torch.isnan(dv[:, 90:200]).all())
    b.device_status()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attention_infinite_scores(dtype):
    """Scores of -inf take no part; a row of nothing else, or with one of +inf, has no softmax."""
    import torch
    from paper_1810_08313_b200 import binding as b
    q, k, v = _attn_case(1, 40, 1, 1, 64, dtype, seed=8)
    q[..., 0] = 1.0
    k[0, 20, 0, 0] = -float("inf")
    out, lse = b.attention(q, k, v)
    keep = [i for i in range(40) if i != 20]
    _attn_check(q[:, keep], k[:, keep], v[:, keep], [[0, 39]], 0.125, out[:, keep], lse[:, :, keep], dtype)
    k[0, 0, 0, 0], k[0, 30, 0, 0] = -float("inf"), float("inf")
    out, lse = b.attention(q, k, v)
    assert bool(torch.isnan(out[0, 0]).all()) and float(lse[0, 0, 0]) == -math.inf
    assert bool(torch.isfinite(out[0, 1:30]).all()) and bool(torch.isnan(out[0, 30:]).all())
    assert bool((lse[0, 0, 30:] == math.inf).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("off", [0, 1])
def test_attention_of_a_projection(dtype, off):
    """q, k and v as parts of one projection's rows, the gradients as parts of its gradient; misaligned by one element."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, tokens, heads, kv, hd = 2, 150, 6, 2, 64
    width = (heads + 2 * kv) * hd + 16
    g = _gen(2)

    def parts(flat):
        rows = flat[:, off:off + tokens * width].unflatten(1, (tokens, width))
        cuts = [0, heads * hd, (heads + kv) * hd, (heads + 2 * kv) * hd]
        return [rows[..., a:e].unflatten(-1, ((e - a) // hd, hd)) for a, e in zip(cuts, cuts[1:])] + [rows[..., cuts[3]:]]

    base = _randn(g, m, tokens * width + 16).to(_t(dtype))
    q, k, v, _ = parts(base)
    rows, seq = _starts([0, 70, 141], m)
    out, lse = b.attention(q, k, v, seq)
    _attn_check(q, k, v, rows, 0.125, out, lse, dtype)
    dst = torch.full_like(base, 7.0)
    dq, dk, dv, rest = parts(dst)
    dout = _randn(g, *out.shape).to(out.dtype)
    b.attention_grad(dout, q, k, v, out, lse, seq, dq=dq, dk=dk, dv=dv)
    _attn_grad_check(dout, q, k, v, out, lse, rows, 0.125, (dq, dk, dv), dtype)
    assert bool((rest == 7.0).all()) and bool((dst[:, off + tokens * width:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attention_offsets_beyond_32_bits(dtype):
    """Rows so far apart that the last ones lie beyond 2^31 elements."""
    import torch
    from paper_1810_08313_b200 import binding as b
    tokens, row, heads, kv, hd = 260, 2 ** 23 + 64, 2, 1, 64
    big = torch.zeros(tokens * row, dtype=_t(dtype), device="cuda")
    rows = big.view(tokens, row)
    g = _gen(3)
    rows[:, :(heads + 2 * kv) * hd] = _randn(g, tokens, (heads + 2 * kv) * hd).to(big.dtype)
    q, k, v = (rows[:, a:e].unflatten(-1, ((e - a) // hd, hd)) for a, e in ((0, 128), (128, 192), (192, 256)))
    out, lse = rows[:, 1024:1152].unflatten(-1, (2, hd)), None
    out, lse = b.attention(q, k, v, out=out)
    _attn_check(q[None], k[None], v[None], [[0, tokens]], 0.125, out[None], lse[None], dtype)
    dout = _randn(g, tokens, heads, hd).to(big.dtype)
    dq, dk, dv = (rows[:, a:e].unflatten(-1, ((e - a) // hd, hd)) for a, e in ((2048, 2176), (2176, 2240), (2240, 2304)))
    b.attention_grad(dout, q, k, v, out, lse, dq=dq, dk=dk, dv=dv)
    _attn_grad_check(dout[None], q[None], k[None], v[None], out[None], lse[None], [[0, tokens]], 0.125, (dq[None], dk[None], dv[None]), dtype)


def test_attention_boundaries_that_make_no_sense():
    """Descending boundaries, or ones outside the rows, give some result without an access outside."""
    import torch
    from paper_1810_08313_b200 import binding as b
    for dtype in ("fp32", "bf16"):
        q, k, v = _attn_case(1, 300, 2, 1, 64, dtype)
        for cuts in ([0, 200, 100, 300], [-50, 120, 9000], [300, 0, 300], [2 ** 31 - 1, -2 ** 31, 5, 7]):
            seq = torch.tensor([cuts], dtype=torch.int32, device="cuda")
            out, lse = b.attention(q, k, v, seq)
            b.attention_grad(torch.ones_like(q), q, k, v, out, lse, seq)
            b.device_status()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attention_grad_against_differences(dtype):
    """<gradient, direction> against a central difference of the 64-bit function at the same (rounded) inputs; bf16 adds the
    rounding of P, dS, out and the results: four times 2^-8 of the terms' absolute sums."""
    import torch
    from paper_1810_08313_b200 import binding as b
    q, k, v = _attn_case(1, 140, 4, 2, 64, dtype, seed=5)
    rows, seq = _starts([0, 50, 133], 1)
    g = _gen(6)
    dout = _randn(g, *q.shape).to(q.dtype)
    see = _mask(140, rows[0])

    def value(q, k, v):
        total = 0.0
        for h in range(4):
            s = (q[0, :, h] @ k[0, :, h // 2].T) * 0.125
            p = torch.softmax(s.masked_fill(~see, -1e30), 1) * see
            total += float((p @ v[0, :, h // 2] * dout[0, :, h].double()).sum())
        return total

    at = [t.double() for t in (q, k, v)]
    out, lse = b.attention(q, k, v, seq)
    grads = b.attention_grad(dout, q, k, v, out, lse, seq)
    for i in range(3):
        u = _randn(g, *at[i].shape).double()
        h = 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * u, at[i] - h * u
        want = (value(*up) - value(*down)) / (2 * h)
        terms = grads[i].double() * u
        assert abs(float(terms.sum()) - want) <= (1e-5 if dtype == "fp32" else 2.0 ** -6) * float(terms.abs().sum()), (i, want)


@pytest.mark.parametrize("dtype,hd", [("fp32", 40), ("bf16", 64), ("bf16", 128)])
def test_attention_is_repeatable_and_captured(dtype, hd):
    """The same bits on every run, on another stream, and from a graph replayed on new inputs."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, tokens, heads, kv = 2, 700, 6, 2
    rows, seq = _starts([0, 333, 690], m)
    a = [_attn_case(m, tokens, heads, kv, hd, dtype, seed=s) for s in (1, 2)]
    douts = [_randn(_gen(s), m, tokens, heads, hd).to(_t(dtype)) for s in (3, 4)]

    def both(q, k, v, dout, **kw):
        out, lse = b.attention(q, k, v, seq, **kw)
        return (out, lse, *b.attention_grad(dout, q, k, v, out, lse, seq, **kw))

    want = [both(*x, d) for x, d in zip(a, douts)]
    for _ in range(3):
        for x, d, w in zip(a, douts, want):
            assert all(torch.equal(i, j) for i, j in zip(both(*x, d), w))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(*a[0], douts[0], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(i, j) for i, j in zip(got, want[0]))
    x, d = [t.clone() for t in a[0]], douts[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(*x, d)
    for i in (1, 0, 1):
        for t, s in zip(x + [d], (*a[i], douts[i])):
            t.copy_(s)
        graph.replay()
        assert all(torch.equal(p, w) for p, w in zip(got, want[i]))
    b.device_status()


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_replayed_with_other_boundaries(hd):
    """A captured pair of calls reads its boundaries when it runs."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, tokens = 2, 900
    q, k, v = _attn_case(m, tokens, 4, 2, hd, "bf16")
    dout = _randn(_gen(5), m, tokens, 4, hd).bfloat16()
    tables = [_starts(s, m)[1] for s in ([0, 900, 900, 900], [0, 1, 450, 880], [100, 100, 100, 101], [7, 300, 301, 900])]

    def both(seq):
        out, lse = b.attention(q, k, v, seq)
        return (out, lse, *b.attention_grad(dout, q, k, v, out, lse, seq))

    want = [both(s) for s in tables]
    seq = tables[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(seq)
    for i in (1, 2, 0, 3):
        seq.copy_(tables[i])
        graph.replay()
        assert all(torch.equal(p, w) for p, w in zip(got, want[i]))
    b.device_status()


def test_attention_on_several_streams_at_once():
    """Calls of different shapes and types that share the SMs give what they give alone."""
    import torch
    from paper_1810_08313_b200 import binding as b
    cases = [(1, 1000, 4, 1, 64, "bf16"), (1, 2048, 8, 1, 128, "bf16"), (2, 513, 6, 2, 64, "fp32"), (1, 1000, 4, 1, 64, "bf16")]
    data = []
    for i, (m, tokens, heads, kv, hd, dtype) in enumerate(cases):
        x = _attn_case(m, tokens, heads, kv, hd, dtype, seed=i)
        data.append((*x, _randn(_gen(10 + i), m, tokens, heads, hd).to(_t(dtype)), _starts([3, tokens // 2, tokens], m)[1]))

    def both(q, k, v, dout, seq, **kw):
        out, lse = b.attention(q, k, v, seq, **kw)
        return (out, lse, *b.attention_grad(dout, q, k, v, out, lse, seq, **kw))

    want = [both(*d) for d in data]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [both(*d, stream=s) for d, s in zip(data, streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, r) for p, r in zip(g, w))
    b.device_status()


# ---- gradient clipping ----------------------------------------------------------------------------------------------

def _clip_check(grads, max_norm, norm, got, before):
    """before: the gradients as they were; got: results."""
    import torch
    m = before[0].shape[0]
    total = torch.zeros(m, dtype=torch.float64, device="cuda")
    for t in before:
        total += t.double().square().flatten(1).sum(1)
    want = total.sqrt()
    # 8 squares, 3 additions and the fp32 result: halved by the root
    _within(norm, want, 7 * U * want + 1e-45, "norm")
    for i in range(m):
        by = 1.0 if float(want[i]) <= max_norm else max_norm / float(want[i])
        for t, o in zip(before, got):
            w = t[i].double() * by
            half = 2.0 ** -8 if o.dtype == torch.bfloat16 else U
            small = 2.0 ** -134 if o.dtype == torch.bfloat16 else 2.0 ** -150          # half a step of the smallest numbers
            _within(o[i], w, (9 * U + half) * w.abs() + small, "out")


CLIP_SHAPES = [[(1,)], [(7,), (3, 5)], [(8192,)], [(8193,), (1,), (0,), (16384,)], [(250, 251), (64,), (1000, 33)],
               [(3,)] * 70 + [(4099,)], [(2,)] * 1203, [(0,), (5,), (0,)]]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m", [1, 3])
@pytest.mark.parametrize("case", range(len(CLIP_SHAPES)))
def test_clip_grads(case, m, dtype):
    import torch
    from paper_1810_08313_b200 import binding as b
    g = _gen(case)
    shapes = CLIP_SHAPES[case]
    for by in (0.3, 1.5):
        grads = [(0.1 * _randn(g, m, *s)).to(_t(dtype)) for s in shapes]
        before = [t.clone() for t in grads]
        total = math.sqrt(max(sum(float(t[i].double().square().sum()) for t in grads) for i in range(m)))
        for out_type in (None, "fp32", "bf16"):
            out = None if out_type is None else [torch.full_like(t, 7.0, dtype=_t(out_type)) for t in grads]
            norm = b.clip_grads(grads, by * total, out=out)
            _clip_check(grads, by * total, norm, grads if out is None else out, before)
            if out is not None:
                assert all(torch.equal(t, s) for t, s in zip(grads, before))
            elif by > 1:
                assert all(torch.equal(t, s) for t, s in zip(grads, before))
            for t, s in zip(grads, before):
                t.copy_(s)


def test_clip_grads_range_and_norm_only():
    """Squares beyond fp32 on both sides, zeros, infinities and NaN; each replica by itself."""
    import torch
    from paper_1810_08313_b200 import binding as b
    big, tiny = torch.full((2, 1000), 1e30, device="cuda"), torch.full((2, 9000), 1e-30, device="cuda")
    zero = torch.zeros(2, 20000, device="cuda")
    for t in (big, tiny):
        s = t.clone()
        norm = b.clip_grads([zero, t], math.inf)
        _clip_check([zero, t], math.inf, norm, [zero, t], [torch.zeros_like(zero), s])
        norm = b.clip_grads([zero, t], 1e-32)
        _clip_check([zero, t], float(torch.tensor(1e-32)), norm, [zero, t], [torch.zeros_like(zero), s])
    assert not bool(b.clip_grads([zero], 1.0).any()) and not bool(zero.any())
    x = torch.ones(3, 50, device="cuda")
    x[1, 7], x[2, 9] = float("nan"), float("inf")
    norm = b.clip_grads([x], 1.0)
    assert abs(float(norm[0]) - math.sqrt(50)) < 1e-5 and math.isnan(float(norm[1])) and math.isinf(float(norm[2]))
    assert bool(torch.isfinite(x[0]).all()) and bool(torch.isnan(x[1]).all())
    assert bool(torch.isnan(x[2, 9])) and not bool(x[2, :9].any())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_clip_grads_of_views(dtype):
    """Replicas a distance apart, tensors that start on odd elements, and the elements between them untouched."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = _gen(4)
    base = _randn(g, 3, 60001).to(_t(dtype))
    keep = base.clone()
    views = [base[:, 1:20001], base[:, 20008:20008 + 96 * 200].unflatten(1, (96, 200)), base[:, 50000:50003]]
    before = [t.clone() for t in views]
    norm = b.clip_grads(views, 1.0)
    _clip_check(views, 1.0, norm, views, before)
    used = torch.zeros(60001, dtype=torch.bool, device="cuda")
    used[1:20001] = used[20008:20008 + 96 * 200] = used[50000:50003] = True
    assert torch.equal(base[:, ~used], keep[:, ~used])


def test_clip_grads_refusals():
    import torch
    from paper_1810_08313_b200 import binding as b
    x, y = torch.ones(2, 5, device="cuda"), torch.ones(2, 5, device="cuda")
    for call in (lambda: b.clip_grads([x, x], 1.0), lambda: b.clip_grads([x, y], 1.0, out=[y, y]), lambda: b.clip_grads([x], 1.0, out=[]),
                 lambda: b.clip_grads([x, x.double()], 1.0), lambda: b.clip_grads([x, y[:1]], 1.0), lambda: b.clip_grads([x, y.cpu()], 1.0),
                 lambda: b.clip_grads([x.t()], 1.0), lambda: b.clip_grads([x], 1.0, out=[y[:, :3]]), lambda: b.clip_grads([x[0, 0]], 1.0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(b.LsError):
        b.clip_grads([x], 0.0)
    assert bool((x == 1).all()) and bool((y == 1).all())


def test_clip_grads_is_repeatable_and_captured():
    import torch
    from paper_1810_08313_b200 import binding as b
    g = _gen(6)
    src = [[_randn(g, 2, n) for n in (100003, 64, 70000)] for _ in range(2)]
    out = [torch.zeros_like(t) for t in src[0]]
    want = []
    for s in src:
        norm = b.clip_grads(s, 2.0, out=out)
        want.append([norm.clone()] + [t.clone() for t in out])
    for _ in range(3):
        norm = b.clip_grads(src[0], 2.0, out=out)
        assert all(torch.equal(i, j) for i, j in zip([norm] + out, want[0]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm = b.clip_grads(src[1], 2.0, out=out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(i, j) for i, j in zip([norm] + out, want[1]))
    x = [t.clone() for t in src[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = b.clip_grads(x, 2.0, out=out)
    for i in (1, 0):
        for t, s in zip(x, src[i]):
            t.copy_(s)
        graph.replay()
        assert all(torch.equal(p, w) for p, w in zip([norm] + out, want[i]))


# ---- all of them, as a job uses them -----------------------------------------------------------------------------------

def test_a_training_step_of_one_block():
    """Two replicas of one attention block under a cross entropy: every gradient against automatic differentiation in 64 bits,
    then clipping, the momentum step and the averaging step.  fp32, so that the two agree to some 1e-5 of each gradient's norm
    (bound: 3e-4, products of 64 to 300 terms through six operators)."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, tokens, heads, kv, hd, d, vocab = 2, 150, 4, 2, 32, 96, 300
    g = _gen(1)
    rows, seq = _starts([0, 60, 140], m)
    pos = torch.cat([torch.arange(e - a) for a, e in zip([0, 60, 140], [60, 140, 150])]).int().cuda().expand(m, -1).contiguous()
    freq = b.rope_frequencies(hd)
    x = _randn(g, m, tokens, d)
    wqkv, wo = _randn(g, m, (heads + 2 * kv) * hd, d) / 8, _randn(g, m, d, heads * hd) / 8
    W = _randn(g, m, vocab, d) / 8
    ln, qw, kw = 1 + 0.1 * _randn(g, m, d), 1 + 0.1 * _randn(g, m, hd), 1 + 0.1 * _randn(g, m, hd)
    labels = torch.randint(0, vocab, (m, tokens), generator=g, device="cuda", dtype=torch.int32)
    labels[:, 140:] = -1

    def cut(t):
        a, e = heads * hd, (heads + kv) * hd
        return t[..., :a].unflatten(-1, (heads, hd)), t[..., a:e].unflatten(-1, (kv, hd)), t[..., e:].unflatten(-1, (kv, hd))

    # the framework's operators; plain products of the projections between them
    qkv = x @ wqkv.transpose(1, 2)
    q, k, v = cut(qkv)
    qr, kr = b.qk_norm_rope(q, k, qw, kw, pos, freq)
    o, lse = b.attention(qr, kr, v, seq)
    y = x + o.flatten(2) @ wo.transpose(1, 2)
    h, mean, rstd = b.layer_norm(y, ln)
    loss, _, _, dh, dW = b.vocab_loss_grad(h, W, labels)
    dy, dln, _ = b.layer_norm_grad(dh, y, ln, mean, rstd)
    do = (dy @ wo).view(m, tokens, heads, hd)
    dwo = dy.transpose(1, 2) @ o.flatten(2)
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = cut(dqkv)
    dqr, dkr, _ = b.attention_grad(do, qr, kr, v, o, lse, seq, dv=dv)
    _, _, dqw, dkw = b.qk_norm_rope_grad(dqr, dkr, q, k, qw, kw, pos, freq, dq=dq, dk=dk)
    dwqkv = dqkv.transpose(1, 2) @ x
    grads = [dwqkv, dwo, dW, dln, dqw, dkw]
    # the same in 64 bits
    leaves = [t.double().requires_grad_() for t in (wqkv, wo, W, ln, qw, kw)]
    w1, w2, w3, l64, a64, c64 = leaves
    total = 0.0
    for r in range(m):
        q6, k6, v6 = cut(x[r].double() @ w1[r].T)
        angle = pos[r].double()[:, None, None] * freq

        def turn(t, w):
            z = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
            a, e = z[..., :hd // 2], z[..., hd // 2:]
            return torch.cat((a * angle.cos() - e * angle.sin(), a * angle.sin() + e * angle.cos()), -1)

        q6, k6 = turn(q6, a64[r]), turn(k6, c64[r])
        see = _mask(tokens, rows[r])
        s = torch.einsum("ihd,jhd->hij", q6, k6.repeat_interleave(heads // kv, 1)) / math.sqrt(hd)
        p = torch.softmax(s.masked_fill(~see, -1e30), -1) * see
        o6 = torch.einsum("hij,jhd->ihd", p, v6.repeat_interleave(heads // kv, 1)).flatten(1)
        y6 = x[r].double() + o6 @ w2[r].T
        h6 = torch.nn.functional.layer_norm(y6, (d,)) * l64[r]
        total = total + torch.nn.functional.cross_entropy(h6 @ w3[r].T, labels[r].long(), ignore_index=-1)
    total.backward()
    for got, leaf in zip(grads, leaves):
        assert float((got - leaf.grad).norm() / leaf.grad.norm()) < 3e-4
    before = [t.clone() for t in grads]
    norm = b.clip_grads(grads, 0.05)
    _clip_check(grads, float(torch.tensor(0.05)), norm, grads, before)
    for w, gr in ((wqkv, grads[0]), (wo, grads[1])):
        vel = torch.zeros_like(w)
        b.muon_step(w, vel, gr, lr=0.02)
        b.average_flat(w.view(-1), m, w[0].numel())
        assert torch.equal(w[0], w[1]) and bool(torch.isfinite(w).all())
    b.device_status()
