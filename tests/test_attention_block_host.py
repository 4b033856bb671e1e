"""Refusals and workspace sizes of head norm with rotation, attention and gradient clipping: answered before any CUDA call."""
import ctypes as C
import math

import pytest

from paper_1810_08313_b200 import binding as b

OK, INV, BIG, WS = b.LS_OK, b.LS_ERR_INVALID_ARG, b.LS_ERR_TOO_LARGE, b.LS_ERR_STATE_SIZE
P = 1 << 20            # a non-null, well-aligned address that no refused call looks at


def _bytes(name, *args):
    n = C.c_size_t()
    return getattr(b._lib(), name)(*args, C.byref(n)), n.value


def test_workspace_sizes():
    rc, n = _bytes("ls_qk_norm_rope_grad_ws_bytes", 2, 100, 64)
    assert rc == OK and n >= 2 * 2 * 64 * 4
    assert _bytes("ls_qk_norm_rope_grad_ws_bytes", 1, 0, 64)[0] == OK
    rc, n = _bytes("ls_attention_grad_ws_bytes", 2, 100, 8, 2, 64)
    assert rc == OK and n >= 2 * 100 * 8 * 4
    assert n < 2 * 8 * 100 * 100 * 2                          # no scores
    assert _bytes("ls_attention_grad_ws_bytes", 1, 0, 8, 2, 64)[0] == OK
    sizes = (C.c_int64 * 3)(5, 0, 1 << 20)
    rc, n = _bytes("ls_clip_grads_ws_bytes", sizes, 3, 4)
    assert rc == OK and n >= 4 * 8
    assert _bytes("ls_clip_grads_ws_bytes", None, 0, 1)[0] == OK
    assert b.qk_norm_rope_grad_workspace(1, 10, 64) > 0 and b.attention_grad_workspace(1, 10, 2, 1, 64) > 0
    assert b.clip_grads_workspace([10, 20], 2) > 0
    lib = b._lib()
    assert lib.ls_qk_norm_rope_grad_ws_bytes(1, 1, 8, None) == INV
    assert lib.ls_attention_grad_ws_bytes(1, 1, 1, 1, 8, None) == INV
    assert lib.ls_clip_grads_ws_bytes(sizes, 3, 1, None) == INV


def test_frequencies():
    f = b.rope_frequencies(8, 100.0, device="cpu")
    assert [abs(float(x) - 100.0 ** (-p / 4)) < 1e-15 for p, x in enumerate(f)] == [True] * 4
    assert b.rope_frequencies(0, device="cpu").numel() == 0
    with pytest.raises(ValueError):
        b.rope_frequencies(3, device="cpu")


def _rope(q=P, k=P, qw=P, kw=P, pos=P, freq=P, m=2, tokens=3, heads=4, kv=2, hd=8, rot=8, inter=0, qr=32, kr=16, qs=96, ks=48, ws=8,
          dt=0, eps=1e-6, qo=P, ko=P, qor=32, kor=16, qos=96, kos=48):
    return b._lib().ls_qk_norm_rope(q, k, qw, kw, pos, freq, m, tokens, heads, kv, hd, rot, inter, qr, kr, qs, ks, ws, dt, eps, qo, ko,
                                    qor, kor, qos, kos, None)


def _rope_grad(gq=P, gk=P, q=P, k=P, qw=P, kw=P, pos=P, freq=P, m=2, tokens=3, heads=4, kv=2, hd=8, rot=8, inter=0, gqr=32, gkr=16,
               qr=32, kr=16, gqs=96, gks=48, qs=96, ks=48, ws=8, dt=0, eps=1e-6, dq=P, dk=P, dqr=32, dkr=16, dqs=96, dks=48, dqw=P,
               dkw=P, dws=8, wsp=P, nb=1 << 40):
    return b._lib().ls_qk_norm_rope_grad(gq, gk, q, k, qw, kw, pos, freq, m, tokens, heads, kv, hd, rot, inter, gqr, gkr, qr, kr, gqs,
                                         gks, qs, ks, ws, dt, eps, dq, dk, dqr, dkr, dqs, dks, dqw, dkw, dws, wsp, nb, None)


def test_qk_norm_rope_arguments():
    common = [dict(q=None), dict(k=None), dict(qw=None), dict(kw=None), dict(pos=None), dict(freq=None), dict(m=0), dict(tokens=-1),
              dict(heads=0), dict(kv=0), dict(hd=0), dict(rot=3), dict(rot=10), dict(rot=-2), dict(inter=2), dict(inter=-1),
              dict(qr=31), dict(kr=15), dict(qs=95), dict(ks=47), dict(ws=7), dict(dt=2), dict(dt=-1), dict(eps=-1.0),
              dict(eps=float("nan")), dict(eps=float("inf")), dict(q=P + 2), dict(k=P + 1), dict(qw=P + 2), dict(kw=P + 2),
              dict(pos=P + 2), dict(freq=P + 4), dict(dt=1, q=P + 1), dict(qr=1 << 60)]
    for kw in common:
        assert _rope(**kw) == INV, kw
        assert _rope_grad(**kw) == INV, kw
    for kw in (dict(qo=None), dict(ko=None), dict(qor=31), dict(kor=15), dict(qos=95), dict(kos=47), dict(qo=P + 2)):
        assert _rope(**kw) == INV, kw
    for kw in (dict(gq=None), dict(gk=None), dict(dq=None), dict(dk=None), dict(dqw=None), dict(dkw=None), dict(gqr=31), dict(gkr=15),
               dict(gqs=95), dict(gks=47), dict(dqr=31), dict(dkr=15), dict(dqs=95), dict(dks=47), dict(dws=7), dict(wsp=None),
               dict(dqw=P + 2), dict(dkw=P + 1)):
        assert _rope_grad(**kw) == INV, kw
    for kw in (dict(m=65536), dict(tokens=(1 << 30) + 1), dict(heads=65537), dict(hd=257)):
        assert _rope(**kw) == BIG, kw
        assert _rope_grad(**kw) == BIG, kw
    assert _rope_grad(nb=16) == WS and _rope_grad(wsp=P + 8) == WS


def _attn(q=P, k=P, v=P, seq=P, m=2, tokens=3, n=2, heads=4, kv=2, hd=8, qr=32, kr=16, vr=16, qs=96, ks=48, vs=48, dt=0, scale=1.0,
          out=P, outr=32, outs=96, lse=P):
    return b._lib().ls_attention(q, k, v, seq, m, tokens, n, heads, kv, hd, qr, kr, vr, qs, ks, vs, dt, scale, out, outr, outs, lse, None)


def _attn_grad(g=P, q=P, k=P, v=P, out=P, lse=P, seq=P, m=2, tokens=3, n=2, heads=4, kv=2, hd=8, gr=32, qr=32, kr=16, vr=16, outr=32,
               gs=96, qs=96, ks=48, vs=48, outs=96, dt=0, scale=1.0, dq=P, dk=P, dv=P, dqr=32, dkr=16, dvr=16, dqs=96, dks=48, dvs=48,
               wsp=P, nb=1 << 40):
    return b._lib().ls_attention_grad(g, q, k, v, out, lse, seq, m, tokens, n, heads, kv, hd, gr, qr, kr, vr, outr, gs, qs, ks, vs,
                                      outs, dt, scale, dq, dk, dv, dqr, dkr, dvr, dqs, dks, dvs, wsp, nb, None)


def test_attention_arguments():
    common = [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(lse=None), dict(seq=None), dict(m=0), dict(tokens=-1),
              dict(n=-1), dict(heads=0), dict(kv=0), dict(heads=3), dict(hd=0), dict(dt=2), dict(dt=-1), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(qr=31), dict(kr=15), dict(vr=15), dict(outr=31), dict(qs=95), dict(ks=47), dict(vs=47),
              dict(outs=95), dict(q=P + 2), dict(v=P + 1), dict(out=P + 2), dict(lse=P + 2), dict(seq=P + 2), dict(dt=1, k=P + 1),
              dict(kr=1 << 60)]
    for kw in common:
        assert _attn(**kw) == INV, kw
        assert _attn_grad(**kw) == INV, kw
    for kw in (dict(g=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(gr=31), dict(gs=95), dict(dqr=31), dict(dkr=15),
               dict(dvr=15), dict(dqs=95), dict(dks=47), dict(dvs=47), dict(dq=P + 2), dict(dk=P + 1), dict(wsp=None)):
        assert _attn_grad(**kw) == INV, kw
    for kw in (dict(m=65536), dict(tokens=(1 << 30) + 1), dict(heads=65538), dict(hd=257), dict(tokens=1 << 30, heads=65536, m=60000)):
        assert _attn(**kw) == BIG, kw
        assert _attn_grad(**kw) == BIG, kw
    assert _attn_grad(nb=16) == WS and _attn_grad(wsp=P + 8) == WS
    # nothing to do
    assert _attn(tokens=0) == OK and _attn_grad(tokens=0) == OK and _rope(tokens=0) == OK


def _clip(ptrs=(P, P), sizes=(5, 6), steps=(5, 6), types=(0, 1), n=None, m=2, most=1.0, outs=None, osteps=(5, 6), otypes=(0, 1), norm=P,
          ws=P, nb=1 << 40, **null):
    n = len(sizes) if n is None else n
    arr = {"p": (C.c_void_p * 2)(*ptrs), "n": (C.c_int64 * 2)(*sizes), "s": (C.c_int64 * 2)(*steps), "t": (C.c_int32 * 2)(*types),
           "o": None if outs is None else (C.c_void_p * 2)(*outs), "os": (C.c_int64 * 2)(*osteps), "ot": (C.c_int32 * 2)(*otypes)}
    for k in null:
        arr[k] = None
    return b._lib().ls_clip_grads(arr["p"], arr["n"], arr["s"], arr["t"], n, m, most, arr["o"], arr["os"], arr["ot"], norm, ws, nb, None)


def test_clip_grads_arguments():
    for kw in (dict(ptrs=(None, P)), dict(sizes=(-1, 6)), dict(steps=(4, 6)), dict(types=(2, 0)), dict(types=(-1, 0)), dict(n=-1),
               dict(m=0), dict(most=0.0), dict(most=-1.0), dict(most=float("nan")), dict(norm=None), dict(norm=P + 2), dict(ws=None),
               dict(ptrs=(P + 2, P)), dict(ptrs=(P, P + 1)), dict(p=1), dict(t=1), dict(s=1), dict(outs=(None, P)),
               dict(outs=(2 * P, 2 * P + 1)), dict(outs=(2 * P, 2 * P), osteps=(4, 6)), dict(outs=(2 * P, 2 * P), otypes=(3, 0)),
               dict(outs=(P, 2 * P), otypes=(1, 1)), dict(outs=(P, 2 * P), osteps=(6, 6)), dict(outs=(2 * P, 2 * P), ot=1),
               dict(outs=(2 * P, 2 * P), os=1)):
        assert _clip(**kw) == INV, kw
    assert _clip(m=65536, steps=(5, 6)) == BIG and _clip(sizes=((1 << 40) + 1, 6), steps=(1 << 41, 6)) == BIG
    assert _clip(nb=8) == WS and _clip(ws=P + 16) == WS


def test_wrappers_refuse_cpu_tensors():
    import torch
    x = torch.zeros(4, 2, 8)
    w, pos, f = torch.ones(8), torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.float64)
    for call in (lambda: b.qk_norm_rope(x, x, w, w, pos, f), lambda: b.qk_norm_rope_grad(x, x, x, x, w, w, pos, f),
                 lambda: b.attention(x, x, x), lambda: b.attention_grad(x, x, x, x, x, torch.zeros(2, 4)),
                 lambda: b.clip_grads([x], 1.0), lambda: b.clip_grads([], math.inf)):
        with pytest.raises(ValueError):
            call()
