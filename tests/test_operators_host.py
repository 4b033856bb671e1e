"""Refusals and workspace sizes of the operators on raw buffers: answered before any CUDA call (no GPU needed)."""
import ctypes as C

import pytest

from paper_1810_08313_b200 import binding as b

OK, INV, BIG, WS = b.LS_OK, b.LS_ERR_INVALID_ARG, b.LS_ERR_TOO_LARGE, b.LS_ERR_STATE_SIZE
P = 1 << 20            # a non-null, well-aligned address that no refused call looks at


def _bytes(name, *args):
    n = C.c_size_t()
    return getattr(b._lib(), name)(*args, C.byref(n)), n.value


def test_workspace_sizes():
    rc, n = _bytes("ls_layer_norm_grad_ws_bytes", 2, 100, 64)
    assert rc == OK and n >= 2 * 2 * 64 * 4
    assert _bytes("ls_layer_norm_grad_ws_bytes", 1, 0, 64)[0] == OK
    rc, loss = _bytes("ls_vocab_loss_ws_bytes", 1, 4096, 32000, 1024, 1, 0)
    rc2, grad = _bytes("ls_vocab_loss_ws_bytes", 1, 4096, 32000, 1024, 1, 1)
    assert rc == rc2 == OK
    assert loss < 4096 * 32000 * 2 / 16               # statistics, not logits
    assert 4096 * 32000 * 2 <= grad
    # the probabilities of a gradient are bounded whatever the number of rows
    rc, many = _bytes("ls_vocab_loss_ws_bytes", 1, 1 << 20, 131072, 1024, 1, 1)
    assert rc == OK and many < 3 * 2 ** 30
    assert _bytes("ls_vocab_loss_ws_bytes", 3, 0, 10, 8, 0, 1)[0] == OK
    rc, n = _bytes("ls_orthogonalize_ws_bytes", 2, 64, 100)
    assert rc == OK and n >= 2 * 2 * 2 * 64 * 100 * 2
    assert b.layer_norm_grad_workspace(1, 10, 10) > 0
    assert b.vocab_loss_workspace(1, 10, 10, 8, "fp32", True) > 0
    assert b.orthogonalize_workspace(1, 8, 8) > 0
    for name, args in [("ls_layer_norm_grad_ws_bytes", (1, 1, 1)), ("ls_vocab_loss_ws_bytes", (1, 1, 1, 1, 0, 0)),
                       ("ls_orthogonalize_ws_bytes", (1, 1, 1))]:
        assert getattr(b._lib(), name)(*args, None) == INV


@pytest.mark.parametrize("m,rows,d,want", [(0, 1, 8, INV), (1, -1, 8, INV), (1, 1, 0, INV), (1, 1, 16385, BIG),
                                           (65536, 1, 8, BIG), (1, 1 << 31, 8, BIG)])
def test_layer_norm_sizes(m, rows, d, want):
    lib = b._lib()
    n = rows * d if rows > 0 else 0
    assert lib.ls_layer_norm(P, P, P, m, rows, d, n, d, 0, 1e-5, P, n, P, P, None) == want
    assert lib.ls_layer_norm_grad(P, P, P, P, P, m, rows, d, n, n, d, 0, P, n, P, P, d, P, 1 << 40, None) == want
    assert _bytes("ls_layer_norm_grad_ws_bytes", m, rows, d)[0] == want


def test_layer_norm_arguments():
    lib = b._lib()

    def fwd(x=P, w=P, bias=P, m=2, rows=3, d=8, xs=24, ps=8, dt=0, eps=1e-5, y=P, ys=24, mean=P, rstd=P):
        return lib.ls_layer_norm(x, w, bias, m, rows, d, xs, ps, dt, eps, y, ys, mean, rstd, None)

    def bwd(dy=P, x=P, w=P, mean=P, rstd=P, m=2, rows=3, d=8, dys=24, xs=24, ps=8, dt=0, dx=P, dxs=24, dw=P, db=P, dps=8,
            ws=P, nb=1 << 30):
        return lib.ls_layer_norm_grad(dy, x, w, mean, rstd, m, rows, d, dys, xs, ps, dt, dx, dxs, dw, db, dps, ws, nb, None)

    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(dt=2), dict(dt=-1), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(xs=23), dict(ys=23), dict(ps=7), dict(x=P + 2), dict(w=P + 2), dict(mean=P + 1),
               dict(rstd=P + 2), dict(bias=P + 2), dict(y=P + 1), dict(dt=1, x=P + 1)):
        assert fwd(**kw) == INV, kw
    for kw in (dict(dy=None), dict(x=None), dict(w=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(dw=None),
               dict(ws=None), dict(dt=5), dict(dys=23), dict(xs=23), dict(dxs=23), dict(ps=7), dict(dps=7), dict(dx=P + 2),
               dict(dw=P + 2), dict(db=P + 3)):
        assert bwd(**kw) == INV, kw
    assert bwd(nb=16) == WS and bwd(ws=P + 4) == WS


@pytest.mark.parametrize("m,rows,vocab,d,want", [(0, 1, 8, 8, INV), (1, -1, 8, 8, INV), (1, 1, 0, 8, INV), (1, 1, 8, 0, INV),
                                                 (1, 1, (1 << 24) + 1, 8, BIG), (1, 1, 8, 65537, BIG),
                                                 (1, 1 << 31, 8, 8, BIG), (65536, 1, 8, 8, BIG)])
def test_vocab_loss_sizes(m, rows, vocab, d, want):
    lib = b._lib()
    hs, ws = max(rows, 0) * d, vocab * d
    assert lib.ls_vocab_loss(P, P, P, m, rows, vocab, d, hs, ws, 1, P, P, P, P, 1 << 50, None) == want
    assert lib.ls_vocab_loss_grad(P, P, P, m, rows, vocab, d, hs, ws, 1, 1.0, P, P, P, P, hs, P, ws, P, 1 << 50, None) == want
    assert _bytes("ls_vocab_loss_ws_bytes", m, rows, vocab, d, 1, 1)[0] == want


def test_vocab_loss_arguments():
    lib = b._lib()

    def grad(h=P, W=P, y=P, m=2, rows=4, V=16, d=8, hs=32, ws_=128, dt=1, scale=1.0, loss=P, rl=P, lse=P, dh=P, dhs=32, dW=P,
             dws=128, ws=P, nb=1 << 40):
        return lib.ls_vocab_loss_grad(h, W, y, m, rows, V, d, hs, ws_, dt, scale, loss, rl, lse, dh, dhs, dW, dws, ws, nb, None)

    def loss(h=P, W=P, y=P, m=2, rows=4, V=16, d=8, hs=32, ws_=128, dt=1, out=P, rl=P, lse=P, ws=P, nb=1 << 40):
        return lib.ls_vocab_loss(h, W, y, m, rows, V, d, hs, ws_, dt, out, rl, lse, ws, nb, None)

    for kw in (dict(h=None), dict(W=None), dict(y=None), dict(ws=None), dict(dt=2), dict(hs=31), dict(ws_=127), dict(hs=33),
               dict(ws_=129), dict(h=P + 2), dict(W=P + 8), dict(y=P + 2), dict(rl=P + 2), dict(lse=P + 1)):
        assert grad(**kw) == INV, kw
        assert loss(**kw) == INV, kw
    assert loss(out=None) == INV
    for kw in (dict(loss=None), dict(dh=None), dict(dW=None), dict(scale=float("nan")), dict(scale=float("inf")), dict(dhs=31),
               dict(dhs=33), dict(dws=120), dict(dws=129), dict(dh=P + 2), dict(dW=P + 2)):
        assert grad(**kw) == INV, kw
    assert grad(dt=0, h=P + 4) == INV                 # fp32 rows of whole 16 bytes start on one too
    assert grad(nb=64) == WS and loss(nb=64) == WS and grad(ws=P + 128) == WS


def test_orthogonalize_and_muon_arguments():
    lib = b._lib()

    def orth(u=P, m=2, r=8, c=8, us=64, dt=0, steps=5, out=P, os=64, ws=P, nb=1 << 40):
        return lib.ls_orthogonalize(u, m, r, c, us, dt, steps, out, os, ws, nb, None)

    def muon(w=P, v=P, g=P, m=2, r=8, c=8, s=64, vs=64, gs=64, dt=0, lr=0.1, mu=0.9, nest=1, steps=5, ws=P, nb=1 << 40):
        return lib.ls_muon_step(w, v, g, m, r, c, s, vs, gs, dt, lr, mu, nest, steps, ws, nb, None)

    for kw in (dict(u=None), dict(out=None), dict(ws=None), dict(m=0), dict(r=0), dict(c=0), dict(us=63), dict(os=63),
               dict(dt=2), dict(steps=0), dict(steps=65), dict(u=P + 2), dict(out=P + 2), dict(dt=1, u=P + 1)):
        assert orth(**kw) == INV, kw
    for kw in (dict(w=None), dict(v=None), dict(g=None), dict(ws=None), dict(m=0), dict(r=0), dict(c=-1), dict(s=63),
               dict(vs=63), dict(gs=63), dict(dt=-1), dict(lr=float("nan")), dict(mu=1.0), dict(mu=-0.1), dict(mu=float("nan")),
               dict(nest=2), dict(steps=0), dict(steps=65), dict(w=P + 2), dict(v=P + 1), dict(g=P + 2)):
        assert muon(**kw) == INV, kw
    assert orth(r=32769) == BIG and muon(c=32769) == BIG and orth(m=65536) == BIG
    assert orth(nb=8) == WS and muon(nb=8) == WS and orth(ws=P + 16) == WS and muon(ws=P + 16) == WS


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    x = torch.zeros(4, 8)
    for call in (lambda: b.layer_norm(x, x[0]), lambda: b.layer_norm_grad(x, x, x[0], x[:, 0], x[:, 0]),
                 lambda: b.vocab_loss(x, x, torch.zeros(4, dtype=torch.int32)),
                 lambda: b.vocab_loss_grad(x, x, torch.zeros(4, dtype=torch.int32)),
                 lambda: b.orthogonalize(x), lambda: b.muon_step(x, x, x, 0.1)):
        with pytest.raises(ValueError):
            call()


def test_muon_step_of_a_layer_needs_a_handle():
    lib = b._lib()
    assert lib.ls_muon_step_layer(None, 0, P, 64, 0, 0.1, 0.9, 1, 5, P, 1 << 40) == b.LS_ERR_BAD_HANDLE


class _FakeDeviceBytes:
    """What the wrapper looks at of a uint8 tensor on a GPU."""
    is_cuda = True

    def __init__(self, torch, device, start, numel):
        self.dtype, self.device, self._start, self._numel = torch.uint8, device, start, numel

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self._start

    def numel(self):
        return self._numel


@pytest.mark.parametrize("start,numel,want", [(P, 4096, (P, 4096)), (P + 1, 4096, (P + 256, 4096 - 255)), (P + 255, 1, (P + 256, 0)),
                                              (P + 1, 255, (P + 256, 0)), (P + 1, 254, None), (P + 1, 100, None), (P + 200, 3, None)])
def test_workspace_that_ends_before_its_first_aligned_byte(start, numel, want):
    """A view that holds no 256-byte boundary has no usable byte; its size must not wrap round to a huge one."""
    import torch
    op = object.__new__(b._Op)
    op.torch, op.device, op.stream, op.raw = torch, torch.device("cpu"), None, 0
    base, nbytes, _ = op.workspace(None, _FakeDeviceBytes(torch, op.device, start, numel), 64)
    assert base % 256 == 0
    assert (base, nbytes) == (want if want is not None else (P + 256, 0))
    assert b._lib().ls_orthogonalize(P, 1, 8, 8, 64, 0, 5, P, 64, base, nbytes, None) == WS      # needs more than 4096


def test_sizes_that_do_not_fit_a_c_int():
    """Their low 32 bits name another, smaller call."""
    big = 2 ** 32 + 8
    for call in (lambda: b.orthogonalize_workspace(1, big, 8), lambda: b.orthogonalize_workspace(1, 8, big),
                 lambda: b.orthogonalize_workspace(big, 8, 8), lambda: b.layer_norm_grad_workspace(1, 8, big),
                 lambda: b.layer_norm_grad_workspace(big, 8, 8), lambda: b.vocab_loss_workspace(big, 8, 8, 8),
                 lambda: b.vocab_loss_workspace(1, 8, 8, big), lambda: b.orthogonalize_workspace(1, 8 - 2 ** 32, 8)):
        with pytest.raises(b.LsError) as e:
            call()
        assert e.value.code == BIG
    for steps in (2 ** 32 + 5, 5 - 2 ** 32):
        with pytest.raises(b.LsError) as e:
            b._int32(steps, INV, "steps")
        assert e.value.code == INV


def test_selftest_of_the_report_path_refuses_limits():
    for limit in (0, -1, 2 * 10 ** 9 + 1):
        assert b._lib().ls_selftest_device_timeout(limit, None) == INV


def test_workspace_of_a_gradient_serves_the_loss():
    for m in (1, 2, 7):
        for rows in (0, 1, 3, 4, 5, 16, 17, 32, 33, 64, 300, 5000, 70000):
            for V in (1, 100, 301, 32000, 131072, 1 << 23):
                for d in (1, 8, 72, 77, 4096):
                    for dt in (0, 1):
                        loss, grad = (_bytes("ls_vocab_loss_ws_bytes", m, rows, V, d, dt, g) for g in (0, 1))
                        assert loss[0] == grad[0] == OK and grad[1] >= loss[1], (m, rows, V, d, dt)
