"""Paths of the operators beside the plain call: on a handle's weights, replica by replica, in pieces, with failures."""
import math

import numpy as np
import pytest

from oracle import localsgd_oracle as orc
from paper_1810_08313_b200 import workloads as wl
from tests.helpers import f32, max_rel_err_per_tensor, small_problem, tensor_slices, to_device

pytestmark = pytest.mark.gpu


# ---- the momentum step on a handle's weights -----------------------------------------------------------------------

def _newton(u):
    import torch
    x = u / (torch.linalg.norm(u) + 1e-7)
    x = x.T if u.shape[0] > u.shape[1] else x
    for _ in range(5):
        a = x @ x.T
        x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
    return x.T if u.shape[0] > u.shape[1] else x


@pytest.mark.parametrize("gdtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dims,dtype,B,layer", [
    ((24, 40, 10), "fp32", 8, 1),                # CUDA-core layers
    ((256, 384, 128, 10), "fp32", 128, 0),       # tensor-core layers of an fp32 model: row-major, read from the synchronized copy
    ((256, 384, 128, 10), "fp32", 128, 1),
    ((384, 512, 256, 10), "bf16", 256, 0),       # blocked matrices with their operand copies, tall and wide
    ((384, 512, 256, 10), "bf16", 256, 1),
    ((384, 512, 256, 10), "bf16", 256, 2),       # the narrow output layer
    ((200, 136, 72, 10), "bf16", 48, 1),         # row-major matrices with operand copies
])
def test_muon_step_of_a_handles_layer(dims, dtype, B, layer, gdtype):
    """After set_params and after an averaging step, when the handle knows its replicas to be equal: the step's weights and
    momentum against 64 bits, every other tensor untouched, and local steps that go on from them as a handle does that was
    given the same state from the host."""
    import torch
    from paper_1810_08313_b200.binding import LocalSGD
    m, bf = 3, dtype == "bf16"
    spec, X, y, x1 = small_problem(dims, "softmax_ce", True, 1024, 31, bf16=bf)
    xd, yd = to_device(X, y, bf16=bf)
    offs = wl.batch_row_offsets(3, 4, m, 1024, B)
    eng, other = [LocalSGD(m, dims, gemm_dtype=dtype, lr=0.05, momentum=0.9, batch=B) for _ in range(2)]
    for e in (eng, other):
        e.bind_dataset(xd, yd)
    eng.set_params(x1)
    rows, cols = dims[layer + 1], dims[layer]
    mine = dict(tensor_slices(dims, True))[f"W{layer + 1}"]
    gen = torch.Generator(device="cuda").manual_seed(5)
    lr, mu = 0.3, 0.95
    for turn in range(2):
        g = torch.randn(m, rows, cols, generator=gen, device="cuda").to(torch.bfloat16 if gdtype == "bf16" else torch.float32)
        p0, v0 = eng.get_all()
        assert np.array_equal(p0[0], p0[1])
        eng.muon_step(layer, g, lr=lr, momentum=mu)
        p1, v1 = eng.get_all()
        for i in range(m):
            g64 = g[i].double()
            v64 = f32(mu) * torch.from_numpy(v0[i][mine]).cuda().double().view(rows, cols) + g64
            w64 = torch.from_numpy(p0[i][mine]).cuda().double().view(rows, cols) - \
                f32(lr) * math.sqrt(max(1.0, rows / cols)) * _newton(g64 + f32(mu) * v64)
            # v: two roundings.  w: five steps turn the products' 2^-22 into at most 4^5 of it, relative to the norm of O
            assert float((torch.from_numpy(v1[i][mine]).cuda().double().view(rows, cols) - v64).abs().max()) \
                <= 2.0 ** -22 * float(v64.abs().max())
            err = torch.linalg.norm(torch.from_numpy(p1[i][mine]).cuda().double().view(rows, cols) - w64)
            assert float(err) <= lr * math.sqrt(max(1.0, rows / cols) * min(rows, cols)) * 2.0 ** -12 + 2.0 ** -23 * float(w64.norm())
            keep = np.ones(p0.shape[1], dtype=bool)
            keep[mine] = False
            assert np.array_equal(p1[i][keep], p0[i][keep]) and np.array_equal(v1[i][keep], v0[i][keep])
        losses = []
        for e in (eng, other):
            if e is other:
                for i in range(m):
                    e.set_state(i, p1[i], v1[i])
            out = torch.zeros(2, m, device="cuda")
            e.local_steps(2, offs[2 * turn:2 * turn + 2], out)
            e.sync()
            losses.append(out.cpu().numpy())
        assert np.array_equal(losses[0], losses[1])
        for a, c in zip(eng.get_all(), other.get_all()):
            assert np.array_equal(a, c)
        for i in range(m):
            r0 = int(offs[2 * turn, i])
            want, grad = orc.loss_and_grad(spec, p1[i], X[r0:r0 + B], y[r0:r0 + B])
            assert abs(losses[0][0, i] - want) <= (2e-2 if bf else 1e-5) * want
            if not bf:
                step = p1[i] - f32(0.05) * (f32(0.9) * v1[i].astype(np.float64) + grad)
                r1 = int(offs[2 * turn + 1, i])
                want = orc.batch_loss(spec, step.astype(np.float32), X[r1:r1 + B], y[r1:r1 + B])
                assert abs(losses[0][1, i] - want) <= 1e-4 * want
        eng.average()
    eng.sync()
    with pytest.raises(ValueError):
        eng.muon_step(len(dims) - 1, g, lr=lr)
    with pytest.raises(ValueError):
        eng.muon_step(layer, g[:, :-1], lr=lr)
    eng.close()
    other.close()


@pytest.mark.parametrize("gdtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dims,dtype,B", [((384, 512, 256, 10), "bf16", 256), ((24, 40, 10), "fp32", 8)])
def test_muon_step_of_a_handles_layer_from_strided_gradients(dims, dtype, B, gdtype):
    """Gradients with gaps between the replicas and an odd start take the element-wise reads: the bits of a dense call."""
    import torch
    from paper_1810_08313_b200.binding import LocalSGD
    m, rows, cols = 2, dims[1], dims[0]
    x1 = wl.random_mlp_point(3, dims, True)
    g = torch.randn(m, rows, cols, device="cuda").to(torch.bfloat16 if gdtype == "bf16" else torch.float32)
    gap = rows * cols + 7
    buf = torch.zeros(m * gap + 1, device="cuda", dtype=g.dtype)
    apart = torch.as_strided(buf, (m, rows, cols), (gap, cols, 1), 1)
    apart.copy_(g)
    got = []
    for grad in (g, apart):
        eng = LocalSGD(m, dims, gemm_dtype=dtype, lr=0.05, momentum=0.9, batch=B)
        eng.set_params(x1)
        for _ in range(2):
            eng.muon_step(0, grad, lr=0.1, nesterov=False)
        got.append(eng.get_all())
        eng.close()
    for a, c in zip(*got):
        assert np.array_equal(a, c)


def test_muon_step_of_a_handles_layer_in_a_capture_is_refused():
    """A replay would change the weights behind the handle's back, after an averaging step for instance.  Nothing is captured, and the
    handle goes on."""
    import torch
    from paper_1810_08313_b200 import binding as b
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        eng = b.LocalSGD(2, (24, 40, 10), lr=0.1, momentum=0.9, batch=8, stream=stream)
        gr = torch.randn(2, 40, 24, device="cuda")
        ws = torch.empty(b.orthogonalize_workspace(2, 40, 24), device="cuda", dtype=torch.uint8)
        eng.set_params(np.linspace(-1, 1, eng.P, dtype=np.float32))
        eng.muon_step(0, gr, lr=0.1, workspace=ws)
        before = eng.get_all()
    g = torch.cuda.CUDAGraph()
    out = torch.zeros(4, device="cuda")
    with torch.cuda.graph(g, stream=stream):
        out += 1.0
        with pytest.raises(b.LsError) as e:
            eng.muon_step(0, gr, lr=0.1, workspace=ws)
        assert e.value.code == b.LS_ERR_UNSUPPORTED
    g.replay()
    torch.cuda.synchronize()
    assert float(out.min()) == 1.0
    for a, c in zip(before, eng.get_all()):
        assert np.array_equal(a, c)
    eng.muon_step(0, gr, lr=0.1, workspace=ws)
    assert not np.array_equal(eng.get_all()[0], before[0])
    eng.close()


# ---- sizes beyond a C int ------------------------------------------------------------------------------------------

def test_sizes_beyond_32_bits_are_refused():
    import torch
    from paper_1810_08313_b200 import binding as b
    big = 2 ** 32 + 8
    wide = torch.empty(big, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(8, device="cuda")
    for call in (lambda: b.layer_norm(wide.view(1, big), w), lambda: b.layer_norm(wide.view(big, 1, 1), w),
                 lambda: b.orthogonalize(wide.view(big, 1), out=wide.view(big, 1)),
                 lambda: b.orthogonalize(wide.view(1, big), out=wide.view(1, big))):
        with pytest.raises(b.LsError) as e:
            call()
        assert e.value.code == b.LS_ERR_TOO_LARGE
    with pytest.raises(b.LsError) as e:
        b.orthogonalize(torch.randn(8, 8, device="cuda"), steps=2 ** 32 + 5)
    assert e.value.code == b.LS_ERR_INVALID_ARG
    buf = torch.empty(4096, device="cuda", dtype=torch.uint8)
    with pytest.raises(b.LsError) as e:
        b.orthogonalize(torch.randn(8, 8, device="cuda"), workspace=buf[1:100])
    assert e.value.code == b.LS_ERR_STATE_SIZE
    torch.cuda.empty_cache()


# ---- a wait that runs out ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("side", [False, True])
def test_wait_that_runs_out_is_reported_once_and_operators_go_on(side):
    """A kernel of one thread waits about a millisecond on a barrier on which nothing arrives and records it, as an operator
    would.  device_status() raises once; results before and after are the same bits, and a handle's own record stays clear."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2, 90, 72, generator=g, device="cuda")
    w = torch.ones(2, 72, device="cuda")
    W = torch.randn(2, 200, 72, generator=g, device="cuda") / 8
    y = torch.randint(0, 200, (2, 90), generator=g, device="cuda").int()

    def run():
        n, mean, rstd = b.layer_norm(x, w)
        out = b.vocab_loss_grad(n, W, y)
        return (n, mean, rstd) + out + b.layer_norm_grad(out[3], x, w, mean, rstd) + (b.orthogonalize(out[4]),)

    ref = [t.clone() for t in run()]
    stream = torch.cuda.Stream() if side else None
    b.device_status(stream)
    eng = b.LocalSGD(2, (24, 16, 10), lr=0.1, momentum=0.9, batch=8)
    b.selftest_device_timeout(2_000_000, stream)
    with pytest.raises(b.LsError) as e:
        b.device_status(stream)
    assert e.value.code == b.LS_ERR_DEVICE_TIMEOUT
    b.device_status(stream)
    b.device_status()
    eng.sync()
    # not asked for: calls go on, the record waits
    b.selftest_device_timeout(2_000_000, stream)
    got = run()
    torch.cuda.synchronize()
    with pytest.raises(b.LsError):
        b.device_status()
    b.device_status()
    for t, r in zip(got, ref):
        assert torch.equal(t, r)
    # the handle's record is another one
    eng.selftest_wait_timeout(2_000_000)
    torch.cuda.synchronize()
    b.device_status()
    with pytest.raises(b.LsError):
        eng.sync()
    eng.close()


# ---- cross entropy: replicas one after another, pieces of rows, strides, outputs left out ---------------------------

def _vocab(m, rows, d, V, dtype, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    h = torch.randn(m, rows, d, generator=g, device="cuda").to(dt)
    W = (torch.randn(m, V, d, generator=g, device="cuda") / math.sqrt(d)).to(dt)
    y = torch.randint(0, V, (m, rows), generator=g, device="cuda")
    y[torch.rand((m, rows), generator=g, device="cuda") < 0.1] = -1
    return h, W, y.int()


@pytest.mark.parametrize("dtype,m,rows,d,V", [
    ("bf16", 2, 2300, 64, 65536),          # one piece a replica, together beyond 512 MB: one replica after another
    ("bf16", 3, 1500, 65, 65536),          # ... with operands laid out anew
    ("fp32", 2, 600, 24, 65536),
    ("bf16", 2, 4400, 32, 131072),         # two pieces a replica
    ("fp32", 2, 1100, 13, 131072),
])
def test_replicas_one_after_another(dtype, m, rows, d, V):
    """Each replica is the bits of a call of its own: the statistics, counters and operand copies of one are not seen by the next.
    The losses also without a gradient."""
    import torch
    from paper_1810_08313_b200 import binding as b
    h, W, y = _vocab(m, rows, d, V, dtype, seed=rows)
    y[1, -7:] = -1
    out = b.vocab_loss_grad(h, W, y, scale=1.5)
    for i in range(m):
        one = b.vocab_loss_grad(h[i], W[i], y[i], scale=1.5)
        for got, want in zip(out, one):
            assert torch.equal(got[i], want.view_as(got[i]))
    plain = b.vocab_loss(h, W, y)
    for i in range(m):
        for got, want in zip(plain, b.vocab_loss(h[i], W[i], y[i])):
            assert torch.equal(got[i], want.view_as(got[i]))
        keep = y[i] >= 0
        want = out[1][i].double().sum() / int(keep.sum())
        assert abs(float(out[0][i]) - float(want)) <= 2.0 ** -23 * abs(float(want))
        assert bool((out[1][i][~keep] == 0).all()) and float(out[3][i][~keep].abs().max()) == 0.0
    b.device_status()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,d,V", [("bf16", 64, 131072), ("fp32", 16, 131072), ("bf16", 65, 131072)])
def test_dh_of_every_piece_of_rows(dtype, d, V):
    """dh of the rows of the last piece, and of the first, as calls of those rows alone give it: apart from 1 / count, whose
    rounding and product are 2^-23, and the output's rounding on both sides (an fp32 sum over V cut another way: 2^-18 of the
    absolute sum, checked against the largest entry of the row)."""
    import torch
    from paper_1810_08313_b200 import binding as b
    rows = (2 ** 29 if dtype == "bf16" else 2 ** 27) // V + 300
    h, W, y = _vocab(1, rows, d, V, dtype, seed=5)
    _, _, _, dh, _ = b.vocab_loss_grad(h, W, y, scale=float((y >= 0).sum()))
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for part in (slice(0, 256), slice(rows - 256, rows)):
        hp, yp = h[:, part].contiguous(), y[:, part].contiguous()
        want = b.vocab_loss_grad(hp, W, yp, scale=float((yp >= 0).sum()))[3].double()
        err = (dh[:, part].double() - want).abs()
        tol = (2 * half + 2.0 ** -22) * want.abs() * 1.01 + 2.0 ** -16 * want.abs().amax(-1, keepdim=True)
        assert bool((err <= tol).all()), float((err / tol.clamp(min=1e-30)).max())
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_more_rows_than_one_launch_of_dz_takes(dtype):
    """A piece of more than 65280 rows: dz is formed by two launches.  Rows on both sides of the border and the last ones against
    64 bits, and dW of the whole (the sum over 65700 rows: u-relative bounds as in the tests of the gradient)."""
    import torch
    from paper_1810_08313_b200 import binding as b
    rows, d, V = 65700, 40, 130
    h, W, y = _vocab(1, rows, d, V, dtype, seed=8)
    y[0, 65270:65275] = -1
    n = int((y >= 0).sum())
    loss, rl, lse, dh, dW = b.vocab_loss_grad(h, W, y, scale=float(n))
    z = h[0].double() @ W[0].double().T
    l64 = torch.logsumexp(z, 1)
    keep = y[0] >= 0
    at = y[0].long().clamp(min=0)[:, None]
    assert bool(((lse[0].double() - l64).abs() <= 2.0 ** -18 * (1 + l64.abs())).all())
    want = torch.where(keep, l64 - z.gather(1, at)[:, 0], 0.0)
    assert bool(((rl[0].double() - want).abs() <= 2.0 ** -16 * (1 + want)).all())
    assert abs(float(loss[0]) - float(want.sum()) / n) <= 2.0 ** -18 * float(want.sum()) / n
    dz = torch.softmax(z, 1).scatter_add_(1, at, torch.full_like(l64, -1.0)[:, None]) * keep[:, None]
    # dz: 2^-11 and 2^-8 (bf16) or the logits' 2^-16; then one rounding of the sum
    one = 2.0 ** -11 + 2.0 ** -8 + 2.0 ** -15 if dtype == "bf16" else 2.0 ** -15
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    for got, a, o in ((dh[0], dz, W[0].double()), (dW[0], dz.T, h[0].double())):
        want = a @ o
        tol = (one + 2.0 ** -15) * (a.abs() @ o.abs()) + half * want.abs()
        assert bool(((got.double() - want).abs() <= tol).all())


def test_loss_of_a_vocabulary_whose_rows_come_in_pieces():
    """Without a gradient a piece is 2^31 logits or 256 rows: two pieces of 300 rows over more than 2^23 columns, each row with the
    bits of a call of its piece alone."""
    import torch
    from paper_1810_08313_b200 import binding as b
    h, W, y = _vocab(1, 300, 8, 2 ** 23 + 77, "bf16", seed=1)
    loss, rl, lse = b.vocab_loss(h, W, y)
    for part in (slice(0, 256), slice(256, 300)):
        _, r, l = b.vocab_loss(h[:, part].contiguous(), W, y[:, part].contiguous())
        assert torch.equal(r, rl[:, part]) and torch.equal(l, lse[:, part])
    want = rl.double().sum() / int((y >= 0).sum())
    assert abs(float(loss) - float(want)) <= 2.0 ** -23 * float(want)


@pytest.mark.parametrize("dtype,d", [("bf16", 96), ("bf16", 97), ("fp32", 96), ("fp32", 33)])
@pytest.mark.parametrize("rows", [3, 12, 30])
def test_few_rows_of_replicas_apart(rows, dtype, d):
    """Replicas with gaps between them give the bits of dense ones, and the gaps stay as they were."""
    import torch
    from paper_1810_08313_b200 import binding as b
    m, V = 2, 301
    h, W, y = _vocab(m, rows, d, V, dtype, seed=rows)
    ref, plain = b.vocab_loss_grad(h, W, y), b.vocab_loss(h, W, y)
    gaps = [rows * d + (64 if d % 8 == 0 else 67), V * d + (128 if d % 8 == 0 else 133)]
    bufs = [torch.full((m * g,), 5.0, device="cuda", dtype=h.dtype) for g in gaps * 2]
    views = [torch.as_strided(t, (m, n, d), (g, d, 1)) for t, g, n in zip(bufs, gaps * 2, (rows, V) * 2)]
    views[0].copy_(h)
    views[1].copy_(W)
    got = b.vocab_loss_grad(views[0], views[1], y, dh=views[2], dW=views[3])
    for t, r in zip(got, ref):
        assert torch.equal(t, r)
    for t, r in zip(b.vocab_loss(views[0], views[1], y), plain):
        assert torch.equal(t, r)
    for t, g, n in zip(bufs, gaps * 2, (rows, V) * 2):
        flat = torch.ones_like(t, dtype=torch.bool)
        torch.as_strided(flat, (m, n, d), (g, d, 1)).fill_(False)
        assert bool((t[flat] == 5.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 12, 70])
def test_row_outputs_left_out(rows, dtype):
    """row_loss, lse, mean, rstd and dbias may be null at the C entry: the rest keeps its bits."""
    import torch
    from paper_1810_08313_b200 import binding as b
    lib = b._lib()
    m, d, V = 2, 72, 301
    code = {"fp32": 0, "bf16": 1}[dtype]
    h, W, y = _vocab(m, rows, d, V, dtype, seed=rows)
    ref, plain = b.vocab_loss_grad(h, W, y), b.vocab_loss(h, W, y)
    st = torch.cuda.current_stream().cuda_stream
    ws = torch.empty(b.vocab_loss_workspace(m, rows, V, d, dtype, True), device="cuda", dtype=torch.uint8)
    base = (ws.data_ptr() + 255) // 256 * 256
    nb = ws.numel() - 256
    loss, dh, dW = torch.full((m,), 9.0, device="cuda"), torch.empty_like(h), torch.empty_like(W)
    assert lib.ls_vocab_loss_grad(h.data_ptr(), W.data_ptr(), y.data_ptr(), m, rows, V, d, rows * d, V * d, code, 1.0,
                                  loss.data_ptr(), None, None, dh.data_ptr(), rows * d, dW.data_ptr(), V * d, base, nb, st) == b.LS_OK
    assert torch.equal(loss, ref[0]) and torch.equal(dh, ref[3]) and torch.equal(dW, ref[4])
    loss.fill_(9.0)
    assert lib.ls_vocab_loss(h.data_ptr(), W.data_ptr(), y.data_ptr(), m, rows, V, d, rows * d, V * d, code, loss.data_ptr(), None,
                             None, base, nb, st) == b.LS_OK
    assert torch.equal(loss, plain[0])
    w = torch.ones(m, d, device="cuda")
    yy, mean, rstd = b.layer_norm(h, w)
    out = torch.empty_like(h)
    assert lib.ls_layer_norm(h.data_ptr(), w.data_ptr(), None, m, rows, d, rows * d, d, code, 1e-5, out.data_ptr(), rows * d, None,
                             None, st) == b.LS_OK
    assert torch.equal(out, yy)
    dx, dw, _ = b.layer_norm_grad(yy, h, w, mean, rstd)
    dx2, dw2 = torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(b.layer_norm_grad_workspace(m, rows, d), device="cuda", dtype=torch.uint8)
    base = (ws.data_ptr() + 255) // 256 * 256
    assert lib.ls_layer_norm_grad(yy.data_ptr(), h.data_ptr(), w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), m, rows, d, rows * d,
                                  rows * d, d, code, dx2.data_ptr(), rows * d, dw2.data_ptr(), None, d, base, ws.numel() - 256,
                                  st) == b.LS_OK
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw)
