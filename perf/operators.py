"""Operators around the last layers and the weight update of a language model trained by local SGD, as measured cases.

A case is one call of one operator: layer norm and its gradient, the softmax cross entropy of a large output matrix
without stored logits and its gradient, the orthogonalisation of a matrix by Newton-Schulz products, and the momentum
step that uses it.  Every operator takes the replicas of a job packed in one tensor (first axis m), as the rest of the
package does.  `run` computes a case in plain torch, in 32 bits, or through the package's entry points (`own`).
"""
import math

import torch

own = False

EPS = 1e-5                             # layer norm
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315
NS_STEPS = 5
NS_EPS = 1e-7
LR, MOMENTUM = 0.02, 0.95

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def listed():
    return [
        # one decoding-sized batch of activations: the time of a call, not of its bytes
        {"name": "layer_norm few rows", "op": "layer_norm", "m": 1, "rows": 16, "d": 1024, "dtype": "bf16"},
        # four replicas' activations of an fp32 job, one row short of a power of two
        {"name": "layer_norm replicas fp32", "op": "layer_norm", "m": 4, "rows": 8191, "d": 2048, "dtype": "fp32"},
        # odd width and few rows, three replicas: the vector loads do not fit
        {"name": "layer_norm_grad odd fp32", "op": "layer_norm_grad", "m": 3, "rows": 777, "d": 1001, "dtype": "fp32"},
        # the tokens of one training step at a usual width
        {"name": "layer_norm_grad step", "op": "layer_norm_grad", "m": 1, "rows": 16384, "d": 4096, "dtype": "bf16"},
        # the loss of a handful of tokens: the output matrix is read once
        {"name": "vocab_loss few rows", "op": "vocab_loss", "m": 1, "rows": 64, "d": 1024, "vocab": 32000, "dtype": "bf16"},
        # validation loss of two replicas, odd vocabulary, ragged rows
        {"name": "vocab_loss odd replicas", "op": "vocab_loss", "m": 2, "rows": 2047, "d": 1024, "vocab": 50001, "dtype": "bf16"},
        # an fp32 job's small model: two replicas, all three sizes odd against the tiles
        {"name": "vocab_loss_grad odd fp32", "op": "vocab_loss_grad", "m": 2, "rows": 513, "d": 760, "vocab": 10007, "dtype": "fp32"},
        # a full training step's tokens against a large vocabulary: the largest case
        {"name": "vocab_loss_grad step", "op": "vocab_loss_grad", "m": 1, "rows": 8192, "d": 2048, "vocab": 65536, "dtype": "bf16"},
        # one small hidden matrix
        {"name": "orthogonalize small", "op": "orthogonalize", "m": 1, "rows": 256, "cols": 256, "dtype": "bf16"},
        # a tall matrix of odd sizes, two replicas
        {"name": "orthogonalize odd tall", "op": "orthogonalize", "m": 2, "rows": 2501, "cols": 1000, "dtype": "fp32"},
        # the wide matrix of a feed-forward block, two replicas with bf16 gradients
        {"name": "muon_step wide", "op": "muon_step", "m": 2, "rows": 1024, "cols": 4096, "dtype": "bf16"},
        # one hidden matrix of the eight replicas of a job
        {"name": "muon_step replicas", "op": "muon_step", "m": 8, "rows": 2048, "cols": 2048, "dtype": "fp32"},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["layer_norm", "layer_norm_grad", "vocab_loss", "vocab_loss_grad", "vocab_loss_grad", "orthogonalize",
                     "muon_step"])
    dtype = rng.choice(["bf16", "fp32"])
    m = rng.choice([1, 1, 1, 2, 3, 4])
    if op.startswith("layer_norm"):
        d = _spread(rng, 64, 8192)
        if rng.random() < 0.5:
            d = (d + 7) // 8 * 8
        rows = _spread(rng, 1, max(1, min(32768, 2 ** 27 // (m * d))))
        return {"op": op, "m": m, "rows": rows, "d": d, "dtype": dtype}
    if op.startswith("vocab_loss"):
        d = _spread(rng, 128, 4096)
        if rng.random() < 0.75:
            d = (d + 7) // 8 * 8
        vocab = _spread(rng, 1000, 131072)
        most = (2 ** 40 if dtype == "bf16" else 2 ** 36) // (2 * m * d * vocab)
        rows = _spread(rng, 1, max(1, min(8192, most)))
        return {"op": op, "m": m, "rows": rows, "d": d, "vocab": vocab, "dtype": dtype}
    rows, cols = _spread(rng, 64, 4096), _spread(rng, 64, 4096)
    if min(rows, cols) > 2048:
        m = 1
    return {"op": op, "m": m, "rows": rows, "cols": cols, "dtype": dtype}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, m = TYPES[case["dtype"]], case["m"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    if case["op"].startswith("layer_norm"):
        rows, d = case["rows"], case["d"]
        # a residual stream: features of unequal scale and an offset
        x = (normal(m, rows, d) * (0.5 + normal(m, 1, d).abs()) + 0.3 + 0.2 * normal(m, rows, 1)).to(dtype)
        s = {"x": x, "weight": 1.0 + 0.1 * normal(m, d), "bias": 0.1 * normal(m, d)}
        if case["op"] == "layer_norm_grad":
            s["dy"] = (normal(m, rows, d) + 0.05 * normal(m, 1, d)).to(dtype)
            x64 = x.double()
            mean = x64.mean(-1)
            s["mean"] = mean.float()
            s["rstd"] = ((x64 - mean[..., None]).square().mean(-1) + EPS).rsqrt().float()
            del s["bias"]
    elif case["op"].startswith("vocab_loss"):
        rows, d, vocab = case["rows"], case["d"], case["vocab"]
        w = (normal(m, vocab, d) / math.sqrt(d)).to(dtype)
        u = torch.rand((m, rows), generator=g, device="cuda")
        labels = (vocab ** u.double()).long().sub_(1).clamp_(0, vocab - 1)          # frequent and rare tokens
        # normalised activations that point at their token more or less strongly: some rows are certain, some are not
        sure = 14.0 * torch.rand((m, rows, 1), generator=g, device="cuda")
        own_row = torch.stack([w[i][labels[i]] for i in range(m)]).float()
        h = (normal(m, rows, d) + sure * own_row).to(dtype)
        labels[:, rows - rows // 32:] = -1                                             # padding behind the last sequence
        s = {"h": h, "W": w, "labels": labels.int()}
    else:
        rows, cols = case["rows"], case["cols"]
        # a gradient: a few strong directions over noise
        r = max(1, min(rows, cols) // 16)
        grad = normal(m, rows, r) @ normal(m, r, cols) / math.sqrt(r) + 0.3 * normal(m, rows, cols)
        s = {"g": (1e-3 * grad).to(dtype)}
        if case["op"] == "muon_step":
            s["w"] = normal(m, rows, cols) / math.sqrt(cols)
            s["v"] = 5e-3 * normal(m, rows, cols)
    s["op"] = case["op"]
    return s


# ---- the operators in plain torch ----------------------------------------------------------------------------

def _layer_norm(x, weight, bias):
    x32 = x.float()
    mean = x32.mean(-1, keepdim=True)
    c = x32 - mean
    rstd = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    y = c * rstd * weight[:, None, :] + bias[:, None, :]
    return y.to(x.dtype), mean[..., 0], rstd[..., 0]


def _layer_norm_grad(dy, x, weight, mean, rstd):
    dy32 = dy.float()
    xhat = (x.float() - mean[..., None]) * rstd[..., None]
    dxhat = dy32 * weight[:, None, :]
    dx = (dxhat - dxhat.mean(-1, keepdim=True) - xhat * (dxhat * xhat).mean(-1, keepdim=True)) * rstd[..., None]
    return dx.to(x.dtype), (dy32 * xhat).sum(1), dy32.sum(1)


def _vocab_loss(h, w, labels, grad):
    h32, w32 = h.float(), w.float()
    z = h32 @ w32.transpose(1, 2)
    kept = labels >= 0
    at = labels.clamp(min=0).long()[..., None]
    top = z.max(-1, keepdim=True).values
    lse = (z - top).exp().sum(-1, keepdim=True).log() + top
    row_loss = torch.where(kept, (lse - z.gather(-1, at))[..., 0], 0.0)
    count = kept.sum(1).clamp(min=1)
    loss = (row_loss.double().sum(1) / count).float()
    if not grad:
        return loss, row_loss, lse[..., 0]
    p = (z - lse).exp()
    p.scatter_add_(-1, at, torch.full_like(lse, -1.0))
    p *= (kept / count[:, None])[..., None]
    return loss, row_loss, lse[..., 0], (p @ w32).to(h.dtype), (p.transpose(1, 2) @ h32).to(w.dtype)


def _newton_schulz(u):
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt().float() + NS_EPS)
    for _ in range(NS_STEPS):
        a = x @ x.transpose(1, 2)
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    return x.transpose(1, 2) if tall else x


def _muon_step(w, v, g):
    g32 = g.float()
    v.mul_(MOMENTUM).add_(g32)
    o = _newton_schulz(g32 + MOMENTUM * v)
    w.sub_(LR * math.sqrt(max(1.0, w.shape[1] / w.shape[2])) * o)
    return w, v


def run(state):
    op = state["op"]
    if own:
        from paper_1810_08313_b200 import binding as b
        if op == "layer_norm":
            return b.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS)
        if op == "layer_norm_grad":
            return b.layer_norm_grad(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"])
        if op == "vocab_loss":
            return b.vocab_loss(state["h"], state["W"], state["labels"])
        if op == "vocab_loss_grad":
            return b.vocab_loss_grad(state["h"], state["W"], state["labels"])
        if op == "orthogonalize":
            return b.orthogonalize(state["g"], steps=NS_STEPS)
        b.muon_step(state["w"], state["v"], state["g"], lr=LR, momentum=MOMENTUM, nesterov=True, steps=NS_STEPS)
        return state["w"], state["v"]
    if op == "layer_norm":
        return _layer_norm(state["x"], state["weight"], state["bias"])
    if op == "layer_norm_grad":
        return _layer_norm_grad(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"])
    if op.startswith("vocab_loss"):
        return _vocab_loss(state["h"], state["W"], state["labels"], op == "vocab_loss_grad")
    if op == "orthogonalize":
        return _newton_schulz(state["g"].float()).to(state["g"].dtype)
    return _muon_step(state["w"], state["v"], state["g"])


def work(case):
    m, e = case["m"], BYTES[case["dtype"]]
    if case["op"] == "layer_norm":
        n = m * case["rows"] * case["d"]
        return {"bytes": 2 * n * e + 8 * m * case["d"] + 8 * m * case["rows"], "flops": 8 * n}
    if case["op"] == "layer_norm_grad":
        n = m * case["rows"] * case["d"]
        return {"bytes": 3 * n * e + 12 * m * case["d"] + 8 * m * case["rows"], "flops": 15 * n}
    if case["op"].startswith("vocab_loss"):
        acts, matrix = m * case["rows"] * case["d"] * e, m * case["vocab"] * case["d"] * e
        products = 3 if case["op"] == "vocab_loss_grad" else 1
        return {"bytes": (1 + products // 3) * (acts + matrix) + 12 * m * case["rows"],
                "flops": products * 2 * m * case["rows"] * case["d"] * case["vocab"]}
    n, k = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # per Newton-Schulz step: two symmetric products, of which half is enough, and one full one
    flops = NS_STEPS * m * (n * (n + 1) * k + n * n * (n + 1) + 2 * n * n * k)
    size = m * case["rows"] * case["cols"]
    return {"bytes": size * (2 * e if case["op"] == "orthogonalize" else 16 + e), "flops": flops}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "layer_norm":
        outs = []
        for x, weight, bias in zip(s["x"].double(), s["weight"].double(), s["bias"].double()):
            var, mean = torch.var_mean(x, dim=1, unbiased=False)
            rstd = 1.0 / torch.sqrt(var + EPS)
            outs.append(((x - mean[:, None]) * rstd[:, None] * weight + bias, mean, rstd))
        return tuple(torch.stack(o) for o in zip(*outs))
    if case["op"] == "layer_norm_grad":
        # the gradient in the row's own coordinates: project dy * weight off the constant and off x - mean
        outs = []
        for i in range(case["m"]):
            dy, mean, rstd = s["dy"][i].double(), s["mean"][i].double(), s["rstd"][i].double()
            xhat = (s["x"][i].double() - mean[:, None]) * rstd[:, None]
            t = dy * s["weight"][i].double()
            d = t.shape[1]
            along = torch.einsum("rd,rd->r", t, xhat) / d
            dx = rstd[:, None] * (t - t.sum(1, keepdim=True) / d - along[:, None] * xhat)
            outs.append((dx, torch.einsum("rd,rd->d", dy, xhat), dy.sum(0)))
        return tuple(torch.stack(o) for o in zip(*outs))
    if case["op"].startswith("vocab_loss"):
        outs = []
        for i in range(case["m"]):
            h, w, y = s["h"][i].double(), s["W"][i].double(), s["labels"][i].long()
            z = torch.einsum("rd,vd->rv", h, w)
            lse = torch.logsumexp(z, 1)
            rows = (y >= 0).nonzero()[:, 0]
            row_loss = torch.zeros_like(lse)
            row_loss[rows] = lse[rows] - z[rows, y[rows]]
            n = max(1, rows.numel())
            one = [row_loss.sum() / n, row_loss, lse]
            if case["op"] == "vocab_loss_grad":
                z -= lse[:, None]
                dz = z.exp_()
                dz[rows, y[rows]] -= 1.0
                dz /= n
                dz[y < 0] = 0.0
                one += [torch.einsum("rv,vd->rd", dz, w), torch.einsum("rv,rd->vd", dz, h)]
            outs.append(one)
        return tuple(torch.stack(o) for o in zip(*outs))

    def orthogonal(u):
        # from the side of the smaller Gram matrix: X_{k+1} = p(X X^T) X, or X p(X^T X) for a tall matrix
        x = u / (torch.linalg.norm(u) + NS_EPS)
        for _ in range(NS_STEPS):
            gram = x.T @ x if x.shape[0] > x.shape[1] else x @ x.T
            poly = NS_C * (gram @ gram) + NS_B * gram
            poly.diagonal().add_(NS_A)
            x = x @ poly if x.shape[0] > x.shape[1] else poly @ x
        return x

    if case["op"] == "orthogonalize":
        return torch.stack([orthogonal(u) for u in s["g"].double()])
    g, v, w = s["g"].double(), s["v"].double(), s["w"].double()
    v = MOMENTUM * v + g
    o = torch.stack([orthogonal(u) for u in g + MOMENTUM * v])
    return w - LR * max(1.0, case["rows"] / case["cols"]) ** 0.5 * o, v
