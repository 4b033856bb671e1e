"""Operators of a language model's attention block and of its gradients' norm, as measured cases.

A case is one call of one operator: the norm of every query and key head with the rotation by position in the same pass,
and its gradient; causal attention with grouped heads over packed sequences of different lengths, and its gradient; the
global norm of a replica's gradients with their clipping.  Every operator takes the replicas of a job packed in one tensor
(first axis m).  `run` computes a case in plain torch, in 32 bits (angles and long sums in 64), or through the package's
entry points (`own`).
"""
import math
import random

import torch

own = False

EPS = 1e-6                             # RMS norm of a head
BASE = 500000.0                        # of the rotation's frequencies

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def listed():
    return [
        # the heads of one short sequence: the time of a call
        {"name": "qk_norm_rope short", "op": "qk_norm_rope", "m": 1, "tokens": 24, "heads": 8, "kv_heads": 2, "head_dim": 64,
         "rot_dim": 64, "interleaved": False, "dtype": "bf16"},
        # the tokens of a training step, q and k being parts of one projection
        {"name": "qk_norm_rope step", "op": "qk_norm_rope", "m": 1, "tokens": 16384, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "rot_dim": 128, "interleaved": False, "dtype": "bf16"},
        # three fp32 replicas of a small model, odd token count, part of each head rotated in neighbouring pairs
        {"name": "qk_norm_rope_grad odd fp32", "op": "qk_norm_rope_grad", "m": 3, "tokens": 777, "heads": 6, "kv_heads": 3,
         "head_dim": 80, "rot_dim": 32, "interleaved": True, "dtype": "fp32"},
        # the same training step's way back
        {"name": "qk_norm_rope_grad step", "op": "qk_norm_rope_grad", "m": 1, "tokens": 16384, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "rot_dim": 128, "interleaved": False, "dtype": "bf16"},
        # a few short sequences of two small replicas: the time of a call
        {"name": "attention short", "op": "attention", "m": 2, "tokens": 160, "seqs": 3, "pad": 0, "heads": 4, "kv_heads": 4,
         "head_dim": 64, "dtype": "bf16"},
        # a batch packed from documents of all lengths, padded at its end
        {"name": "attention packed", "op": "attention", "m": 1, "tokens": 8191, "seqs": 23, "pad": 100, "heads": 16, "kv_heads": 4,
         "head_dim": 64, "dtype": "bf16"},
        # one long document: the largest forward case
        {"name": "attention long", "op": "attention", "m": 1, "tokens": 16384, "seqs": 1, "pad": 0, "heads": 16, "kv_heads": 4,
         "head_dim": 128, "dtype": "bf16"},
        # two replicas of a small fp32 job
        {"name": "attention_grad fp32", "op": "attention_grad", "m": 2, "tokens": 513, "seqs": 5, "pad": 0, "heads": 6, "kv_heads": 2,
         "head_dim": 64, "dtype": "fp32"},
        # packed documents, heads that fill no whole tile, every head with keys of its own
        {"name": "attention_grad packed", "op": "attention_grad", "m": 2, "tokens": 4095, "seqs": 9, "pad": 37, "heads": 8,
         "kv_heads": 8, "head_dim": 96, "dtype": "bf16"},
        # a training step's tokens in two documents: the largest case
        {"name": "attention_grad step", "op": "attention_grad", "m": 1, "tokens": 8192, "seqs": 2, "pad": 0, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "dtype": "bf16"},
        # four replicas of a small fp32 model, in place, below the limit: a step like most
        {"name": "clip_grads small", "op": "clip_grads", "m": 4, "layers": 6, "d": 250, "vocab": 2003, "dtype": "fp32",
         "out": "same", "clips": False},
        # the fp32 gradient sums of two replicas, clipped into the bf16 gradients of the momentum step
        {"name": "clip_grads step", "op": "clip_grads", "m": 2, "layers": 10, "d": 1536, "vocab": 32000, "dtype": "fp32",
         "out": "bf16", "clips": True},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["qk_norm_rope", "qk_norm_rope_grad", "attention", "attention", "attention_grad", "attention_grad", "clip_grads"])
    if op == "clip_grads":
        d = _spread(rng, 32, 2048)
        m, layers, vocab = rng.choice([1, 2, 3, 4]), rng.randint(1, 10), _spread(rng, 500, 50000)
        layers = max(1, min(layers, (3 * 10 ** 8 // m - vocab * d) // (12 * d * d)))
        dtype = rng.choice(["fp32", "bf16"])
        return {"op": op, "m": m, "layers": layers, "d": d, "vocab": vocab, "dtype": dtype,
                "out": rng.choice(["same", "bf16", "fp32"]), "clips": rng.random() < 0.6}
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    m = rng.choice([1, 1, 1, 2, 3])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 5])
    head_dim = rng.choice([64, 128, 64, 128, 8 * rng.randint(2, 16), rng.randint(9, 160)])
    if op.startswith("qk"):
        rot_dim = rng.choice([head_dim // 2 * 2, head_dim // 2 * 2, head_dim // 4 * 2])
        most = 2 ** 26 // (m * (heads + kv_heads) * head_dim)
        return {"op": op, "m": m, "tokens": _spread(rng, 1, max(1, min(16384, most))), "heads": heads, "kv_heads": kv_heads,
                "head_dim": head_dim, "rot_dim": rot_dim, "interleaved": rng.random() < 0.3, "dtype": dtype}
    fast = dtype == "bf16" and head_dim % 8 == 0 and head_dim <= 128
    # pairs of a query and a key of one sequence over all heads
    pairs = (2 ** 31 if fast else 2 ** 27) // (m * heads * (4 if op == "attention_grad" else 1))
    tokens = _spread(rng, 1, max(1, min(16384, int(math.sqrt(2 * pairs)))))
    seqs = min(tokens, rng.choice([1, 1, 2, 3, 7, 20, 60]))
    return {"op": op, "m": m, "tokens": tokens, "seqs": seqs, "pad": rng.choice([0, 0, (tokens - seqs) // 9]), "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}


def _starts(case):
    """Where the sequences of every replica start, [m][seqs + 1]: a fixed cut of the tokens before the padding."""
    rng = random.Random(case["tokens"] * 1009 + case["seqs"])
    end, out = case["tokens"] - case["pad"], []
    for _ in range(case["m"]):
        inner = rng.sample(range(1, end), case["seqs"] - 1) if case["seqs"] > 1 else []
        out.append([0] + sorted(inner) + [end])
    return out


def _grad_shapes(case):
    """The matrices and vectors of a model of `layers` blocks: embedding, last norm, and six tensors a block."""
    d = case["d"]
    shapes = [(case["vocab"], d), (d,)]
    for _ in range(case["layers"]):
        shapes += [(3 * d, d), (d, d), (4 * d, d), (d, 4 * d), (d,), (d,)]
    return shapes


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    m, op = case["m"], case["op"]
    dtype = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    if op == "clip_grads":
        grads, total = [], 0.0
        for shape in _grad_shapes(case):
            # layers' gradients differ in scale
            t = (normal(m, *shape) * (1e-3 * math.exp(1.5 * float(torch.randn((), generator=g, device="cuda"))))).to(dtype)
            total += float(t.double().square().sum(tuple(range(1, t.dim()))).min())
            grads.append(t)
        norm = math.sqrt(total)
        s = {"grads": grads, "max_norm": 0.37 * norm if case["clips"] else 40.0 * norm, "out": None}
        if case["out"] != "same":
            s["out"] = [torch.zeros_like(t, dtype=TYPES[case["out"]]) for t in grads]
        s["op"] = op
        return s

    tokens, heads, kv, hd = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    if op.startswith("qk"):
        # one projection of the residual stream: q, k and v side by side in a row
        width = (heads + 2 * kv) * hd
        scale = 0.3 + normal(m, 1, heads + 2 * kv, 1).abs()
        qkv = (normal(m, tokens, heads + 2 * kv, hd) * scale).to(dtype).view(m, tokens, width)
        q = qkv[..., :heads * hd].unflatten(-1, (heads, hd))
        k = qkv[..., heads * hd:(heads + kv) * hd].unflatten(-1, (kv, hd))
        inv_freq = BASE ** (-torch.arange(0, case["rot_dim"], 2, device="cuda", dtype=torch.float64) / max(1, case["rot_dim"]))
        # positions in sequences that start anywhere in a long context
        start = torch.randint(0, 100000, (m, 1), generator=g, device="cuda", dtype=torch.int32)
        positions = start + torch.arange(tokens, device="cuda", dtype=torch.int32) % 6007
        s = {"q": q, "k": k, "q_weight": 1.0 + 0.2 * normal(m, hd), "k_weight": 1.0 + 0.2 * normal(m, hd), "inv_freq": inv_freq,
             "positions": positions.contiguous(), "interleaved": case["interleaved"]}
        if op == "qk_norm_rope_grad":
            s["dqr"] = (normal(m, tokens, heads, hd) + 0.1 * normal(m, 1, 1, hd)).to(dtype)
            s["dkr"] = (normal(m, tokens, kv, hd) + 0.1 * normal(m, 1, 1, hd)).to(dtype)
        s["op"] = op
        return s

    starts = _starts(case)
    # normalised heads; some attend broadly, some sharply, and neighbouring keys resemble each other
    drift = normal(m, tokens // 64 + 1, kv, hd).repeat_interleave(64, dim=1)[:, :tokens]
    k = normal(m, tokens, kv, hd) + 0.7 * drift
    q = normal(m, tokens, heads, hd) + 0.5 * drift.repeat_interleave(heads // kv, dim=2)
    q = q * (0.5 + 2.0 * torch.rand((m, 1, heads, 1), generator=g, device="cuda"))
    s = {"q": q.to(dtype), "k": k.to(dtype), "v": normal(m, tokens, kv, hd).to(dtype), "scale": 1.0 / math.sqrt(hd), "starts": starts,
         "seq_start": torch.tensor(starts, dtype=torch.int32, device="cuda"), "op": op}
    if op == "attention_grad":
        out, s["lse"] = _attention(s["q"], s["k"], s["v"], starts, s["scale"])
        s["out"] = out
        s["dout"] = (1e-2 * normal(m, tokens, heads, hd)).to(dtype)
    return s


# ---- the operators in plain torch ----------------------------------------------------------------------------

def _turn(x, cos, sin, interleaved):
    """The leading columns of the last axis in pairs, turned; cos, sin [m][tokens][1][rot / 2]."""
    r = 2 * cos.shape[-1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    ta, tb = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((ta, tb), -1).flatten(-2) if interleaved else torch.cat((ta, tb), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _angles(s):
    angle = s["positions"].double()[..., None, None] * s["inv_freq"]
    return angle.cos().float(), angle.sin().float()


def _norm(x):
    x32 = x.float()
    rstd = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS)
    return x32 * rstd, rstd


def _qk_norm_rope(s):
    cos, sin = _angles(s)
    out = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        xhat, _ = _norm(x)
        out.append(_turn(xhat * w[:, None, None], cos, sin, s["interleaved"]).to(x.dtype))
    return tuple(out)


def _qk_norm_rope_grad(s):
    cos, sin = _angles(s)
    dx, dw = [], []
    for x, w, dy in ((s["q"], s["q_weight"], s["dqr"]), (s["k"], s["k_weight"], s["dkr"])):
        xhat, rstd = _norm(x)
        dz = _turn(dy.float(), cos, -sin, s["interleaved"])
        dw.append((dz * xhat).sum((1, 2)))
        t = dz * w[:, None, None]
        dx.append(((t - xhat * (t * xhat).mean(-1, keepdim=True)) * rstd).to(x.dtype))
    return dx[0], dx[1], dw[0], dw[1]


def _blocks(q, k, starts, bytes_a_score):
    """(replica, first row, end, kv head, its query heads) such that the scores of a block stay within some GB."""
    heads, kv = q.shape[2], k.shape[2]
    group = heads // kv
    for i, cuts in enumerate(starts):
        for a, b in zip(cuts, cuts[1:]):
            most = max(1, int(4e9 / (bytes_a_score * (b - a) ** 2)))
            for h in range(kv):
                for f in range(0, group, most):
                    yield i, a, b, h, slice(h * group + f, h * group + min(group, f + most))


def _attention(q, k, v, starts, scale):
    out = torch.zeros_like(q)
    lse = torch.zeros((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
    for i, a, b, h, at in _blocks(q, k, starts, 12):
        z = (q[i, a:b, at].float().transpose(0, 1) @ k[i, a:b, h].float().T) * scale
        hidden = torch.ones((b - a, b - a), dtype=torch.bool, device=q.device).triu_(1)
        z.masked_fill_(hidden, -math.inf)
        top = z.max(-1, keepdim=True).values
        p = (z - top).exp_()
        total = p.sum(-1, keepdim=True)
        out[i, a:b, at] = ((p @ v[i, a:b, h].float()) / total).transpose(0, 1).to(q.dtype)
        lse[i, at, a:b] = (total.log() + top)[..., 0]
    return out, lse


def _attention_grad(s):
    q, k, v = s["q"], s["k"], s["v"]
    dq = torch.zeros_like(q)
    dk, dv = torch.zeros_like(k, dtype=torch.float32), torch.zeros_like(v, dtype=torch.float32)
    for i, a, b, h, at in _blocks(q, k, s["starts"], 20):
        qs, ds = q[i, a:b, at].float().transpose(0, 1), s["dout"][i, a:b, at].float().transpose(0, 1)
        kh, vh = k[i, a:b, h].float(), v[i, a:b, h].float()
        z = (qs @ kh.T) * s["scale"]
        hidden = torch.ones((b - a, b - a), dtype=torch.bool, device=q.device).triu_(1)
        z.masked_fill_(hidden, -math.inf)
        p = (z - s["lse"][i, at, a:b, None]).exp_()
        dv[i, a:b, h] += (p.transpose(1, 2) @ ds).sum(0)
        dot = (ds * s["out"][i, a:b, at].float().transpose(0, 1)).sum(-1, keepdim=True)
        p *= (ds @ vh.T) - dot
        dq[i, a:b, at] = ((p @ kh) * s["scale"]).transpose(0, 1).to(q.dtype)
        dk[i, a:b, h] += (p.transpose(1, 2) @ qs).sum(0) * s["scale"]
    return dq, dk.to(k.dtype), dv.to(v.dtype)


def _clip_grads(s):
    total = 0.0
    for t in s["grads"]:
        total = total + t.float().square().sum(tuple(range(1, t.dim())), dtype=torch.float64)
    norm = total.sqrt()
    factor = torch.where(norm <= s["max_norm"], 1.0, s["max_norm"] / norm).float()
    out = s["out"] if s["out"] is not None else s["grads"]
    for t, o in zip(s["grads"], out):
        o.copy_(t.float() * factor.view((-1,) + (1,) * (t.dim() - 1)))
    return [norm.float()] + list(out)


def run(state):
    s, op = state, state["op"]
    if own:
        from paper_1810_08313_b200 import binding as b
        if op == "qk_norm_rope":
            return b.qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["positions"], s["inv_freq"], eps=EPS,
                                  interleaved=s["interleaved"])
        if op == "qk_norm_rope_grad":
            return b.qk_norm_rope_grad(s["dqr"], s["dkr"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["positions"], s["inv_freq"],
                                       eps=EPS, interleaved=s["interleaved"])
        if op == "attention":
            return b.attention(s["q"], s["k"], s["v"], s["seq_start"], scale=s["scale"])
        if op == "attention_grad":
            return b.attention_grad(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["seq_start"], scale=s["scale"])
        norm = b.clip_grads(s["grads"], s["max_norm"], out=s["out"])
        return [norm] + list(s["out"] if s["out"] is not None else s["grads"])
    if op == "qk_norm_rope":
        return _qk_norm_rope(s)
    if op == "qk_norm_rope_grad":
        return _qk_norm_rope_grad(s)
    if op == "attention":
        return _attention(s["q"], s["k"], s["v"], s["starts"], s["scale"])
    if op == "attention_grad":
        return _attention_grad(s)
    return _clip_grads(s)


def work(case):
    m, e = case["m"], BYTES[case["dtype"]]
    if case["op"] == "clip_grads":
        n = m * sum(math.prod(shape) for shape in _grad_shapes(case))
        if case["out"] == "same":
            return {"bytes": n * e * (2 if case["clips"] else 1), "flops": (3 if case["clips"] else 2) * n}
        return {"bytes": n * (e + BYTES[case["out"]]), "flops": 3 * n}
    tokens, heads, kv, hd = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"].startswith("qk"):
        n = m * tokens * (heads + kv) * hd
        back = case["op"] == "qk_norm_rope_grad"
        return {"bytes": n * e * (3 if back else 2) + 4 * m * tokens, "flops": n * (16 if back else 8)}
    pairs = heads * sum((b - a) * (b - a + 1) // 2 for cuts in _starts(case) for a, b in zip(cuts, cuts[1:]))
    own_rows, shared, sums = m * tokens * heads * hd * e, m * tokens * kv * hd * e, 4 * m * tokens * heads
    if case["op"] == "attention":
        return {"bytes": 2 * own_rows + 2 * shared + sums, "flops": 4 * hd * pairs}
    return {"bytes": 4 * own_rows + 4 * shared + sums, "flops": 10 * hd * pairs}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip_grads":
        flat = [torch.cat([t[i].double().flatten().norm().view(1) for t in s["grads"]]).norm() for i in range(case["m"])]
        norm = torch.stack(flat)
        factor = (s["max_norm"] / norm).clamp(max=1.0)
        return [norm] + [torch.stack([t[i].double() * factor[i] for i in range(case["m"])]) for t in s["grads"]]
    if case["op"].startswith("qk"):
        r = case["rot_dim"]
        unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           s["positions"].double()[:, :, None, None] * s["inv_freq"])

        def as_pairs(x):
            x = x[..., :r]
            return torch.complex(x[..., 0::2], x[..., 1::2]) if case["interleaved"] else torch.complex(*x.split(r // 2, -1))

        def rotate(x, by):
            c = as_pairs(x.contiguous()) * by
            head = torch.view_as_real(c).flatten(-2) if case["interleaved"] else torch.cat((c.real, c.imag), -1)
            return torch.cat((head, x[..., r:]), -1) if r else x

        outs, sums = [], []
        for x, w, dy in ((s["q"], s["q_weight"], s.get("dqr")), (s["k"], s["k_weight"], s.get("dkr"))):
            x, w = x.double(), w.double()[:, None, None, :]
            size = (x.square().sum(-1, keepdim=True) / case["head_dim"] + EPS).sqrt()
            if dy is None:
                outs.append(rotate(x / size * w, unit))
            else:
                back = rotate(dy.double(), unit.conj())
                sums.append(torch.einsum("mthd,mthd->md", back, x / size))
                along = torch.einsum("mthd,mthd->mth", back * w, x)[..., None]
                outs.append(back * w / size - x * along / (case["head_dim"] * size ** 3))
        return tuple(outs + sums)
    q, k, v = s["q"], s["k"], s["v"]
    group, tokens = case["heads"] // case["kv_heads"], case["tokens"]
    back = case["op"] == "attention_grad"
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((case["m"], case["heads"], tokens), dtype=torch.float64, device="cuda")
    dk = torch.zeros(k.shape, dtype=torch.float64, device="cuda") if back else None
    dv = torch.zeros(k.shape, dtype=torch.float64, device="cuda") if back else None
    for i, cuts in enumerate(s["starts"]):
        for a, b in zip(cuts, cuts[1:]):
            for h in range(case["heads"]):
                kh, vh = k[i, a:b, h // group].double(), v[i, a:b, h // group].double()
                for r0 in range(a, b, 2048):             # some rows against the keys up to the last of them
                    r1 = min(b, r0 + 2048)
                    kr, vr = kh[:r1 - a], vh[:r1 - a]
                    z = torch.einsum("id,jd->ij", q[i, r0:r1, h].double(), kr) * s["scale"]
                    later = torch.arange(a, r1, device="cuda")[None, :] > torch.arange(r0, r1, device="cuda")[:, None]
                    z[later] = -math.inf
                    if not back:
                        lse[i, h, r0:r1] = torch.logsumexp(z, 1)
                        out[i, r0:r1, h] = torch.softmax(z, 1) @ vr
                        continue
                    p = torch.exp(z - s["lse"][i, h, r0:r1, None].double())
                    do = s["dout"][i, r0:r1, h].double()
                    dv[i, a:r1, h // group] += p.T @ do
                    dz = p * (do @ vr.T - torch.einsum("id,id->i", do, s["out"][i, r0:r1, h].double())[:, None]) * s["scale"]
                    out[i, r0:r1, h] = dz @ kr
                    dk[i, a:r1, h // group] += dz.T @ q[i, r0:r1, h].double()
    return (out, dk, dv) if back else (out, lse)
