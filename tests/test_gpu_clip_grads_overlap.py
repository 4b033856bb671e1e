"""Gradient clipping of tensors that lie between one another: told apart where they share no memory, refused where they do."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _views(flat, cuts):
    return [flat[:, a:e] for a, e in zip(cuts, cuts[1:])]


def _check(before, got, norm, most):
    """Against 64 bits: a sum of fp32 squares, its root, the factor, the product and the result's rounding, half a step each."""
    import torch
    want = torch.stack([t.double().square().sum(1) for t in before]).sum(0).sqrt()
    assert bool(((norm.double() - want).abs() <= 7 * 2.0 ** -24 * want).all())
    for t, o in zip(before, got):
        w = t.double() * (most / want).clamp(max=1.0)[:, None]
        half = 2.0 ** -8 if o.dtype == torch.bfloat16 else 2.0 ** -24
        assert bool(((o.double() - w).abs() <= (9 * 2.0 ** -24 + half) * w.abs() + 1e-40).all())


@pytest.mark.parametrize("layout", ["in place", "two halves of a row", "other distances", "bf16 beside", "between the replicas"])
def test_tensors_between_one_another(layout):
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(3)
    m, cuts = 3, [0, 700, 701, 9001, 20000]
    rows = torch.randn((m, 50000), generator=g, device="cuda")
    grads, out = _views(rows, cuts), None
    if layout == "two halves of a row":
        out = [rows[:, 25000 + a:25000 + e] for a, e in zip(cuts, cuts[1:])]
    elif layout == "other distances":
        out = _views(torch.zeros(m, 23456, device="cuda"), cuts)
    elif layout == "bf16 beside":
        out = _views(rows.view(torch.bfloat16)[:, 40000:], cuts)             # behind the gradients of each row
    elif layout == "between the replicas":
        # replicas of one tensor a third of the others' distance apart, all in the first row behind the gradients
        grads = grads + [rows.view(-1)[20000:50000].unflatten(0, (m, 10000))]
    before = [t.clone() for t in grads]
    norm = b.clip_grads(grads, 2.5, out=out)
    _check(before, grads if out is None else out, norm, 2.5)
    if out is not None:
        assert all(torch.equal(t, s) for t, s in zip(grads, before))


def test_shared_memory_is_refused_and_left():
    import torch
    from paper_1810_08313_b200 import binding as b
    x, y = torch.ones(2, 5000, device="cuda"), torch.full((2, 5000), 2.0, device="cuda")
    z = torch.ones(2, 10000, device="cuda")
    for call in (lambda: b.clip_grads([x, y], 1.0, out=[y, x]), lambda: b.clip_grads([x, y], math.inf, out=[y, x]),
                 lambda: b.clip_grads([z[:, :6000], z[:, 5999:]], 1.0), lambda: b.clip_grads([z[:, :6000]], 1.0, out=[z[:, 1:6001]])):
        with pytest.raises(b.LsError):
            call()
    assert bool((x == 1).all()) and bool((y == 2).all()) and bool((z == 1).all())
    # only read
    assert abs(float(b.clip_grads([z[:, :6000], z[:, 5999:]], math.inf)[0]) - math.sqrt(10001)) < 1e-3
    assert bool((z == 1).all())
