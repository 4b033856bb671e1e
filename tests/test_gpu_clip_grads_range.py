"""Norms that fp32 does not hold: written as infinity, but the gradients are clipped by what they are."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most", [1.0, 1e-30, 3e38])
def test_clip_grads_by_a_norm_beyond_fp32(most):
    import torch
    from paper_1810_08313_b200 import binding as b
    x, y = torch.full((2, 3000), 3e38, device="cuda"), torch.ones(2, 500, device="cuda")
    x[1] = 2.0
    most = float(torch.tensor(most))
    before = [x.double(), y.double()]
    norm = b.clip_grads([x, y], most)
    want = sum(t.square().sum(1) for t in before).sqrt()
    assert math.isinf(float(norm[0])) and abs(float(norm[1] / want[1]) - 1.0) < 1e-6
    for t, o in zip(before, (x, y)):
        w = t * (most / want).clamp(max=1.0)[:, None]
        # the factor, in two, and two products: half a step each, and the norm's 7; half a step of the smallest numbers
        assert bool(((o.double() - w).abs() <= 11 * 2.0 ** -24 * w.abs() + 2.0 ** -150).all())


def test_clip_grads_by_a_limit_that_fp32_does_not_hold():
    """The limit is a double: a norm of exactly 5, and factors that are rounded once."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator().manual_seed(2)
    for most in torch.rand(200, generator=g, dtype=torch.float64).tolist():
        x = torch.tensor([[3.0, 4.0]], device="cuda")
        b.clip_grads([x], most)
        want = torch.tensor([[3.0, 4.0]]) * torch.tensor(most / 5.0, dtype=torch.float64).float()
        assert torch.equal(x.cpu(), want), most
