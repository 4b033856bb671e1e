"""Newton-Schulz orthogonalisation beside the same steps in fp32 arithmetic, both measured against 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315


def _steps(x, steps=5):
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        a = x @ x.T
        x = A * x + (B * a + C * (a @ a)) @ x
    return x.T if tall else x


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("rows,cols", [(1524, 65), (626, 67), (65, 3235), (72, 166), (224, 73), (64, 64), (200, 90), (128, 500), (257, 130), (763, 189), (722, 805), (3801, 420),
                                       (522, 481), (931, 762), (1577, 604), (1191, 1058), (517, 3802), (2048, 2048)])
def test_error_beside_fp32_arithmetic(rows, cols, seed):
    """A few strong directions over noise, as gradients have them: the singular values of the strong ones and of the noise each
    move together, so that a bias of the products shows.  The error may be at most 1.5 times that of fp32 arithmetic (rounded to
    nearest, 2^-24 an operation), in which the operands' 22 bits and the products' truncation have their room."""
    import torch
    from paper_1810_08313_b200 import binding as b
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + rows + cols)
    r = max(1, min(rows, cols) // 16)
    u = torch.randn(rows, r, generator=g, device="cuda") @ torch.randn(r, cols, generator=g, device="cuda") / r ** 0.5
    u = 1e-3 * (u + 0.3 * torch.randn(rows, cols, generator=g, device="cuda"))
    x = u.double() / (torch.linalg.norm(u.double()) + 1e-7)
    want = _steps(x)
    keep = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    plain = _steps(u / (torch.linalg.norm(u.double()).float() + 1e-7))
    torch.backends.cuda.matmul.allow_tf32 = keep
    got = b.orthogonalize(u)
    size = torch.linalg.norm(want)
    err, ref = (float(torch.linalg.norm(t.double() - want) / size) for t in (got, plain))
    assert err <= 1.5 * ref, (err, ref)
    b.device_status()
