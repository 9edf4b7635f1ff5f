"""The gradient at the tokens that the teacher names, in the bits that its difference needs."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("V,K,near", [(50, 50, 1e-3), (1000, 1000, 1e-3), (700, 700, 1e-5), (5000, 40, 1e-3), (60000, 300, 1e-4)])
@pytest.mark.parametrize("T", [0.7, 1.0, 3.0])
def test_a_student_near_its_teacher(V, K, near, T):
    """q - p is a small difference.  Its bar: half a step of the result, 2^-33 of q by the sums in 64 bits (their terms' steps of 2^-44, up to 2^10 of
    them), and 2^-15 of what the other tokens have of the whole, whose terms are in 32 bits."""
    g = torch.Generator().manual_seed(V)
    named = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(3)])
    x = torch.randn(3, V, generator=g).clamp(-5, 5) - (40.0 if V > K else 0.0)
    x.scatter_(1, named, torch.randn(3, K, generator=g).clamp(-5, 5))
    value = x.gather(1, named)
    z = x + near * torch.randn(3, V, generator=g)
    loss, grad, status = dsbd.distill(z.cuda(), value.cuda(), named.int().cuda(), temperature=T)
    assert int(status) == 0
    T = float(torch.tensor(T, dtype=F32))
    for r in range(3):
        p, q = torch.softmax(value[r].double() / T, 0), torch.softmax(z[r].double() / T, 0)
        want = T * (q[named[r]] - p)
        others = float(1 - q[named[r]].sum()) if V > K else 0.0
        bar = 2.0 ** -24 * want.abs() + T * q[named[r]] * (2.0 ** -33 + 2.0 ** -15 * abs(others))
        err = (grad[r, named[r].cuda()].double().cpu() - want).abs()
        assert bool((err <= bar).all()), float((err / bar).max())
