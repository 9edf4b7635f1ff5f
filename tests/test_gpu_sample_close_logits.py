"""Draws from rows whose largest logits are neighbours in fp32, at temperatures of parts of their distance."""
import pytest
import torch

import rows_util as ru
from draws_util import F32, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [20.0, 30.0, 1e6, 1.0, -5.0])
@pytest.mark.parametrize("V", [40, 9000])
def test_neighbours_of_the_largest_logit(top, V):
    """Differences of 47 to 28000 temperatures: ever so little mass, or none, and a few of equal size."""
    step = float(torch.nextafter(torch.tensor(abs(top)), torch.tensor(1e30)) - abs(top))
    g = torch.Generator().manual_seed(V)
    z = top - 100.0 * torch.rand(3, V, generator=g) - 50 * step
    near = (top - step * torch.arange(1, 21).double()).float()
    for r in range(3):
        at = torch.randperm(V, generator=g)
        z[r, at[:20]] = near
        z[r, at[20:22 + r]] = top
    assert int((z.max(1).values == top).sum()) == 3
    u = 0.01 + 0.98 * torch.rand(3, 5, generator=g)
    for part in (1400, 1200, 1000, 800, 700, 500, 400, 200, 100, 60, 47):
        for k, p, m in [(0, 1.0, 0.0), (20, 1.0, 0.0), (20, 0.9, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.1), (300, 0.9, 0.0), (600, 0.95, 0.0), (5000, 0.9, 0.0)]:
            check(z.cuda(), u, step / part, k, p, m)
