"""Draws whose top-p ends where the bins of masses end, 16 octaves below the largest logit: tokens there are compared with one another like those
before and behind them."""
import itertools
import math

import pytest
import torch

import rows_util as ru
from draws_util import F32, check, f32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def row_of(n, T, dtype, seed):
    """One logit and n - 1 far below it: before, inside and behind the last of 512 bins of 16 / 511 octaves (bf16: its numbers there, below a
    largest logit that puts one of them inside)."""
    g = torch.Generator().manual_seed(seed)
    wide = 16 * ru.LN2 * f32(T) / 511
    if dtype == F32:
        top = 0.0
        bins = torch.cat([505 + 5.9 * torch.rand(n // 4, generator=g), 512.1 + 8 * torch.rand(min(n // 8, 200), generator=g)])
        bins = torch.cat([bins, 511.1 + 0.8 * torch.rand(n - 1 - len(bins), generator=g)])
        low = -bins.double() * wide
    else:
        near = torch.tensor(-511.5 * wide).to(BF).double()
        step = 2.0 ** (math.floor(math.log2(511.5 * wide)) - 7)
        if float(near) < -511.5 * wide:
            near += step                                       # the largest logit is then 0 or more
        top = float(torch.tensor(511.5 * wide + float(near)).to(BF))
        assert 511.05 * wide < top - float(near) < 511.95 * wide
        low = near + step * torch.tensor([0.0, 0.0, 0.0, 0.0, 1.0, 1.0, -1.0, 2.0], dtype=torch.double)[torch.randint(0, 8, (n - 1,), generator=g)]
    x = torch.cat([torch.tensor([top], dtype=torch.double), low]).to(dtype)
    return x[torch.randperm(n, generator=g)]


@pytest.mark.parametrize("dtype,T", list(itertools.product([F32, BF], [0.9, 1.0, 2.0])))
@pytest.mark.parametrize("n,V", [(50, 50), (300, 300), (2001, 2001), (4096, 4096), (900, 33000)])
def test_prefixes_that_end_in_the_last_bin(n, V, dtype, T):
    z = torch.full((3, V), -math.inf, dtype=dtype)
    for r in range(3):
        at = torch.randperm(V, generator=torch.Generator().manual_seed(r))[:n].sort().values
        z[r, at] = row_of(n, T, dtype, seed=n + r)
    z = z.cuda()
    u = torch.rand(3, 6, generator=torch.Generator().manual_seed(n))
    u[:, 0], u[:, 1] = 1.0, 1.0 - 2.0 ** -10
    down = z[0].double().cpu().sort(descending=True).values[:n]
    w = torch.exp((down - down[0]) / f32(T))
    s = w.cumsum(0)
    for part in (0.1, 0.2, 0.3, 0.55, 0.8, 0.97):              # of the tokens: the p that ends a prefix there, in the middle of a token's cell
        end = int(part * n)
        p = float((s[end] - w[end] / 2) / s[-1])
        for m in (0.0, math.exp(-511.5 * 16 * ru.LN2 / 511)):
            check(z, u, T, 0, p, m)
