"""The rest of rows whose tokens all weigh nearly the same: sums of as many terms as kept words have."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("K", [40, 300, 1000])
def test_high_temperatures(K, dtype):
    """A term is off by 2^-22 and three roundings of its argument, which is below 1; a thread adds up to 256 in 32 bits; the result is rounded once."""
    z = ru.rows_of(500, 50257, dtype, seed=K, zipf=False)
    first = dsbd.top_logits(z, K, temperature=1000.0)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(first[:3], dsbd.top_logits(z, K, temperature=1000.0)))
    for r in (0, 250, 499):
        x = z[r].double().cpu()
        v, at, rest = ru.top(x, K, 1000.0)
        assert torch.equal(first[0][r].double().cpu(), v) and torch.equal(first[1][r].long().cpu(), at)
        assert abs(float(first[2][r]) - float(rest)) <= 2.0 ** -24 * float(rest) + 2.0 ** -22 + 3 * 2.0 ** -24 + 256 * 2.0 ** -24
