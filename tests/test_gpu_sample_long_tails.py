"""Top-p of rows with a few likely tokens and a long tail of unlikely ones: how much of the tail is kept, to the token."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from draws_util import F32, prefix

pytestmark = pytest.mark.gpu
BF = torch.bfloat16

# By how much of the whole a cut may be off: a mass is off by 4e-14 of itself and by a last step of up to 2^-41 of itself, and the whole likewise.
OFF = 2 * (4e-14 + 2.0 ** -41)


def rows(V, dtype, likely, deep, seed):
    """Falling from token to token: `likely` tokens about 0, the others about -deep."""
    g = torch.Generator().manual_seed(seed)
    x = -deep + 0.5 * torch.randn(3, V, generator=g)
    x[:, :likely] = 0.3 * torch.randn(3, likely, generator=g)
    return x.to(dtype).sort(dim=1, descending=True).values


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V,likely,deep,T,p,k", [
    (262144, 1, 20.8, 1.0, 0.9999, 0), (128256, 1, 24.0, 1.0, 0.999999, 0), (128256, 1, 16.0, 1.0, 0.995, 0), (151936, 40, 20.0, 1.0, 0.99999, 0),
    (262144, 1, 13.0, 0.6, 0.9999, 0), (50257, 3, 40.0, 2.0, 0.99999, 0), (262144, 1, 20.8, 1.0, 0.9999, 200000), (128256, 1, 9.0, 1.0, 0.9, 60000),
    (128256, 1, 12.5, 1.0, 0.3, 0), (393216, 1, 23.0, 1.0, 1 - 2.0 ** -20, 0)])
def test_the_tail_s_end(V, likely, deep, T, p, k, dtype):
    x = rows(V, dtype, likely, deep, seed=V)
    token, logp, status = dsbd.sample_rows(x.cuda(), torch.ones(3, 1, device="cuda"), temperature=T, top_p=p, top_k=k)
    assert int(status) == 0
    for r in range(3):
        n, log_sum, margin = prefix(x[r].double().numpy(), T, p, k)
        assert margin > OFF, "the inputs leave the cut open"
        assert int(token[r, 0]) == n - 1                       # u = 1: the last kept token
        want = (float(x[r, n - 1]) - float(x[r, 0])) / float(torch.tensor(T)) - log_sum
        assert abs(float(logp[r, 0]) - want) <= 2.0 ** -24 * abs(want) + 1e-12


@pytest.mark.parametrize("V,p", [(50257, 0.99998), (262144, 0.9999)])
def test_the_tail_in_any_order_and_the_same_bits(V, p):
    """The same row with its tokens shuffled keeps as many: the last kept of them is the last in the tokens' order."""
    x = rows(V, F32, 1, 20.8, seed=3)[:1]
    n, log_sum, margin = prefix(x[0].double().numpy(), 1.0, p)
    assert margin > OFF
    at = torch.randperm(V, generator=torch.Generator().manual_seed(1))
    z = torch.empty_like(x)
    z[0, at] = x[0]
    last = int(at[:n].max())
    z = z.cuda()
    for _ in range(3):
        token, logp, _ = dsbd.sample_rows(z, torch.ones(1, 1, device="cuda"), top_p=p)
        want = float(z[0, last].cpu()) - float(x[0, 0]) - log_sum
        assert int(token) == last and abs(float(logp) - want) <= 2.0 ** -24 * abs(want) + 1e-12
