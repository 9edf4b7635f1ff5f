"""Numbers beyond 32 bits, which the C ABI does not take: refused, or what they mean there."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
MORE = 1 << 32


def test_a_top_k_beyond_32_bits_is_off():
    z = ru.rows_of(4, 3000, F32, seed=1)
    u = torch.rand(4, 5, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    want = dsbd.sample_rows(z, u)
    for k in (MORE + 1, MORE // 2, 10 ** 30, 1 - MORE, -10 ** 30):
        got = dsbd.sample_rows(z, u, top_k=k)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), k
    for k in (2.5, 20.0, "3"):
        with pytest.raises(TypeError):
            dsbd.sample_rows(z, u, top_k=k)


@pytest.mark.parametrize("shape", [(1, MORE + 5), (MORE + 3, 1)])
def test_rows_and_lengths_beyond_32_bits_are_refused(shape):
    z = torch.empty(shape, dtype=BF, device="cuda")
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.top_logits(z, 1)
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.sample_rows(z, torch.zeros(1, device="cuda").expand(shape[0]))
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.distill(z, torch.zeros(1, 1, device="cuda"), torch.zeros(1, 1, dtype=I32, device="cuda"))


def test_draws_and_entries_beyond_32_bits_are_refused():
    z = torch.zeros(1, 100, device="cuda")
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.sample_rows(z, torch.empty(1, MORE + 1, device="cuda"))
    for K in (MORE + 1, MORE // 2, 10 ** 30):
        with pytest.raises(dsbd.DsbdError, match="unsupported"):
            dsbd.top_logits(z, K)
    value = torch.empty(1, MORE + 1, device="cuda")
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.distill(z, value, value.view(I32), grad=None)
