"""Losses and gradients of rows with logits of +inf and NaN."""
import math

import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_a_logit_without_a_softmax(rest, bad):
    """A student's +inf or NaN, wherever it stands: no share of its row is a number.  The rows beside it are as ever."""
    V, K = 6000, 20
    teacher = ru.rows_of(6, V, F32, seed=1)
    value, index, left, _ = dsbd.top_logits(teacher, K)
    clean = teacher + torch.randn(6, V, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    left = left if rest else None
    want = dsbd.distill(clean, value, index, rest=left)
    z = clean.clone()
    inside = set(index[4].tolist())
    z[1, int(index[1, 0])] = bad                               # named, with the teacher's most mass
    value[2, 5] = -math.inf
    z[2, int(index[2, 5])] = bad                               # named, without mass
    z[3, int(index[3, 7])] = bad                               # named, and nothing beside the named ones
    mask = torch.ones(V, dtype=torch.bool, device="cuda")
    mask[index[3].long()] = False
    z[3, mask] = -math.inf
    z[4, next(t for t in range(V) if t not in inside)] = bad   # not named
    z[4, int(index[4, 2])] = bad                               # and named
    z[5, next(t for t in range(V) if t not in set(index[5].tolist()))] = bad
    loss, grad, status = dsbd.distill(z, value, index, rest=left)
    assert int(status) == 0
    assert bool(loss[1:].isnan().all()) and bool(grad[1:].isnan().all())
    assert torch.equal(loss[:1], want[0][:1]) and torch.equal(grad[:1], want[1][:1])
    assert bool(dsbd.distill(z, value, index, rest=left, grad=None)[0][1:].isnan().all())
