"""What the C ABI of the draws, the largest logits and the distillation refuses on the host, before anything is launched (so without a device:
the addresses are never followed)."""
import ctypes as C
import math

import pytest

import paper_2409_16560_b200 as dsbd
from paper_2409_16560_b200.binding import DTYPE_BF16, DTYPE_F32, DistillParamsT, RowsT, SampleParamsT

OK, INVALID, UNSUPPORTED = 0, -1, -2
AT = 1 << 20                                                   # an aligned address that nobody reads


def rows(logits=AT, stride=100, n=3, V=100, dtype=DTYPE_F32):
    return RowsT(logits, stride, n, V, dtype)


def sample(r=None, uniform=AT, token=AT, logp=AT, status=AT, **kw):
    p = SampleParamsT(**dict(dict(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0, draws=1), **kw))
    return dsbd.load().dsbd_sample_rows(C.addressof(r) if r else None, C.addressof(p), uniform, token, logp, status, None)


def top(r=None, K=5, T=1.0, value=AT, index=AT, rest=AT, status=AT):
    return dsbd.load().dsbd_top_logits(C.addressof(r) if r else None, K, T, value, index, rest, status, None)


def distill(r=None, loss=AT, grad=AT, stride=100, status=AT, **kw):
    p = DistillParamsT(**dict(dict(K=5, temperature=1.0, value=AT, index=AT), **kw))
    return dsbd.load().dsbd_distill(C.addressof(r) if r else None, C.addressof(p), loss, grad, stride, status, None)


@pytest.mark.parametrize("call", [sample, top, distill])
def test_rows(call):
    assert call(None) == INVALID
    for bad in (dict(n=-1), dict(V=0), dict(V=-3), dict(stride=99), dict(stride=0), dict(stride=-100), dict(logits=None)):
        assert call(rows(**bad)) == INVALID, bad
    for bad in (dict(dtype=7), dict(logits=AT + 2), dict(logits=AT + 1, dtype=DTYPE_BF16), dict(V=393217, stride=400000),
                dict(V=786433, stride=800000, dtype=DTYPE_BF16), dict(n=1 << 28)):
        assert call(rows(**bad)) == UNSUPPORTED, bad
    assert call(rows(n=0)) == OK                               # nothing to do: nothing is launched
    assert call(rows(n=0, logits=None)) == OK
    assert call(rows(), status=None) == INVALID


def test_sample_settings():
    for bad in (dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan), dict(top_p=0.0), dict(top_p=-0.5),
                dict(top_p=math.nan), dict(min_p=-0.1), dict(min_p=1.1), dict(min_p=math.nan), dict(draws=-1)):
        assert sample(rows(), **bad) == INVALID, bad
    assert sample(rows(), uniform=None) == INVALID and sample(rows(), token=None) == INVALID
    assert sample(rows(), draws=0) == OK


def test_top_settings():
    for bad in (dict(K=0), dict(K=-1), dict(K=101), dict(T=0.0), dict(T=-1.0), dict(T=math.inf), dict(T=math.nan), dict(value=None),
                dict(index=None)):
        assert top(rows(), **bad) == INVALID, bad
    assert top(rows(V=5000, stride=5000), K=1025) == UNSUPPORTED


def test_distill_settings():
    for bad in (dict(K=0), dict(K=101), dict(temperature=0.0), dict(temperature=-2.0), dict(temperature=math.inf), dict(temperature=math.nan),
                dict(value=None), dict(index=None), dict(loss=None), dict(stride=99), dict(stride=-1)):
        assert distill(rows(), **bad) == INVALID, bad
    assert distill(rows(V=5000, stride=5000), K=1025, stride=5000) == UNSUPPORTED
    assert distill(rows(), grad=AT + 2) == UNSUPPORTED and distill(rows(dtype=DTYPE_BF16), grad=AT + 1) == UNSUPPORTED


def test_temperatures_that_sums_in_32_bits_do_not_reach():
    for T in (2.0 ** -127, 1e-40, 2.0 ** 101, 3e38):
        assert top(rows(), T=T) == INVALID and distill(rows(), temperature=T) == INVALID
    for T in (2.0 ** -126, 2.0 ** 100):
        assert top(rows(n=0), T=T) == OK and distill(rows(n=0), temperature=T) == OK
