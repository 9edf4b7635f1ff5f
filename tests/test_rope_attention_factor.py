"""The factor on cosines and sines of the RAMP scaling: given, left to the formula, or refused."""
import math

import pytest

import paper_2409_16560_b200 as dsbd

RAMP = dict(kind="ramp", factor=16.0, original=4096, low=1, high=32)


def test_given_and_default():
    assert dsbd.rope_frequencies(64, scaling=dict(RAMP, attention=1.25))[1] == 1.25
    assert dsbd.rope_frequencies(64, scaling=dict(RAMP, attention=0.0))[1] == 0.1 * math.log(16.0) + 1.0
    assert dsbd.rope_frequencies(64, scaling=dict(kind="linear", factor=2.0, attention=7.0))[1] == 1.0


@pytest.mark.parametrize("attention", [-1.0, -1e-300, float("nan"), float("inf"), float("-inf")])
def test_a_factor_that_is_none_is_refused(attention):
    with pytest.raises(dsbd.DsbdError) as e:
        dsbd.rope_frequencies(64, scaling=dict(RAMP, attention=attention))
    assert e.value.code == -1
