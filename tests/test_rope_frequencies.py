"""Frequencies of the rotations and their changes for long contexts (host side), against plain statements of the formulas."""
import math

import numpy as np
import pytest

import paper_2409_16560_b200 as dsbd


def test_plain_linear_and_base():
    for rot in (2, 16, 96, 128):
        want = np.array([10000.0 ** (-2 * i / rot) for i in range(rot // 2)])
        f, att = dsbd.rope_frequencies(rot)
        assert np.allclose(f, want, rtol=1e-14) and att == 1.0
        f, att = dsbd.rope_frequencies(rot, scaling=dict(kind="linear", factor=4.0))
        assert np.allclose(f, want / 4, rtol=1e-14) and att == 1.0
        if rot > 2:
            f, _ = dsbd.rope_frequencies(rot, scaling=dict(kind="base", factor=8.0))
            # the first frequency stays 1, the last is divided by the factor
            assert f[0] == 1.0 and abs(f[-1] * 8 / want[-1] - 1) < 1e-12
    f, _ = dsbd.rope_frequencies(64, base=5e5, scaling=dict(kind="linear", factor=1.0))
    assert np.allclose(f, dsbd.rope_frequencies(64, base=5e5)[0], rtol=0)


def test_wavelength():
    rot, base, s, o, low, high = 128, 500000.0, 8.0, 8192.0, 1.0, 4.0
    got, att = dsbd.rope_frequencies(rot, base, dict(kind="wavelength", factor=s, original=o, low=low, high=high))
    seen = set()
    for f, w in zip(got, dsbd.rope_frequencies(rot, base)[0]):
        length = 2 * math.pi / w
        if length < o / high:
            want, kind = w, "kept"
        elif length > o / low:
            want, kind = w / s, "divided"
        else:
            t = (o / length - low) / (high - low)
            want, kind = (1 - t) * w / s + t * w, "blended"
        seen.add(kind)
        assert abs(f / want - 1) < 1e-12
    assert att == 1.0 and seen == {"kept", "divided", "blended"}


def test_ramp():
    rot, base, s, o, low, high = 128, 10000.0, 16.0, 4096.0, 1.0, 32.0
    got, att = dsbd.rope_frequencies(rot, base, dict(kind="ramp", factor=s, original=o, low=low, high=high))
    at = lambda turns: rot * math.log(o / (turns * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
    for i, (f, w) in enumerate(zip(got, dsbd.rope_frequencies(rot, base)[0])):
        t = min(max((i - lo) / (hi - lo), 0), 1)
        assert abs(f / (w / s * t + w * (1 - t)) - 1) < 1e-12
    assert abs(att - (0.1 * math.log(s) + 1)) < 1e-15
    assert dsbd.rope_frequencies(rot, base, dict(kind="ramp", factor=s, original=o, low=low, high=high, attention=0.5))[1] == 0.5


@pytest.mark.parametrize("rot,base,scaling,code", [
    (3, 1e4, None, -1), (0, 1e4, None, -1), (130, 1e4, None, -1), (64, 1.0, None, -1), (64, float("nan"), None, -1),
    (64, 1e4, dict(kind="linear", factor=0.5), -1), (2, 1e4, dict(kind="base", factor=2.0), -1),
    (64, 1e4, dict(kind="wavelength", factor=2.0, original=0, low=1, high=4), -1),
    (64, 1e4, dict(kind="ramp", factor=2.0, original=100, low=4, high=4), -1),
    (64, 1e4, dict(kind="ramp", factor=float("inf"), original=100, low=1, high=4), -1)])
def test_refusals(rot, base, scaling, code):
    with pytest.raises(dsbd.DsbdError) as e:
        dsbd.rope_frequencies(rot, base, scaling)
    assert e.value.code == code


def test_no_cpu_path():
    import torch
    with pytest.raises(RuntimeError):
        dsbd.rope_table(4, 16, table=torch.zeros(4, 2, 8))
    with pytest.raises(RuntimeError):
        dsbd.Rope(torch.zeros(4, 2, 8))
