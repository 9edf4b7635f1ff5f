"""The cubic that the attention of a chunk takes some of its weights by, over its range, in fp32 on the host: its coefficients are read
from the source, its steps are those of a fused multiply-add (a product and a sum in 64 bits, rounded once)."""
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_16560_b200", "csrc",
                      "dsbd_chunk_attention.cu")


def _coefficients():
    body = open(SOURCE).read().split("F2 exp2_poly(F2 z) {")[1].split("\n}")[0]
    c = [np.float32(x) for x in re.findall(r"F2\{(0\.\d+)f, 0\.\d+f\}", body)]
    assert len(c) == 3
    return c[0], c[1], c[2], np.float32(1.0)


def _exp2(z):
    f32 = np.float32
    z = np.fmax(z.astype(f32), f32(-127.0))
    r = (z + f32(12582912.0)).astype(f32)
    f = z - (r - f32(12582912.0))                             # exact
    c3, c2, c1, c0 = _coefficients()
    fma = lambda a, b, c: (a.astype(np.float64) * b.astype(np.float64) + np.float64(c)).astype(f32)
    p = fma(f, np.full_like(f, c3), c2)
    p = fma(p, f, c1)
    p = fma(p, f, c0)
    return (p.view(np.int32) + (r.view(np.int32) << 23)).view(f32)


def test_relative_error_over_the_range():
    # the weights' exponents: up to 8 above the reference, down to the smallest normal number
    z = np.linspace(-126.0, 8.5, 4_000_001).astype(np.float32)
    err = _exp2(z).astype(np.float64) / np.exp2(z.astype(np.float64)) - 1
    assert np.abs(err).max() <= 1.02e-4                       # what the cubic's fit leaves, 1.014e-4, and roundings of 2^-24
    whole = np.arange(-126, 9).astype(np.float32)
    assert np.array_equal(_exp2(whole), np.exp2(whole))       # exact where the fraction is 0


def test_below_the_range():
    z = np.array([-127.0, -127.5, -1e4, -3e38, -np.inf], np.float32)
    assert not _exp2(z).any()
    z = np.linspace(-127.0, -126.0, 10001).astype(np.float32)
    got = _exp2(z).astype(np.float64)
    assert (got >= 0).all() and (got <= 2.0 ** -126 * (1 + 2e-4)).all()
