"""What the coefficients of the block kernels' GELU are good for, as they stand in the source, in float arithmetic with the exponential correctly rounded."""
import os
import re

import numpy as np
from scipy.special import log_ndtr, ndtr

from paper_1902_04610_amd import build


def coefficients(function):
    with open(os.path.join(build.CSRC, "block.hpp")) as f:
        body = re.search(r"float %s\(float c\)\n\{(.*?)\n\}" % function, f.read(), re.S).group(1)
    return [np.float32(v) for v in re.findall(r"(-?\d+\.\d+(?:e-\d+)?)f", body.split("__builtin")[0])]


def horner(coef, c):
    p = np.full_like(c, coef[0])
    for k in coef[1:]:
        p = np.float32(p.astype(np.float64) * c.astype(np.float64) + np.float64(k))      # one rounding: the product of two floats is exact
    return p


def test_gelu_of_float_results_is_right_in_its_tail():
    near, far = coefficients("tail_exponent"), coefficients("normal_tail_far")
    assert (len(near), len(far)) == (9, 8)
    x = np.linspace(3.25, 13, 1 << 18)
    assert np.abs(np.polyval(np.float64(far), x) * np.log(2) - log_ndtr(-x)).max() < 1.1e-5
    z = np.concatenate([np.linspace(-12.9, 12.9, 1 << 20), [-3.25, np.nextafter(np.float32(-3.25), np.float32(0))]]).astype(np.float32)
    c = np.minimum(np.abs(z), np.float32(13))
    q = np.exp2(np.where(c < np.float32(3.25), horner(near, c), horner(far, c)).astype(np.float64)).astype(np.float32)
    got = np.float64(np.float32(-c.astype(np.float64) * q + np.maximum(z, 0).astype(np.float64)))
    want = np.float64(z) * ndtr(np.float64(z))
    off, below = np.abs(got - want), z < 0
    assert (off <= 1.2e-7 * np.abs(np.float64(z))).all()
    assert (off[below] <= 2.1e-5 * np.abs(want[below])).all()
    assert (off[below & (z > -3.25)] <= 2.5e-6 * np.abs(want[below & (z > -3.25)])).all()
