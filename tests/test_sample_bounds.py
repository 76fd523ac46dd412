"""The bound on what a 32-bit weight's power of two costs, which decides what 32-bit sums may decide: the arithmetic of the kernels worked
through in numpy, with scales chosen for the largest errors.  u = 2^-24.

y = x (scale log2 e) is made from a rounded constant (0.22 u), a rounded product (up to u) and a multiply-add (up to u of y); the weight 2^y is
then off by ln 2 times the error of y, relatively: 2.22 ln 2 = 1.54 |y| u at most."""
import os
import re

import numpy as np

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_17506_b200", "csrc", "vl_sample.cuh")
U = 2.0 ** -24


def _worst_error():
    """Largest |relative error of the weight| / (|y| u) that was found."""
    rng = np.random.default_rng(1)
    log2e = np.log2(np.e)                       # (64 bits)
    s = np.exp2(rng.random(400000)).astype(np.float32)
    c = s * np.float32(1.44269504088896341)     # one rounded product, as in the kernels
    off = c.astype(np.float64) / (s.astype(np.float64) * log2e) - 1.0
    worst = 0.0
    for j in (int(np.argmax(off)), int(np.argmin(off))):
        x = -(rng.random(400000) * 40).astype(np.float32)
        exact = x.astype(np.float64) * c[j].astype(np.float64)      # 48 bits: no error here
        y = exact.astype(np.float32).astype(np.float64)             # the multiply-add's rounding, relative to a largest logit of 0
        true = x.astype(np.float64) * (s[j].astype(np.float64) * log2e)
        some = np.abs(true) > 2.0 ** -10
        worst = max(worst, float((np.log(2.0) * np.abs(y - true) / (np.abs(true) * U))[some].max()))
    return worst


def test_the_stated_bound_covers_the_arithmetic():
    bound = float(re.search(r"POWER_ERROR = ([0-9.]+)f;", open(HEADER).read()).group(1))
    worst = _worst_error()
    assert 1.4 < worst <= 2.22 * np.log(2.0) + 0.01 <= bound
