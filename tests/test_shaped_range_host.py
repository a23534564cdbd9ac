"""What the calls over the paged cache make of their arguments at the ends of the ranges, and the polynomials there; no GPU needed."""
import os
import re

import numpy as np

from paper_2605_06068_b200 import binding as pda


def source(name):
    return open(os.path.join(os.path.dirname(pda.__file__), "csrc", name)).read()


def test_polynomial_of_scores_below_a_cap_is_within_its_bound():
    """Relative to the score, in 64 bits and in 32 (a rounding for each of its steps)."""
    text = re.search(r"PDA_TANH_COEFFICIENTS \\\n\s*\{([^}]*)\}", source("shaped.cuh")).group(1)
    c = [float(x.strip().rstrip("f")) for x in text.split(",")]
    reach = float(re.search(r"kTanhReach = ([\d.]+)f", source("shaped.cuh")).group(1))
    x = np.linspace(1e-6, reach, 400001)
    assert np.abs(x * np.polyval(c[::-1], x * x) / np.tanh(x) - 1).max() < 2.0 ** -24.9
    f = x.astype(np.float32)
    t = f * f
    y = np.full(f.shape, c[-1], dtype=np.float32)
    for a in c[-2::-1]:
        y = y * t + np.float32(a)
    assert np.abs((f * y).astype(np.float64) / np.tanh(f.astype(np.float64)) - 1).max() < 2.0 ** -24.9 + (2 * len(c) + 2) * 2.0 ** -24
