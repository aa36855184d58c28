"""Constants of the attention kernels against the functions they stand for, in 64 bits."""
from __future__ import annotations

import os
import re

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_cap_s_polynomial_is_as_close_to_tanh_as_its_comment_says():
    text = open(os.path.join(ROOT, "paper_2607_10987_b200", "csrc", "attend_wide.cu")).read()
    stated = float(re.search(r"linear programming: ([0-9.e-]+) with the coefficients", text).group(1))
    most = float(re.search(r"TANH_POLY_MAX = ([0-9.]+)f;", text).group(1))
    c = [np.float32(m) for m in re.findall(r"c\[[1-4]\] = (-?[0-9.]+)f \* times", text)]
    assert re.search(r"c\[0\] = times;", text) and len(c) == 4
    y = np.linspace(1e-4, most, 200001)
    p = 1.0 + sum(float(k) * y ** (2 * i + 2) for i, k in enumerate(c))
    assert np.abs(p * y / np.tanh(y) - 1).max() <= stated
