"""The formula that bf16 results of GELU take for the tail of the normal distribution, with its constants as they stand in the source, against the
function itself: off by 6e-8 and by 2.5e-4 of itself at most, without the roundings of fp32."""
import os
import re

import numpy as np
from scipy import special

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_11469_amd", "csrc")


def constants():
    text = open(os.path.join(CSRC, "zr_act.h")).read()
    body = text[text.index("void gelu_of("):text.index("const float tail")]
    body = body[body.index("rcpf("):]
    slope = float(re.search(r"rcpf\(fmaf\(([-.\d]+)f, fabsf\(z\), 1\.f\)\)", body)[1])
    first = float(re.search(r"float p = ([-.\d]+)f;", body)[1])
    return slope, [first] + [float(v) for v in re.findall(r"p = fmaf\(p, t, ([-.\d]+)f\);", body)]


def test_tail_of_the_normal_distribution():
    slope, c = constants()
    assert len(c) == 6
    x = np.concatenate([np.linspace(0, 13.2, 400001), 2.0 ** np.arange(-30, 0)])
    t = 1 / (1 + slope * x)
    T = np.polyval(c, t) * t * np.exp(-x * x / 2)
    true = special.ndtr(-x)
    assert (abs(T - true) <= 6e-8).all() and (abs(T - true) <= 2.5e-4 * true).all()
