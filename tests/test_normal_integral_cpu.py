"""The polynomial of the normal distribution's integral, as the gated block's source has it, against the function that it stands for."""
import os
import re

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_05632_amd", "csrc")


def source():
    text = open(os.path.join(CSRC, "compams_gated.hip")).read()
    at = text.index("float normal_cdf(")
    return text[:at], text[at:at + text[at:].index("\n}\n")]


def test_polynomial_is_as_near_as_its_comment_says():
    """The coefficients of the source, from the highest power down, in 64 bits."""
    erfcx = pytest.importorskip("scipy.special").erfcx
    before, body = source()
    first = re.search(r"float p = (-?[0-9.e-]+)f;", body).group(1)
    powers = [np.float64(np.float32(v)) for v in [first] + re.findall(r"p = fmaf\(p, t, (-?[0-9.e-]+)f\);", body)]
    off, of_value = (float(v) for v in re.findall(r"off by ([0-9.]+e-[0-9]+) at most, ([0-9.]+e-[0-9]+) of the value", before)[-1])
    z = np.linspace(0.0, 10.2, 200001)
    want = (1.0 + 2.0 * z) * erfcx(z)
    got = np.polyval(powers, (z - 2.0) / (z + 2.0))
    assert len(powers) == 10
    assert 0.9 * off < np.abs(got - want).max() <= off and 0.9 * of_value < np.abs(got / want - 1.0).max() <= of_value
