"""The polynomial by which GELU's kernels compute the normal distribution's share, as it stands in their source, against erfc in 64 bits."""
import math
import os
import re

import numpy as np
import pytest

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2102_08124_amd", "csrc", "tmask_norm.hip")


@pytest.fixture(scope="module")
def source():
    with open(SOURCE) as f:
        return f.read()


def share(source, a):
    """of -a, for a >= 0"""
    body = source[source.index("float gelu(float u)"):]
    scale = float(re.search(r"rcpf\(fmaf\(([\d.]+)f, a, 1\.f\)\)", body).group(1))
    highest, c = re.search(r"float q = fmaf\((-?[\d.]+)f, t, (-?[\d.]+)f\);", body).groups()
    coefficients = [highest, c] + re.findall(r"q = fmaf\(q, t, (-?[\d.]+)f\);", body)
    assert len(coefficients) == 5
    t = 1 / (1 + float(np.float32(scale)) * a)
    q = np.zeros_like(a)
    for k in coefficients:
        q = q * t + float(np.float32(k))
    return q * t * np.exp(-0.5 * a * a)


def test_the_share_is_as_good_as_is_said(source):
    """The most by which it is off, in 64 bits, is the figure that stands beside the coefficients, rounded up to two digits."""
    a = np.linspace(0, 12, 200001)
    exact = 0.5 * np.vectorize(math.erfc)(a / math.sqrt(2))
    worst = np.abs(share(source, a) - exact).max()
    said = float(re.search(r"off by at most ([\d.]+e-\d+)", source).group(1))
    assert worst <= said <= 1.02 * worst


def test_the_tail_is_not_as_good_as_its_own_size(source):
    """What the header says of u = -4, -5 and -6: parts of the value of 4e-4, 1e-3 and 2e-3."""
    for a, part in ((4.0, 4e-4), (5.0, 1e-3), (6.0, 2e-3)):
        exact = 0.5 * math.erfc(a / math.sqrt(2))
        assert part / 4 < abs(share(source, np.array([a]))[0] - exact) / exact < part


def test_the_share_of_fp32_numbers(source):
    """Both of its polynomials, in 64 bits, with the figures that stand beside them; below 1.25 and from there on."""
    body = source[source.index("float gelu(float u)"):]
    scale = float(np.float32(re.search(r"s = __builtin_amdgcn_rcpf\(fmaf\(([\d.]+)f, a, 1\.f\)\)", body).group(1)))
    number = r"(-?[\d.e-]+)f"
    coefficients = {name: list(re.search(r"float %s = fmaf\(%s, %s, %s\);" % (name, number, by, number), body).groups()) +
                    re.findall(r"%s = fmaf\(%s, %s, %s\);" % (name, name, by, number), body) for name, by in (("far", "s"), ("near", "u2"))}
    assert len(coefficients["far"]) == 5 and len(coefficients["near"]) == 6

    def polynomial(name, x):
        v = np.zeros_like(x)
        for k in coefficients[name]:
            v = v * x + float(np.float32(k))
        return v

    a = np.linspace(0, 13, 200001)
    exact = 0.5 * np.vectorize(math.erfc)(a / math.sqrt(2))
    limit = float(re.search(r"a < ([\d.]+)f \?", body).group(1))
    near, far = a <= limit, a >= limit
    t = 1 / (1 + scale * a)
    off_far = np.abs(polynomial("far", t) * t * np.exp(-0.5 * a * a) - exact)
    assert np.abs(0.5 - a * polynomial("near", a * a) - exact)[near].max() <= 3.6e-9
    assert off_far[far].max() <= 1.4e-8 and (off_far / exact)[far].max() <= 1.3e-5
