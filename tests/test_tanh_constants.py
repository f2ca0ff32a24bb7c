"""The tanh polynomials of the log probabilities (csrc/logprob_kernels.h): their constants are the committed fits', and with the powers of scale / cap folded into them x stays within 2^-20 of
itself in float32 wherever the kernel takes them."""
import importlib.util
import os
import re

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_13062_amd", "csrc")
LOG2E = np.float32(1.4426950408889634)


def header(name):
    text = open(os.path.join(CSRC, "logprob_kernels.h")).read()
    return [float(x) for x in re.search(r"%s\[\d\] = \{([^}]*)\}" % name, text).group(1).replace("f", "").split(",")]


def module():
    spec = importlib.util.spec_from_file_location("tanh_fit", os.path.join(CSRC, "tanh_fit.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("name", ["Near", "Wide"])
def test_constants_are_the_committed_fit(name):
    m = module()
    reach, degree = getattr(m, name.upper())
    assert header("kTanh%sFit" % name) == m.fit(reach, degree)
    text = open(os.path.join(CSRC, "logprob_kernels.h")).read()
    assert float(re.search(r"kTanh%s = ([0-9.]+)f" % name, text).group(1)) == reach
    # In units of 2^-24: the fit leaves 0.97 (5.8e-8, the wide one) and its first coefficient's rounding 0.5; the last sum, of 0.83 to 1, is rounded by 0.6, the last product by 1; u^2 by 1, of which
    # a sixth arrives (d log P / d log u^2 up to 0.16); the sums before, below 0.34 and times 0.64, by 0.2 together: 3.5, below 2^-22.
    assert m.max_relative_error(header("kTanh%sFit" % name), reach) < 2.0 ** -22


@pytest.mark.parametrize("name", ["Near", "Wide"])
def test_folded_powers(name):
    """Any scale and cap: either the last coefficient is no normal number, and the kernel takes another form, or all of them are and x is near."""
    m = module()
    reach, degree = getattr(m, name.upper())
    fit, f, rng = [np.float32(c) for c in header("kTanh%sFit" % name)], np.float32, np.random.default_rng(0)
    taken = 0
    with np.errstate(all="ignore"):
        for _ in range(5000):
            scale, cap = f(10 ** rng.uniform(-30, 30)), f(10 ** rng.uniform(-30, 5.7))
            u1 = f(scale * f(f(1) / cap))
            u2, power, c = f(u1 * u1), f(scale * LOG2E), []
            for x in fit:
                c.append(f(power * x))
                power = f(power * u2)
            if not 2.0 ** -126 <= abs(c[-1]) < np.inf:
                continue
            assert all(2.0 ** -126 <= abs(x) < np.inf for x in c)
            u = np.concatenate([rng.uniform(-reach, reach, 50), 10 ** rng.uniform(-8, np.log10(reach), 50)])
            v = (u * float(cap) / float(scale)).astype(f)
            v = v[(np.abs(v) > 1e-37) & (np.abs(v) < 3e38)]
            q, p = (v * v).astype(f), np.full_like(v, c[-1])
            for x in c[-2::-1]:
                p = (p.astype(np.float64) * q + x).astype(f)
            x, want = (v * p).astype(np.float64), np.tanh(float(scale) * v.astype(np.float64) / float(cap)) * float(cap) * 1.4426950408889634
            near = np.abs(want) > 1e-36                       # below it products leave the normal numbers: nothing to a logarithm
            assert (np.abs(x - want)[near] <= 2.0 ** -20 * np.abs(want)[near]).all(), (scale, cap)
            taken += 1
    assert taken > 300
