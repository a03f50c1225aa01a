"""The normal distribution function of gelu and its slope: the FP32 steps of csrc/act.h, repeated here, against float64.

The coefficients are read from the source.  An FP32 operation is float64's rounded to FP32 (a product of two FP32 values is
exact in float64, so a fused multiply-add rounds twice there, which moves its result by 2^-29 of an ulp's weight at most);
the hardware's reciprocal and power of two, good to one ulp, are taken correctly rounded, with one ulp either way.
"""
import math
import os
import re

import numpy as np
import pytest

from tests.libqe import ROOT

SOURCE = open(os.path.join(ROOT, "paper_2609_23536_amd", "csrc", "act.h")).read()
BODY = SOURCE[SOURCE.index("float normal_cdf(float z, float &e)"):]
BODY = BODY[:BODY.index("\n}")]
NUMBER = r"(-?\d\.\d+(?:e-\d+)?)f"
NEAR = [float(v) for v in re.findall(r"\bc = (?:__builtin_fmaf\(c, q, )?" + NUMBER, BODY)]
FAR = [float(v) for v in re.findall(r"\bs = (?:__builtin_fmaf\(s, t, )?" + NUMBER, BODY)]
f32 = np.float32


def fma(a, b, c):
    return f32(a.astype(np.float64) * np.float64(b) + np.float64(c))


def ulps(x, n):
    return (x.view(np.int32) + np.int32(n)).view(f32)


def normal_cdf(z, rcp_off=0, exp_off=0):
    q, a = f32(z * z), np.abs(z)
    c = np.full_like(z, f32(NEAR[0]))
    for k in NEAR[1:]:
        c = fma(c, q, f32(k))
    near = fma(z, c, 0.5)
    t = ulps(f32(1.0 / fma(a, f32(0.45), 1.0).astype(np.float64)), rcp_off)
    e = ulps(f32(np.exp2(f32(q * f32(-0.72134752044448170368)).astype(np.float64))), exp_off)
    s = np.full_like(z, f32(FAR[0]))
    for k in FAR[1:]:
        s = fma(s, t, f32(k))
    s = f32(s * f32(t * e))
    return np.where(a < 1.5, near, np.where(z < 0, s, f32(1.0 - s.astype(np.float64))))


def exact(z):
    return 0.5 * np.vectorize(math.erfc)(-z.astype(np.float64) / math.sqrt(2.0))


def test_the_source_has_the_steps_repeated_here():
    assert len(NEAR) == 11 and len(FAR) == 7
    for line in ("__builtin_fmaf(z, c, 0.5f)", "__builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.45f, 1.0f))",
                 "__builtin_amdgcn_exp2f(q * -0.72134752044448170368f)", "s *= t * e;", "a < 1.5f ? near : (z < 0.0f ? s : 1.0f - s)"):
        assert line in BODY, line


@pytest.mark.parametrize("rcp_off,exp_off", [(0, 0), (1, 1), (-1, -1)])
def test_off_by_less_than_8e_8(rcp_off, exp_off):
    """7.1e-8 with correctly rounded reciprocal and power; an ulp of either is 1.2e-7 of Phi(-a) <= 0.067: 8e-9 each."""
    z = np.concatenate([np.linspace(-9, 9, 400001), np.linspace(-1.6, 1.6, 200001)]).astype(f32)
    most = np.abs(normal_cdf(z, rcp_off, exp_off).astype(np.float64) - exact(z)).max()
    assert most <= (7.15e-8 if rcp_off == 0 else 7.15e-8 + 2 * 8.1e-9)


def test_series_and_fit_without_rounding():
    """The figures of the source's comment: what the two forms are off by in exact arithmetic."""
    z = np.linspace(-1.5, 1.5, 100001)
    omitted = 1.5 ** 23 / (math.sqrt(2 * math.pi) * math.factorial(11) * 2 ** 11 * 23)
    assert 2.3e-9 < omitted < 2.5e-9
    near = 0.5 + z * np.polyval([float(f32(c)) for c in NEAR], z * z)
    assert 9e-9 < np.abs(near - exact(z)).max() < 1.1e-8
    a = np.linspace(1.5, 12, 100001)
    t = 1.0 / (1.0 + float(f32(0.45)) * a)
    fit = t * np.polyval([float(f32(c)) for c in FAR], t) * np.exp(-0.5 * a * a)
    off = np.abs(fit / exact(-a) - 1.0).max()
    assert 2.4e-7 < off < 2.6e-7
