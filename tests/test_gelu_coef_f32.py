"""The GeLU of the few-token layer's fp32 path, checked on the CPU against the oracle's erf form: the kernel's steps (as in
test_gelu_coef.py) with the polynomial of higher degree.  Stated error: below 8e-8 |v|."""
import os
import re

import numpy as np

from oracle import locmoe_oracle as oracle

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2401_13920_amd", "csrc")


def _gelu(v):
    text = open(os.path.join(CSRC, "gelu_coef_f32.h")).read()
    x_max = np.float32(re.search(r"kGeluXMax = ([-0-9.e+]+)f", open(os.path.join(CSRC, "gelu_coef.h")).read()).group(1))
    coef = [np.float32(m) for m in re.findall(r"^\s+([-0-9.e+]+)f,", text, flags=re.M)]
    assert len(coef) == int(re.search(r"kGeluDegreeF32 = (\d+)", text).group(1)) + 1
    v = v.astype(np.float32)
    x = np.minimum(np.abs(v), x_max)
    q = np.full_like(x, coef[-1])
    for c in coef[-2::-1]:  # (a fused multiply-add rounds once)
        q = (q.astype(np.float64) * x + np.float64(c)).astype(np.float32)
    h2 = np.exp2(q.astype(np.float64)).astype(np.float32)
    s = (v + np.abs(v)).astype(np.float32)
    return np.float32(0.5) * (s.astype(np.float64) - x.astype(np.float64) * h2).astype(np.float32)


def test_error_is_a_rounding_step_of_fp32():
    rng = np.random.default_rng(6)
    v = np.concatenate([np.linspace(-40.0, 40.0, 400001), rng.normal(0.0, 1.3, 400000), [0.0, -0.0, 1e-30, -1e-30, 1e30, -1e30]])
    v = v.astype(np.float32)
    err = np.abs(_gelu(v).astype(np.float64) - oracle.gelu(v.astype(np.float64)))
    assert np.all(err <= 8e-8 * np.abs(v.astype(np.float64))), v[np.argmax(err / np.maximum(np.abs(v), 1e-300))]


def test_limits():
    got = _gelu(np.array([np.inf, np.nan, 100.0, -100.0], dtype=np.float32))
    assert got[0] == np.inf and np.isnan(got[1]) and got[2] == 100.0 and abs(got[3]) < 1e-8 * 100
