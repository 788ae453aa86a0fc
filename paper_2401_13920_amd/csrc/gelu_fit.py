"""Writes gelu_coef.h: the polynomial behind the fast GeLU of the bf16 FFN epilogue (Eq. 1's activation), and
gelu_coef_f32.h: one of higher degree, for values that stay in fp32.

GeLU(v) = v Phi(v) = max(v, 0) - |v| Phi(-|v|).  log2(2 Phi(-x)) is smooth on x >= 0 (a parabola plus a slowly
varying term), so one polynomial q(x) of degree 6 on [0, 6] and one exp2 give Phi(-x) to a relative error below
5e-5, forty times finer than the bf16 rounding of the result.  Past x = 6 the argument is clamped: the true
tail is below 6e-9 there.  The fit is weighted least squares on Chebyshev nodes with Lawson's reweighting
(converges to the minimax polynomial).  With degree 11 the error of GeLU(v) is below 8e-8 |v|, a rounding step of fp32.

Run:  python gelu_fit.py   (rewrites gelu_coef.h and gelu_coef_f32.h beside this file)
"""
import os

import numpy as np
from numpy.polynomial import Polynomial, chebyshev
from scipy.special import log_ndtr

X_MAX = 6.0
DEGREE = 6
DEGREE_F32 = 11


def fit(degree):
    t = np.cos(np.pi * (np.arange(4000) + 0.5) / 4000)           # Chebyshev nodes on [-1, 1]
    x = (t + 1.0) * (X_MAX / 2)
    target = log_ndtr(-x) / np.log(2.0) + 1.0                    # log2(2 Phi(-x))
    w = np.ones_like(t)
    for _ in range(200):
        c = chebyshev.chebfit(t, target, degree, w=np.sqrt(w))
        w *= np.abs(chebyshev.chebval(t, c) - target)
        w /= w.sum()
    in_t = Polynomial(chebyshev.cheb2poly(c))
    return in_t(Polynomial([-1.0, 2.0 / X_MAX])).coef            # power basis in x


def write(name, degree, lines):
    coef = [float(np.float32(v)) for v in fit(degree)]
    text = ["// Generated by gelu_fit.py; do not edit.  q(x) = sum c[k] x^k approximates log2(2 Phi(-x)) on [0, 6].",
            "#pragma once", "namespace locmoe {", *lines, *(f"    {v!r}f," for v in coef), "};", "}  // namespace locmoe", ""]
    with open(os.path.join(os.path.dirname(os.path.abspath(__file__)), name), "w") as f:
        f.write("\n".join(text))


def main():
    write("gelu_coef.h", DEGREE, [f"constexpr float kGeluXMax = {X_MAX!r}f;", f"constexpr int kGeluDegree = {DEGREE};",
                                  "constexpr float kGeluCoef[kGeluDegree + 1] = {"])
    write("gelu_coef_f32.h", DEGREE_F32, [f"constexpr int kGeluDegreeF32 = {DEGREE_F32};",
                                          "constexpr float kGeluCoefF32[kGeluDegreeF32 + 1] = {"])


if __name__ == "__main__":
    main()
