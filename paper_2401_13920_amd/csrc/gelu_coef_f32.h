// Generated by gelu_fit.py; do not edit.  q(x) = sum c[k] x^k approximates log2(2 Phi(-x)) on [0, 6].
#pragma once
namespace locmoe {
constexpr int kGeluDegreeF32 = 11;
constexpr float kGeluCoefF32[kGeluDegreeF32 + 1] = {
    6.297657506593168e-08f,
    -1.1511070728302002f,
    -0.4592014253139496f,
    -0.05248810350894928f,
    0.006996306125074625f,
    -2.064089130726643e-05f,
    -0.0002823321265168488f,
    8.251195686170831e-05f,
    -1.347144916508114e-05f,
    1.3597394854514278e-06f,
    -7.925083878035366e-08f,
    2.045260183436426e-09f,
};
}  // namespace locmoe
