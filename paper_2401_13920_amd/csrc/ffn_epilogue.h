// The expert FFN's epilogues, shared by its GEMM kernels.
#pragma once
#include "common.h"
#include "gelu_coef.h"

namespace locmoe {

// What happens to an accumulator on its way to memory
constexpr int kEpiNone = 0;      // rounded and stored
constexpr int kEpiGelu = 1;      // GeLU, then rounded and stored (H of Eq. 1)
constexpr int kEpiGeluSave = 2;  // the same, and the pre-activation Z is stored (bf16) to `aux` for the backward
constexpr int kEpiGeluGrad = 3;  // multiplied by GeLU'(Z), Z read from `aux` (bf16): dZ = dH * GeLU'(Z)
constexpr int kEpiGeluSave8 = 4; // GeLU, stored, and the pre-activation kept in 8 bits (Act8)
constexpr int kEpiGeluGrad8 = 5; // multiplied by GeLU' of what the 8 bits stand for, whose GeLU is stored as well

// The pre-activations in 8 bits: q = rint(z / unit) for blocks of 16 columns of a row, unit = max |z| / 127 rounded to bf16
// (its relative rounding of at most 2^-8 leaves |q| <= 127.497, which rounds to 127).  16 columns are one MFMA tile's, so a
// block lies in four lanes of one wave whatever the tile.  At 9 bits a value it is 0.3 to 0.5 % off (root mean square, of
// normally distributed z), where 8 bits with an exponent each (e4m3) are 2.6 % off.
// A block with an infinity or a NaN reads back as NaN; one below 127 x 2^-126 as zeros.
struct Act8 {
  int8_t* q;       // [rows][N]
  uint16_t* unit;  // [rows][ceil(N / 16)] bf16
  uint16_t* H;     // kEpiGeluGrad8: [rows][N] bf16, GeLU of what q stands for
};
template <int EPI>
struct AuxType { using type = uint16_t*; };
template <>
struct AuxType<kEpiGeluSave8> { using type = Act8; };
template <>
struct AuxType<kEpiGeluGrad8> { using type = Act8; };
template <int EPI>
using AuxOf = typename AuxType<EPI>::type;

namespace {

// GeLU for outputs that are rounded to bf16: GeLU(v) = max(v,0) - |v| Phi(-|v|), with
// 2 Phi(-x) = exp2(q(x)), q the degree-6 polynomial of gelu_coef.h on [0, 6] (argument clamped: the
// tail beyond is below 6e-9).  Relative error below 5e-5, absolute below 7e-6: forty times finer than
// the bf16 rounding that follows, at 10 vector ops and one transcendental per value (a rational erfc
// form with the same tail behaviour costs 15 and two; the epilogue's vector work was a tenth of the
// first GEMM's time with it).
// max(v,0) is formed as (v + |v|)/2 so that a NaN input stays a NaN.
__device__ __forceinline__ float gelu_bf16(float v) {
  const float x = fminf(fabsf(v), kGeluXMax);
  float q = kGeluCoef[kGeluDegree];
#pragma unroll
  for (int k = kGeluDegree - 1; k >= 0; --k) q = fmaf(q, x, kGeluCoef[k]);
  return 0.5f * fmaf(-x, __builtin_amdgcn_exp2f(q), v + fabsf(v));
}

// GeLU'(v) = Phi(v) + v phi(v) for factors of outputs that are rounded to bf16, from the same polynomial:
// Phi(-|v|) = exp2(q(|v|)) / 2 (absolute error below 2.3e-5), phi(v) = exp2(-v^2 log2(e)/2) / sqrt(2 pi).
__device__ __forceinline__ float gelu_grad_bf16(float v) {
  const float x = fminf(fabsf(v), kGeluXMax);
  float q = kGeluCoef[kGeluDegree];
#pragma unroll
  for (int k = kGeluDegree - 1; k >= 0; --k) q = fmaf(q, x, kGeluCoef[k]);
  const float tail = 0.5f * __builtin_amdgcn_exp2f(q);  // Phi(-|v|)
  const float Phi = v >= 0.f ? 1.0f - tail : tail;
  const float phi = 0.3989422804f * __builtin_amdgcn_exp2f(-0.7213475204f * v * v);
  return fmaf(v, phi, Phi);
}

// The largest of four lanes' values, 16 lanes apart, in all four
__device__ __forceinline__ uint32_t max_of_quads(uint32_t v) {
  auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(a[0], a[1]);
}

// One accumulator quad -> memory.  q holds D[n0..n0+3][m] for one row m.  `in`: the quad has columns below ldc (ldc and n0
// are multiples of 4); quads without are passed on for kEpiGeluSave8 alone, whose 16-column blocks are four lanes' work.
template <int EPI, bool OUT_F32>
__device__ __forceinline__ void store_quad(void* C, const AuxOf<EPI>& aux, size_t row, int ldc, int n0, float q0, float q1,
                                           float q2, float q3, bool in = true) {
  static_assert(!(EPI != kEpiNone && OUT_F32), "the hidden activations and their gradients are stored as bf16");
  if constexpr (EPI == kEpiGeluSave) *(uint2*)(aux + row * ldc + n0) = make_uint2(pack_bf16x2(q0, q1), pack_bf16x2(q2, q3));
  if constexpr (EPI == kEpiGeluSave8) {
    // (as whole numbers the magnitudes' bits are in the magnitudes' order, with infinity and NaN above all)
    const uint32_t mine = max(max(__float_as_uint(fabsf(q0)), __float_as_uint(fabsf(q1))),
                              max(__float_as_uint(fabsf(q2)), __float_as_uint(fabsf(q3))));
    const float most = __uint_as_float(max_of_quads(in ? mine : 0u)) * (1.0f / 127.0f);
    const uint16_t unit = most < 1.17549435e-38f ? 0 : f32_to_bf16_bits(most);
    const float inv = unit ? 1.0f / bf16_bits_to_f32(unit) : 0.f;
    if (!in) return;
    auto byte = [&](float v) { return (uint32_t)(int)__builtin_rintf(v * inv) & 0xFFu; };
    *(uint32_t*)(aux.q + row * ldc + n0) = byte(q0) | (byte(q1) << 8) | (byte(q2) << 16) | (byte(q3) << 24);
    if ((n0 & 15) == 0) aux.unit[row * ((ldc + 15) >> 4) + (n0 >> 4)] = unit;
  }
  if constexpr (EPI == kEpiGelu || EPI == kEpiGeluSave || EPI == kEpiGeluSave8) {
    q0 = gelu_bf16(q0); q1 = gelu_bf16(q1); q2 = gelu_bf16(q2); q3 = gelu_bf16(q3);
  }
  if constexpr (EPI == kEpiGeluGrad) {
    const uint2 z = *(const uint2*)(aux + row * ldc + n0);
    q0 *= gelu_grad_bf16(bf16_bits_to_f32(z.x & 0xFFFFu));
    q1 *= gelu_grad_bf16(__uint_as_float(z.x & 0xFFFF0000u));
    q2 *= gelu_grad_bf16(bf16_bits_to_f32(z.y & 0xFFFFu));
    q3 *= gelu_grad_bf16(__uint_as_float(z.y & 0xFFFF0000u));
  }
  if constexpr (EPI == kEpiGeluGrad8) {
    const uint32_t b = *(const uint32_t*)(aux.q + row * ldc + n0);
    const float unit = bf16_bits_to_f32(aux.unit[row * ((ldc + 15) >> 4) + (n0 >> 4)]);
    const float z0 = (float)(int8_t)b * unit, z1 = (float)(int8_t)(b >> 8) * unit;
    const float z2 = (float)(int8_t)(b >> 16) * unit, z3 = (float)(int8_t)(b >> 24) * unit;
    *(uint2*)(aux.H + row * ldc + n0) =
        make_uint2(pack_bf16x2(gelu_bf16(z0), gelu_bf16(z1)), pack_bf16x2(gelu_bf16(z2), gelu_bf16(z3)));
    q0 *= gelu_grad_bf16(z0); q1 *= gelu_grad_bf16(z1); q2 *= gelu_grad_bf16(z2); q3 *= gelu_grad_bf16(z3);
  }
  if (OUT_F32) {
    *(float4*)((float*)C + row * ldc + n0) = make_float4(q0, q1, q2, q3);
  } else {
    *(uint2*)((uint16_t*)C + row * ldc + n0) = make_uint2(pack_bf16x2(q0, q1), pack_bf16x2(q2, q3));
  }
}

}  // namespace
}  // namespace locmoe
