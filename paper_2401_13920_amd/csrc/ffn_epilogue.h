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
constexpr bool kept8(int epi) { return epi == kEpiGeluSave8 || epi == kEpiGeluGrad8; }

// The pre-activations in 8 bits: q = rint(z / unit) for blocks of 16 columns of a row, unit = max |z| / 127 rounded to bf16
// (its relative rounding of at most 2^-8 leaves |q| <= 127.497, which rounds to 127).  16 columns are one MFMA tile's, so a
// block lies in four lanes of one wave whatever the tile.  At 9 bits a value it is 0.3 to 0.5 % off (root mean square, of
// normally distributed z), where 8 bits with an exponent each (e4m3) are 2.6 % off.
// A block with an infinity or a NaN reads back as NaN; one below 127 x 2^-126 as zeros.
// Time, T = 32 768, d = 2048, h = 8192, E = 32, 17 598 rows: the first GEMM 627 us (with Z kept in bf16 637: it stores 0.72 GB for
// 1.15; with nothing kept 560), the two GEMMs of the data gradients 1 255 (1 215: H is formed and stored again, 0.29 GB);
// T = 8192, d = 1024, h = 4096, E = 16: 121 (123; 79 to 98) and 235 (228).  A store instruction writes pieces of 16 and 32 bytes of
// 16 rows, which the GEMM's loop does not cover where a work-group has a compute unit to itself.
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
  const float x = __builtin_amdgcn_fmed3f(fabsf(v), 0.f, kGeluXMax);  // (a minimum takes two instructions, for signalling NaNs)
  float q = kGeluCoef[kGeluDegree];
#pragma unroll
  for (int k = kGeluDegree - 1; k >= 0; --k) q = fmaf(q, x, kGeluCoef[k]);
  return 0.5f * fmaf(-x, __builtin_amdgcn_exp2f(q), v + fabsf(v));
}

// Phi(v) from the same polynomial: Phi(-|v|) = exp2(q(|v|)) / 2, absolute error below 2.3e-5
__device__ __forceinline__ float normal_cdf_bf16(float v) {
  const float x = __builtin_amdgcn_fmed3f(fabsf(v), 0.f, kGeluXMax);
  float q = kGeluCoef[kGeluDegree];
#pragma unroll
  for (int k = kGeluDegree - 1; k >= 0; --k) q = fmaf(q, x, kGeluCoef[k]);
  const float tail = 0.5f * __builtin_amdgcn_exp2f(q);  // Phi(-|v|)
  return v >= 0.f ? 1.0f - tail : tail;
}
// GeLU'(v) = Phi(v) + v phi(v) for factors of outputs that are rounded to bf16, phi(v) = exp2(-v^2 log2(e)/2) / sqrt(2 pi)
__device__ __forceinline__ float gelu_grad_bf16(float v) {
  const float phi = 0.3989422804f * __builtin_amdgcn_exp2f(-0.7213475204f * v * v);
  return fmaf(v, phi, normal_cdf_bf16(v));
}

// The larger value, or NaN if either is one
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// GeLU(v) = v Phi(v) for outputs that are rounded to bf16, beside a GeLU'(v) that uses the same Phi.  Below -6 the polynomial's
// Phi stays at Phi(-6), and so must v: the product is above -6e-9, as gelu_bf16's.
__device__ __forceinline__ float gelu_by_cdf_bf16(float v) { return maximum(v, -kGeluXMax) * normal_cdf_bf16(v); }
// Four values of a lane, each to be the largest of four lanes 16 apart.  The four are reduced together: the lanes of 16-lane
// row r end with the result of value quad_of_row(r), in 3 exchanges instead of 8; spread_rows takes such a register apart again.
__device__ __forceinline__ constexpr int quad_of_row(int r) { return (r >> 1) | ((r & 1) << 1); }
__device__ __forceinline__ float max_to_rows(float v0, float v1, float v2, float v3) {
  auto pair = [](auto s) { return maximum(__uint_as_float(s[0]), __uint_as_float(s[1])); };
  const float a = pair(__builtin_amdgcn_permlane32_swap(__float_as_uint(v0), __float_as_uint(v1), false, false));
  const float b = pair(__builtin_amdgcn_permlane32_swap(__float_as_uint(v2), __float_as_uint(v3), false, false));
  return pair(__builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false));
}
__device__ __forceinline__ void spread_rows(float v, float (&out)[4]) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const auto lo = __builtin_amdgcn_permlane32_swap(a[0], a[0], false, false);
  const auto hi = __builtin_amdgcn_permlane32_swap(a[1], a[1], false, false);
  out[0] = __uint_as_float(lo[0]); out[1] = __uint_as_float(lo[1]);
  out[2] = __uint_as_float(hi[0]); out[3] = __uint_as_float(hi[1]);
}

// One accumulator quad -> memory.  q holds D[n0..n0+3][m] for one row m.
template <int EPI, bool OUT_F32>
__device__ __forceinline__ void store_quad(void* C, uint16_t* aux, size_t row, int ldc, int n0, float q0, float q1,
                                           float q2, float q3) {
  static_assert(!(EPI != kEpiNone && OUT_F32), "the hidden activations and their gradients are stored as bf16");
  if (EPI == kEpiGeluSave) *(uint2*)(aux + row * ldc + n0) = make_uint2(pack_bf16x2(q0, q1), pack_bf16x2(q2, q3));
  if (EPI == kEpiGelu || EPI == kEpiGeluSave) {
    q0 = gelu_bf16(q0); q1 = gelu_bf16(q1); q2 = gelu_bf16(q2); q3 = gelu_bf16(q3);
  }
  if (EPI == kEpiGeluGrad) {
    const uint2 z = *(const uint2*)(aux + row * ldc + n0);
    q0 *= gelu_grad_bf16(bf16_bits_to_f32(z.x & 0xFFFFu));
    q1 *= gelu_grad_bf16(__uint_as_float(z.x & 0xFFFF0000u));
    q2 *= gelu_grad_bf16(bf16_bits_to_f32(z.y & 0xFFFFu));
    q3 *= gelu_grad_bf16(__uint_as_float(z.y & 0xFFFF0000u));
  }
  if (OUT_F32) {
    *(float4*)((float*)C + row * ldc + n0) = make_float4(q0, q1, q2, q3);
  } else {
    *(uint2*)((uint16_t*)C + row * ldc + n0) = make_uint2(pack_bf16x2(q0, q1), pack_bf16x2(q2, q3));
  }
}

// The 8-bit epilogues, a row of this lane at a time: NQ quads, STEP columns apart, the first at column n0 (of which four lanes
// with the same row share a block of 16: n0 mod 16 is 0, 4, 8 and 12 in them).  Quads at or past column N are not there.
constexpr float kLeastUnit = 1.17549435e-38f;  // 2^-126
template <int NQ, int STEP>
struct Row8 {
  // the units of a row's blocks lie side by side, and a lane can take them at once
  static constexpr bool kWide = STEP == 16 && (NQ == 4 || NQ == 8);
  uint32_t q[NQ];     // four whole numbers each
  uint32_t unit[NQ];  // bf16

  __device__ __forceinline__ void load(const Act8& aux, size_t row, int N, int n0) {
    const int8_t* qr = aux.q + (row * N + n0);
#pragma unroll
    for (int i = 0; i < NQ; ++i)
      if (kWide || n0 + i * STEP < N) q[i] = *(const uint32_t*)(qr + i * STEP);
    const uint16_t* u = aux.unit + row * ((N + 15) >> 4) + (n0 >> 4);
    if constexpr (kWide) {
#pragma unroll
      for (int i = 0; i < NQ; i += 4) {
        const uint2 v = *(const uint2*)(u + i);
        unit[i] = v.x & 0xFFFFu; unit[i + 1] = v.x >> 16; unit[i + 2] = v.y & 0xFFFFu; unit[i + 3] = v.y >> 16;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        if (n0 + i * STEP < N) unit[i] = u[i * (STEP / 16)];
    }
  }
  // kEpiGeluGrad8: H = GeLU(q unit), C = acc GeLU'(q unit)
  template <class Acc>
  __device__ __forceinline__ void grad(uint16_t* C, const Act8& aux, size_t row, int N, int n0, Acc&& acc) const {
    const size_t at = row * N + n0;
    uint16_t *Hr = aux.H + at, *Cr = C + at;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      if (!kWide && n0 + i * STEP >= N) continue;
      const float s = bf16_bits_to_f32(unit[i]);
      const float z0 = (float)(int8_t)q[i] * s, z1 = (float)(int8_t)(q[i] >> 8) * s;
      const float z2 = (float)(int8_t)(q[i] >> 16) * s, z3 = (float)(int8_t)(q[i] >> 24) * s;
      const f32x4 a = acc(i);
      *(uint2*)(Hr + i * STEP) = make_uint2(pack_bf16x2(gelu_by_cdf_bf16(z0), gelu_by_cdf_bf16(z1)),
                                            pack_bf16x2(gelu_by_cdf_bf16(z2), gelu_by_cdf_bf16(z3)));
      *(uint2*)(Cr + i * STEP) = make_uint2(pack_bf16x2(a[0] * gelu_grad_bf16(z0), a[1] * gelu_grad_bf16(z1)),
                                            pack_bf16x2(a[2] * gelu_grad_bf16(z2), a[3] * gelu_grad_bf16(z3)));
    }
  }
  // kEpiGeluSave8: q, unit and C = GeLU(acc)
  template <class Acc>
  __device__ __forceinline__ static void save(uint16_t* C, const Act8& aux, size_t row, int N, int n0, Acc&& acc) {
    const size_t at = row * N + n0;
    int8_t* qr = aux.q + at;
    uint16_t *Cr = C + at, *ur = aux.unit + row * ((N + 15) >> 4);
    const int r = (n0 >> 2) & 3;  // this lane's 16-lane row
#pragma unroll
    for (int g = 0; g < NQ; g += 4) {
      float most[4], inv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        most[k] = 0.f;
        if (g + k < NQ && (kWide || n0 + (g + k) * STEP < N)) {
          const f32x4 a = acc(g + k);
          most[k] = maximum(maximum(fabsf(a[0]), fabsf(a[1])), maximum(fabsf(a[2]), fabsf(a[3])));
        }
      }
      const float m = max_to_rows(most[0], most[1], most[2], most[3]) * (1.0f / 127.0f);
      const uint32_t unit = m < kLeastUnit ? 0u : f32_to_bf16_bits(m);
      // (the reciprocal's last bit matters to ties alone; with a unit of 0 it is 2^126, which leaves values below 127)
      spread_rows(__builtin_amdgcn_rcpf(__uint_as_float(max(unit << 16, 0x00800000u))), inv);
      const int mine = g + quad_of_row(r), block = (n0 - 4 * r + mine * STEP) >> 4;
      if (mine < NQ && (kWide || block < ((N + 15) >> 4))) ur[block] = (uint16_t)unit;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = g + k;
        if (i >= NQ || (!kWide && n0 + i * STEP >= N)) continue;
        const f32x4 a = acc(i);
        // 1.5 x 2^23 + v, rounded to nearest, ends in v's eight bits
        auto byte = [&](float v) { return __float_as_uint(fmaf(v, inv[k], 12582912.0f)); };
        const uint32_t lo = __builtin_amdgcn_perm(byte(a[1]), byte(a[0]), 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(byte(a[3]), byte(a[2]), 0x04000C0Cu);
        *(uint32_t*)(qr + i * STEP) = lo | hi;
        *(uint2*)(Cr + i * STEP) =
            make_uint2(pack_bf16x2(gelu_bf16(a[0]), gelu_bf16(a[1])), pack_bf16x2(gelu_bf16(a[2]), gelu_bf16(a[3])));
      }
    }
  }
};

// A tile's rows of one lane -> memory with an 8-bit epilogue: NJ rows, row(j) counted from row0, of which those below rows_left
// are there; acc(j, i): quad i of row j.  The backward fetches the next row's activations while it computes one.
template <int EPI, int NJ, int NQ, int STEP, class Row, class Acc>
__device__ __forceinline__ void store_rows8(uint16_t* C, const Act8& aux, size_t row0, int rows_left, int N, int n0, Row&& row,
                                           Acc&& acc) {
  using R8 = Row8<NQ, STEP>;
  R8 r[2];
  auto load = [&](int j) {
    if (EPI == kEpiGeluGrad8) r[j & 1].load(aux, row0 + min(row(j), rows_left - 1), N, n0);
  };
  load(0);
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (j + 1 < NJ) load(j + 1);
    if (row(j) < rows_left) {
      if (EPI == kEpiGeluGrad8) r[j & 1].grad(C, aux, row0 + row(j), N, n0, [&](int i) { return acc(j, i); });
      else R8::save(C, aux, row0 + row(j), N, n0, [&](int i) { return acc(j, i); });
    }
  }
}

}  // namespace
}  // namespace locmoe
