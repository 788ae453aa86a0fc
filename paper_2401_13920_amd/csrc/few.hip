// The whole layer for at most LOCMOE_FEW_MAX_TOKENS tokens in two kernels, as decoding calls it:
//   few_in_kernel    gate (or the given gating values), top-1, score and first-come capacity; H = GeLU(W_in[e] . x)
//   few_out_kernel   y = w W_out[e] . H
// Every work-group of the first kernel routes all tokens for itself (a few KiB from L2, cheaper than a launch); one of them
// writes the routing down for the second.  The tokens of one expert are a group: a group's weights are read once.
//
// Bound by the stream of weights: 4 d h bytes per expert with tokens.  Weight rows feed the MFMA's A operand, 16 rows x 32 k a
// KiB straight from memory into registers; a group's tokens are the columns, 16 per MFMA, fetched from L2.  A tile of 16
// weight rows is shared by KS waves of a work-group, each with its part of K, where there are fewer tiles than waves; their
// sums meet in LDS and are added in order.
//
// bf16 storage: H is rounded to bf16, as in the layer's other path.  fp32 storage: the activations and H keep all 24 bits: a
// value is the sum of three bf16 parts, whose exact products with the bf16 weights are summed in fp32.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ffn_epilogue.h"

namespace locmoe {
namespace {

constexpr int kFewTokens = LOCMOE_FEW_MAX_TOKENS;
static_assert(kFewTokens == kWave, "the routing of all tokens is one wave's");
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / kWave;
constexpr int kFewRowsTile = 16;

// The routing as the second kernel reads it (front of the workspace; H follows at kFewHOffset)
struct FewTable {
  int32_t groups;               // experts with kept tokens
  int32_t expert[kFewTokens];   // of each group
  int32_t start[kFewTokens + 1];  // group u's tokens: token[start[u] .. start[u + 1])
  int32_t token[kFewTokens];
};
constexpr size_t kFewHOffset = 1024;
static_assert(sizeof(FewTable) <= kFewHOffset, "");

// fp32 -> three bf16 parts whose sum is the value (cut, so that every remainder is exact).  An infinity or a NaN is the first
// part alone.
__device__ __forceinline__ void split3(float v, uint32_t (&p)[3]) {
  uint32_t b = __float_as_uint(v);
  p[0] = b >> 16;
  const bool fin = fabsf(v) < INFINITY;
  if ((b & 0x7F800000u) == 0x7F800000u) p[0] |= (b & 0xFFFFu) ? 1u : 0u;  // (a NaN stays one)
  float r = fin ? v - __uint_as_float(b & 0xFFFF0000u) : 0.f;
  b = __float_as_uint(r);
  p[1] = b >> 16;
  r -= __uint_as_float(b & 0xFFFF0000u);
  p[2] = __float_as_uint(r) >> 16;
}

// GeLU of a value that is kept in fp32
__device__ __forceinline__ float gelu_f32(float z) { return z * (0.5f * erfcf(-0.70710678118654752f * z)); }

// Gating value of token m for expert e by L lanes (this one the l-th): its share of the block's sum
template <bool BF16>
__device__ __forceinline__ float gate_part(const void* x, int m, int e, int d, int blk, int l, int L) {
  constexpr int V = BF16 ? 8 : 4;
  float s = 0.f;
  const size_t at = (size_t)m * d + (size_t)e * blk;
  if (blk % V == 0) {  // (rows are whole chunks too)
    const uint4* p = (const uint4*)x + at / V;
    for (int c = l; c < blk / V; c += L) s += BF16 ? sum8_bf16(p[c]) : sum4_f32(p[c]);
  } else {
    for (int c = l; c < blk; c += L) s += BF16 ? bf16_bits_to_f32(((const uint16_t*)x)[at + c]) : ((const float*)x)[at + c];
  }
  return s;
}

// Top-1 of token m by one wave: eid and score to LDS.  Experts are lane e (L lanes each while E < 64), e + 64, ...
template <bool BF16>
__device__ __forceinline__ void few_route(const void* x, const float* g, const float* eps, int m, int d, int E, int relu,
                                          int32_t* s_eid, float* s_w) {
  const int lane = threadIdx.x & 63, blk = d / E;
  int L = 1;
  while (2 * L * E <= kWave) L *= 2;
  float best = -INFINITY;
  int at = 0x7FFFFFFF;
  const float inv = 1.0f / (float)blk;
  float val[16];  // E <= 1024
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int e = lane / L + k * kWave;
    val[k] = -INFINITY;
    if (k * kWave >= E) continue;
    float v = 0.f;
    if (e < E) v = g ? g[(size_t)m * E + e] : gate_part<BF16>(x, m, e, d, blk, lane % L, L);
    if (!g) {
      for (int o = 1; o < L; o *= 2) v += __shfl_xor(v, o);
      v *= inv;
    }
    if (e < E) {
      if (eps) v += eps[e];
      if (relu) v = fmaxf(v, 0.f);
      val[k] = v;
      if (v > best || at == 0x7FFFFFFF) { best = v; at = e; }  // (ascending e: ties stay with the lower)
    }
  }
  for (int o = 32; o > 0; o >>= 1) {
    const float ov = __shfl_xor(best, o);
    const int oa = __shfl_xor(at, o);
    if (oa != 0x7FFFFFFF && (at == 0x7FFFFFFF || ov > best || (ov == best && oa < at))) { best = ov; at = oa; }
  }
  float z = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k)
    if (k * kWave < E && lane / L + k * kWave < E && lane % L == 0) z += expf(val[k] - best);
  z = group_sum<kWave>(z);
  if (lane == 0) { s_eid[m] = at; s_w[m] = 1.0f / z; }
}

// The groups, by one wave (lane m: token m): first-come capacity, groups in the order of their first tokens
__device__ __forceinline__ void few_groups(const int32_t* s_eid, int T, int C, FewTable* t, int32_t* s_slot) {
  const int m = threadIdx.x;
  const int e = m < T ? s_eid[m] : -1;
  int pos = 0, all = 0;
  for (int q = 0; q < T; ++q) {
    const bool same = s_eid[q] == e;
    pos += same && q < m;
    all += same;
  }
  const bool live = m < T, first = live && pos == 0;
  const uint64_t leaders = __ballot(first);
  const int n = first ? min(all, C) : 0;  // kept tokens of the group that this lane leads
  int sum = n;                            // inclusive over the leaders up to this lane
  for (int o = 1; o < kWave; o <<= 1) {
    const int up = __shfl_up(sum, o);
    if (m >= o) sum += up;
  }
  int lead = 0;  // the lane that leads this token's group
  for (int q = T - 1; q >= 0; --q)
    if (s_eid[q] == e) lead = q;
  const int start = __shfl(sum - n, lead);
  if (first) {
    const int u = __builtin_popcountll(leaders & ((1ull << m) - 1ull));
    t->expert[u] = e;
    t->start[u] = sum - n;
  }
  const bool kept = live && pos < C;
  if (kept) t->token[start + pos] = m;
  if (live) s_slot[m] = kept ? m : -1;
  if (m == kWave - 1) {
    t->groups = __builtin_popcountll(leaders);
    t->start[__builtin_popcountll(leaders)] = sum;
  }
}

// A group's share of a GEMM: the KS-th part of K of one 16-row tile of weights by one wave, NB column tiles of 16 tokens.
// W: the expert's weights.  Operand B is the tokens' rows: bf16 (X_F32 false, NP planes `plane` elements apart) or fp32.
template <bool PACKED, bool X_F32, int NP, int NB>
__device__ __forceinline__ void few_dot(f32x4 (&acc)[NB], const char* __restrict__ W, const void* __restrict__ X,
                                        size_t plane, const int32_t* tok, int n, int tile, int Kdim, int Ndim, int s0,
                                        int s1) {
  constexpr int D = NB * NP <= 2 ? 8 : NB * NP <= 4 ? 4 : 2;  // k-steps whose weights are in flight
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  const int row = min(tile * kFewRowsTile + l16, Ndim - 1);
  const char* pw;
  size_t wstep;
  if (PACKED) {
    pw = W + (size_t)(row >> 8) * Kdim * 512 + (row & 255) * 64 + ((q ^ ((row >> 1) & 3)) << 4);
    wstep = 16384;
  } else {
    pw = W + (size_t)row * Kdim * 2 + q * 16;
    wstep = 64;
  }
  const char* px[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)  // columns past the group's tokens repeat the last one (not stored)
    px[b] = (const char*)X + ((size_t)tok[min(16 * b + l16, n - 1)] * Kdim + q * 8) * (X_F32 ? 4 : 2);
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  // steps s .. s + D - 1; TAIL: the one step that ends behind K, where both operands are zeros past it
  auto steps = [&](auto depth, auto tail, int s) {
    constexpr int D = decltype(depth)::value;
    constexpr bool TAIL = decltype(tail)::value;
    u32x4 w[D], x[D][NB][X_F32 ? 2 : NP];
    const u32x4 zero = {0u, 0u, 0u, 0u};
    const bool in = !TAIL || s * 32 + q * 8 < Kdim;
#pragma unroll
    for (int u = 0; u < D; ++u) {
      w[u] = in ? *(const u32x4*)(pw + (size_t)(s + u) * wstep) : zero;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int p = 0; p < (X_F32 ? 2 : NP); ++p) {
          const char* a = px[b] + (X_F32 ? (size_t)(s + u) * 128 + p * 16 : (size_t)(s + u) * 64 + p * plane * 2);
          x[u][b][p] = in ? *(const u32x4*)a : zero;
        }
    }
#pragma unroll
    for (int u = 0; u < D; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        u32x4 part[NP];
        if constexpr (X_F32) {
          uint32_t v[8][3];
#pragma unroll
          for (int i = 0; i < 8; ++i) split3(__uint_as_float(x[u][b][i / 4][i % 4]), v[i]);
#pragma unroll
          for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[p][i] = v[2 * i][p] | (v[2 * i + 1][p] << 16);
        } else {
#pragma unroll
          for (int p = 0; p < NP; ++p) part[p] = x[u][b][p];
        }
#pragma unroll
        for (int p = 0; p < NP; ++p)
          acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[u]),
                                                           __builtin_bit_cast(bf16x8, part[p]), acc[b], 0, 0, 0);
      }
  };
  using No = std::false_type;
  const int full = min(s1, Kdim / 32);
  int s = s0;
  for (; s + D <= full; s += D) steps(std::integral_constant<int, D>{}, No{}, s);
  if constexpr (D > 4) { if (s + 4 <= full) { steps(std::integral_constant<int, 4>{}, No{}, s); s += 4; } }
  if constexpr (D > 2) { if (s + 2 <= full) { steps(std::integral_constant<int, 2>{}, No{}, s); s += 2; } }
  if constexpr (D > 1) { if (s < full) { steps(std::integral_constant<int, 1>{}, No{}, s); ++s; } }
  if (s < s1) steps(std::integral_constant<int, 1>{}, std::true_type{}, s);
}

// All tiles of all groups, over the grid's waves: epilogue(u, tile, token's place in the group, row of weights, 4 sums).
// MAXB: column tiles at most (of all tokens).
template <bool PACKED, bool X_F32, int NP, int MAXB, class F>
__device__ __forceinline__ void few_gemm(const FewTable* t, const char* W, const void* X, size_t plane, int Kdim, int Ndim,
                                         float4* red, F&& epilogue) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int tiles = (Ndim + kFewRowsTile - 1) / kFewRowsTile, steps = (Kdim + 31) / 32;
  const long long items = (long long)t->groups * tiles;
  int ks = 1;  // waves per tile
  while (ks < kFewWaves && items * ks < (long long)gridDim.x * kFewWaves && steps >= 4 * ks) ks *= 2;
  const int per = kFewWaves / ks, sub = wave % ks, mine = wave / ks;
  const int s0 = (int)((long long)steps * sub / ks), s1 = (int)((long long)steps * (sub + 1) / ks);
  for (long long i0 = (long long)blockIdx.x * per; i0 < items; i0 += (long long)gridDim.x * per) {
    const long long item = i0 + mine;
    const bool have = item < items;
    const int u = have ? (int)(item / tiles) : 0, tile = have ? (int)(item % tiles) : 0;
    const int32_t* tok = t->token + t->start[u];
    const int n = t->start[u + 1] - t->start[u];
    const char* We = W + (size_t)t->expert[u] * Ndim * Kdim * 2;
    f32x4 acc[MAXB];
#define LOCMOE_FEW_DOT(NB)                                                                                     \
  {                                                                                                            \
    f32x4 a[NB];                                                                                               \
    few_dot<PACKED, X_F32, NP, NB>(a, We, X, plane, tok, n, tile, Kdim, Ndim, s0, s1);                         \
    _Pragma("unroll") for (int b = 0; b < NB; ++b) acc[b] = a[b];                                              \
  }
    if (have) {
      if (MAXB == 1 || n <= 16) LOCMOE_FEW_DOT(1)
      else if constexpr (MAXB > 1) {
        if (n <= 32) LOCMOE_FEW_DOT(2)
        else LOCMOE_FEW_DOT(4)
      }
    }
#undef LOCMOE_FEW_DOT
    const int nb = (n + 15) / 16;
    if (ks > 1) {
      __syncthreads();
      if (have && sub) {
#pragma unroll
        for (int b = 0; b < MAXB; ++b)
          if (b < nb) red[(wave * MAXB + b) * 64 + lane] = make_float4(acc[b][0], acc[b][1], acc[b][2], acc[b][3]);
      }
      __syncthreads();
      if (have && !sub) {
        for (int j = 1; j < ks; ++j)
#pragma unroll
          for (int b = 0; b < MAXB; ++b)
            if (b < nb) {
              const float4 v = red[((wave + j) * MAXB + b) * 64 + lane];
              acc[b][0] += v.x; acc[b][1] += v.y; acc[b][2] += v.z; acc[b][3] += v.w;
            }
      }
    }
    if (have && !sub) {
#pragma unroll
      for (int b = 0; b < MAXB; ++b) {
        const int c = 16 * b + (lane & 15), r = tile * kFewRowsTile + (lane >> 4) * 4;
        if (c < n && r < Ndim) epilogue(tok[c], r, acc[b]);  // (Ndim is a multiple of 8: the quad is inside or outside)
      }
    }
  }
}

// waves per SIMD: two work-groups per compute unit, or one where the tokens' operands take the registers
constexpr int few_occupancy(int maxb) { return maxb == 1 ? 4 : 2; }

template <bool BF16, bool PACKED, int MAXB>
__global__ __launch_bounds__(kFewThreads, few_occupancy(MAXB)) void few_in_kernel(const void* __restrict__ x, const float* __restrict__ g,
                                                                const float* __restrict__ eps,
                                                                const char* __restrict__ W, int32_t* __restrict__ eid,
                                                                float* __restrict__ w, int32_t* __restrict__ slot,
                                                                FewTable* __restrict__ table, uint16_t* __restrict__ H,
                                                                int T, int d, int E, int h, int C, int relu) {
  __shared__ int32_t s_eid[kFewTokens], s_slot[kFewTokens];
  __shared__ float s_w[kFewTokens];
  __shared__ FewTable t;
  __shared__ float4 red[kFewWaves * MAXB * 64];
  const int wave = threadIdx.x >> 6;
  for (int m = wave; m < T; m += kFewWaves) few_route<BF16>(x, g, eps, m, d, E, relu, s_eid, s_w);
  __syncthreads();
  if (wave == 0) few_groups(s_eid, T, C, &t, s_slot);
  __syncthreads();
  if (blockIdx.x == 0) {
    if (threadIdx.x < T) {
      eid[threadIdx.x] = s_eid[threadIdx.x];
      w[threadIdx.x] = s_w[threadIdx.x];
      slot[threadIdx.x] = s_slot[threadIdx.x];
    }
    for (int i = threadIdx.x; i < (int)(sizeof(FewTable) / 4); i += kFewThreads) ((int32_t*)table)[i] = ((int32_t*)&t)[i];
  }
  constexpr int NP = BF16 ? 1 : 3;
  const size_t plane = (size_t)T * h;
  few_gemm<PACKED, !BF16, NP, MAXB>(&t, W, x, 0, d, h, red, [&](int m, int r, const f32x4& a) {
    uint16_t* dst = H + (size_t)m * h + r;
    if constexpr (BF16) {
      *(uint2*)dst = make_uint2(pack_bf16x2(gelu_bf16(a[0]), gelu_bf16(a[1])), pack_bf16x2(gelu_bf16(a[2]), gelu_bf16(a[3])));
    } else {
      uint32_t v[4][3];
#pragma unroll
      for (int i = 0; i < 4; ++i) split3(gelu_f32(a[i]), v[i]);
#pragma unroll
      for (int p = 0; p < 3; ++p)
        *(uint2*)(dst + p * plane) = make_uint2(v[0][p] | (v[1][p] << 16), v[2][p] | (v[3][p] << 16));
    }
  });
}

template <bool BF16, bool PACKED, int MAXB>
__global__ __launch_bounds__(kFewThreads, few_occupancy(MAXB)) void few_out_kernel(const uint16_t* __restrict__ H,
                                                                 const FewTable* __restrict__ table,
                                                                 const int32_t* __restrict__ slot,
                                                                 const float* __restrict__ w,
                                                                 const char* __restrict__ W, void* __restrict__ y, int T,
                                                                 int d, int h, int weighted) {
  __shared__ FewTable t;
  __shared__ float4 red[kFewWaves * MAXB * 64];
  for (int i = threadIdx.x; i < (int)(sizeof(FewTable) / 4); i += kFewThreads) ((int32_t*)&t)[i] = ((const int32_t*)table)[i];
  __syncthreads();
  if (weighted) {  // dropped tokens
    const int chunks = d / (BF16 ? 8 : 4);
    for (int m = blockIdx.x; m < T; m += gridDim.x)
      if (slot[m] < 0)
        for (int c = threadIdx.x; c < chunks; c += kFewThreads) ((uint4*)y)[(size_t)m * chunks + c] = make_uint4(0, 0, 0, 0);
  }
  few_gemm<PACKED, false, BF16 ? 1 : 3, MAXB>(&t, W, H, (size_t)T * h, h, d, red, [&](int m, int r, const f32x4& a) {
    const float f = weighted ? w[m] : 1.0f;
    if constexpr (BF16)
      *(uint2*)((uint16_t*)y + (size_t)m * d + r) = make_uint2(pack_bf16x2(f * a[0], f * a[1]), pack_bf16x2(f * a[2], f * a[3]));
    else
      *(float4*)((float*)y + (size_t)m * d + r) = make_float4(f * a[0], f * a[1], f * a[2], f * a[3]);
  });
}

}  // namespace
}  // namespace locmoe

extern "C" size_t locmoe_layer_few_workspace_bytes(const locmoe_desc* desc) {
  using namespace locmoe;
  if (check_desc(desc) != LOCMOE_OK || desc->T > kFewTokens) return 0;
  const size_t planes = desc->x_dtype == LOCMOE_BF16 ? 1 : 3;
  return (kFewHOffset + planes * (size_t)desc->T * (size_t)desc->h * 2 + 255) & ~(size_t)255;
}

extern "C" int locmoe_layer_few(const locmoe_desc* desc, const void* x, const float* g, const float* eps, const void* W_in,
                                const void* W_out, int32_t weighted, int32_t* eid, float* w, int32_t* slot, void* y,
                                void* ws, size_t ws_bytes, void* stream) {
  using namespace locmoe;
  if (!desc || !x || !W_in || !W_out || !eid || !w || !slot || !y) return LOCMOE_ERR_NULL;
  const int st = check_desc(desc);
  if (st != LOCMOE_OK) return st;
  if (desc->T > kFewTokens) return LOCMOE_ERR_SHAPE;
  if (weighted != 0 && weighted != 1) return LOCMOE_ERR_ARG;
  const bool bf = desc->x_dtype == LOCMOE_BF16;
  if (desc->w_packed && (!bf || locmoe_packed_weights_bytes(desc) == 0)) return LOCMOE_ERR_ARG;
  if (!ws || ws_bytes < locmoe_layer_few_workspace_bytes(desc)) return LOCMOE_ERR_WORKSPACE;
  const int T = desc->T, d = desc->d, E = desc->E, h = desc->h;
  hipStream_t s = as_stream(stream);
  FewTable* table = (FewTable*)ws;
  uint16_t* H = (uint16_t*)((char*)ws + kFewHOffset);
  // two work-groups per compute unit, no more than there can be tiles (of up to eight waves each)
  auto grid = [&](int n) {
    return dim3((unsigned)std::min<long long>(2 * cu_count(), (long long)std::min(T, E) * ceil_div(n, kFewRowsTile)));
  };
  auto launch = [&](auto bf16, auto packed, auto maxb) {
    constexpr bool BF = decltype(bf16)::value, PK = decltype(packed)::value;
    constexpr int MAXB = decltype(maxb)::value;
    hipLaunchKernelGGL((few_in_kernel<BF, PK, MAXB>), grid(h), dim3(kFewThreads), 0, s, x, g, eps, (const char*)W_in, eid, w,
                       slot, table, H, T, d, E, h, desc->C, desc->relu);
    hipLaunchKernelGGL((few_out_kernel<BF, PK, MAXB>), grid(d), dim3(kFewThreads), 0, s, H, table, slot, w,
                       (const char*)W_out, y, T, d, h, weighted);
  };
  auto with_tokens = [&](auto bf16, auto packed) {
    if (T <= 16) launch(bf16, packed, std::integral_constant<int, 1>{});
    else launch(bf16, packed, std::integral_constant<int, 4>{});
  };
  if (!bf) with_tokens(std::false_type{}, std::false_type{});
  else if (desc->w_packed) with_tokens(std::true_type{}, std::true_type{});
  else with_tokens(std::true_type{}, std::false_type{});
  return launch_status();
}
