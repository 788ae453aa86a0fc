// The whole layer for at most LOCMOE_FEW_MAX_TOKENS tokens in two kernels, as decoding calls it:
//   few_in_kernel    gate (or the given gating values), top-1, score and first-come capacity; H = GeLU(W_in[e] . x)
//   few_out_kernel   y = w W_out[e] . H
// Every work-group of the first kernel routes all tokens for itself (a few KiB from L2, cheaper than a launch); one of them
// writes the routing down for the second.  The tokens of one expert are a group: a group's weights are read once.
//
// Bound by the stream of weights: 4 d h bytes per expert with tokens.  Weight rows feed the MFMA's A operand, 16 rows x 32 k a
// KiB straight from memory into registers; a group's tokens are the columns, 16 per MFMA, fetched from L2.  A tile of 16
// weight rows is shared by up to eight waves of a work-group, each with its part of K, where there are fewer tiles than waves;
// their sums meet in LDS and are added in order.  Measured (both kernels, one call after another): 64 tokens on 16 to 27 of 64
// experts in turn, gating values given, d = 4096, h = 16384, 4.3 to 7.2 GB of weights: 6.5 to 6.6 TB/s packed, 5.7 to 6.5 row-major (a
// copy-free read of as much: 6.3 to 7.0); one token, d = 1024, h = 4096, 16.8 MB: 11.5 us, of which the launches, the routing
// and a round trip to memory each are most.  Far from the stream's rate: many tokens on one expert, and fp32 storage, where the
// tokens' operands, which every tile fetches again from L2, are several times the weights (64 tokens on one expert,
// d = 2048, h = 8192, 67 MB: 67 us).
//
// bf16 storage: H is rounded to bf16, as in the layer's other path.  fp32 storage: the activations and H keep all 24 bits: a
// value is the sum of three bf16 parts, whose exact products with the bf16 weights are summed in fp32.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ffn_epilogue.h"
#include "gelu_coef_f32.h"

namespace locmoe {
namespace {

constexpr int kFewTokens = LOCMOE_FEW_MAX_TOKENS;
static_assert(kFewTokens == kWave, "the routing of all tokens is one wave's");
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / kWave;
constexpr int kFewRowsTile = 16;
// Weights of more than this in one launch, which the last-level cache does not hold until the next call anyway, are loaded past
// it: packed, d = 4096, h = 16384, 20 experts 1 003 -> 917 us; below, a loop over one layer finds them there (d = 1024, h = 4096,
// one expert 12.9 -> 14.6).  Row-major ones if their rows are whole lines of memory.
constexpr long long kFewStreamBytes = 100ll << 20;

// The routing as the second kernel reads it (front of the workspace; H follows at kFewHOffset)
struct FewTable {
  int32_t groups;               // experts with kept tokens
  int32_t expert[kFewTokens];   // of each group
  int32_t start[kFewTokens + 1];  // group u's tokens: token[start[u] .. start[u + 1])
  int32_t token[kFewTokens];
};
constexpr size_t kFewHOffset = 1024;
// Values from row to row of H: where rows would be whole lines, half a line more, so that the 64 bytes that a load takes of each of 16
// rows are not all first or all second halves (64 tokens on one expert, d = 2048, h = 8192: 73 -> 67 us; a whole line more: nothing)
__host__ __device__ constexpr int few_h_row(int h) { return h % 64 == 0 ? h + 32 : h; }
static_assert(sizeof(FewTable) <= kFewHOffset, "");

// Two fp32 values -> three bf16 parts of each (bits 0..7, 8..15 and 16..23 of the significand: cut, so that every remainder is
// exact), the first value's in the low halves.  An infinity leaves NaN for its second part.
__device__ __forceinline__ void split3(float a, float b, uint32_t (&p)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    p[k] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);  // the upper halves
    a -= __uint_as_float(ua & 0xFFFF0000u);
    b -= __uint_as_float(ub & 0xFFFF0000u);
  }
}

// GeLU of a value that is kept in fp32: as gelu_bf16, with a polynomial whose error is below 8e-8 |v|
__device__ __forceinline__ float gelu_f32(float v) {
  const float x = __builtin_amdgcn_fmed3f(fabsf(v), 0.f, kGeluXMax);
  float q = kGeluCoefF32[kGeluDegreeF32];
#pragma unroll
  for (int k = kGeluDegreeF32 - 1; k >= 0; --k) q = fmaf(q, x, kGeluCoefF32[k]);
  return 0.5f * fmaf(-x, __builtin_amdgcn_exp2f(q), v + fabsf(v));
}

// Eight loads in flight of a lane's share of the sum over the blk features from x[at] on: every L-th 16-byte chunk (or feature,
// where chunks do not fit) from the l-th on; L = 2^lL
template <bool BF16>
__device__ __forceinline__ float gate_part(const void* x, size_t at, int blk, int l, int lL) {
  constexpr int V = BF16 ? 8 : 4, U = 8;
  float s = 0.f;
  if (blk % V == 0) {  // (rows are whole chunks too)
    const uint4* p = (const uint4*)x + at / V;
    const int n = blk / V;
    for (int c = l; c < n; c += U << lL) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = p[min(c + (u << lL), n - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u) s += c + (u << lL) < n ? (BF16 ? sum8_bf16(v[u]) : sum4_f32(v[u])) : 0.f;
    }
  } else {
    for (int c = l; c < blk; c += 1 << lL) s += BF16 ? bf16_bits_to_f32(((const uint16_t*)x)[at + c]) : ((const float*)x)[at + c];
  }
  return s;
}

// How a work-group routes all tokens: S lanes share a token, as many as let every token have its own, so that all of them wait for
// their loads together; P experts side by side (the next ones in further turns), S / P lanes each.  Powers of two.
struct FewRoute {
  int lS, lP, blk;
  float inv_blk;
};
FewRoute few_route_plan(int T, int d, int E) {
  FewRoute r = {6, 0, d / E, 1.0f / (float)(d / E)};
  while ((T << r.lS) > kFewThreads) --r.lS;
  while (r.lP < r.lS && (1 << r.lP) < E) ++r.lP;
  return r;
}

// Top-1 of all tokens by the work-group: eid and score to LDS.  The largest value and the sum of exponentials up to it are kept
// as the experts go by.  Short rather than unrolled: a launch of this size spends much of its time fetching and issuing its own
// instructions (16 tokens, d = 128, E = 8, fp32, this kernel: 13.6 us with the experts' turns unrolled and a long GeLU, 7.3 so).
template <bool BF16>
__device__ __forceinline__ void few_route(const FewRoute& r, const void* x, const float* g, const float* eps, int T, int d, int E,
                                          int relu, int32_t* s_eid, float* s_w) {
  const int S = 1 << r.lS, P = 1 << r.lP, lL = r.lS - r.lP, L = 1 << lL, l = threadIdx.x & (S - 1);
  constexpr float kLog2e = 1.44269504f;
  {  // (S T <= kFewThreads: every token has its lanes; the lanes left over repeat the last one)
    const int m0 = threadIdx.x >> r.lS, m = min(m0, T - 1);
    float best = -INFINITY, z = 0.f;
    int at = E;
    auto seen = [&](int e, float v) {
      if (eps) v += eps[e];
      if (relu) v = fmaxf(v, 0.f);
      const float f = v == best ? 1.0f : __builtin_amdgcn_exp2f(-kLog2e * fabsf(v - best));  // (both may be -inf: a masked expert)
      const bool more = v > best;  // (ascending e: ties stay with the lower; a NaN is never the largest, but stays in z)
      z = more ? fmaf(z, f, 1.0f) : z + f;
      best = more ? v : best;
      at = more ? e : at;
    };
    if (g) {
#pragma unroll 4
      for (int e = l >> lL; e < E; e += P) seen(e, g[(size_t)m * E + e]);
    } else {
      for (int e = l >> lL; e < E; e += P)
        seen(e, lanes_sum(gate_part<BF16>(x, (size_t)m * d + (size_t)e * r.blk, r.blk, l & (L - 1), lL), L) * r.inv_blk);
    }
    float top = best;
    int who = at;
    for (int o = S / 2; o > 0; o >>= 1) {
      const float ov = __shfl_xor(top, o);
      const int oa = __shfl_xor(who, o);
      const bool take = who == E || (oa < E && (ov > top || (ov == top && oa < who)));
      top = take ? ov : top;
      who = take ? oa : who;
    }
    // (lanes without an expert have z = 0; nothing above -inf at all: expert 0 and NaN, as locmoe_route)
    const float sum = lanes_sum((l & (L - 1)) == 0 ? z * __builtin_amdgcn_exp2f(kLog2e * (best - top)) : 0.f, S);
    if (l == 0 && m0 < T) { s_eid[m] = who < E ? who : 0; s_w[m] = 1.0f / sum; }
  }
}

// The groups, by one wave (lane m: token m): first-come capacity, groups in the order of their first tokens
__device__ __forceinline__ void few_groups(const int32_t* s_eid, int T, int C, FewTable* t, int32_t* s_slot) {
  const int m = threadIdx.x;
  if (T == 1) {  // (a single sequence's decoding)
    if (m == 0) { t->groups = 1; t->expert[0] = s_eid[0]; t->start[0] = 0; t->start[1] = 1; t->token[0] = 0; s_slot[0] = 0; }
    return;
  }
  const bool live = m < T;
  const int e = live ? s_eid[m] : 0;
  uint64_t same = __ballot(live);  // the tokens of the same expert: a vote on every bit of its number (E <= 1024)
#pragma unroll
  for (int b = 0; b < 10; ++b) {
    const uint64_t ones = __ballot((e >> b) & 1);
    same &= (e >> b) & 1 ? ones : ~ones;
  }
  const uint64_t below = (1ull << m) - 1ull;
  const int pos = __builtin_popcountll(same & below), all = __builtin_popcountll(same);
  const int lead = live ? __builtin_ctzll(same) : 0;  // the lane that leads this token's group
  const bool first = live && pos == 0;
  const uint64_t leaders = __ballot(first);
  const int n = first ? min(all, C) : 0;  // kept tokens of the group that this lane leads
  int sum = n;                            // inclusive over the leaders up to this lane
  for (int o = 1; o < kWave; o <<= 1) {
    const int up = __shfl_up(sum, o);
    if (m >= o) sum += up;
  }
  const int start = __shfl(sum - n, lead), u = __builtin_popcountll(leaders & below);
  if (first) {
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

// k-steps of weights in flight, and products whose tokens' operands (XL 16-byte loads each) are, of the NB column tiles of these
// steps: what 128 registers hold beside the sums.  16 waves of a compute unit have 128 KiB of weights in flight with 8 steps, which
// is enough: d = 4096, h = 16384, 24 experts took 902 us with the tokens' operands of all steps in flight too, 929 with these in LDS
// and 16 steps of weights (8 steps: 897), 906 with loads kept in flight across the products, 931 with pairs of tiles that share
// the operands.  For more than one column tile the operands come in behind the products they are for: 64 tokens on 4 experts,
// d = 2048, h = 8192, packed, 104 us with 2 steps of weights and all their operands in flight, 96 so.
constexpr int few_depth(int XL) { return XL == 1 ? 8 : 4; }
constexpr int few_ahead(int XL, int NB) { return NB == 1 ? few_depth(XL) : (NB == 2 ? 2 : 1) * (5 - XL); }

// A k-step's products of a column tile: weights w, tokens' operand x as loaded
template <bool X_F32, int NP>
__device__ __forceinline__ void few_mul(f32x4& acc, const u32x4& w, const u32x4 (&x)[X_F32 ? 2 : NP]) {
  u32x4 part[NP];
  if constexpr (X_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v[3];
      split3(__uint_as_float(x[i / 2][2 * i % 4]), __uint_as_float(x[i / 2][2 * i % 4 + 1]), v);
#pragma unroll
      for (int p = 0; p < NP; ++p) part[p][i] = v[p];
    }
  } else {
#pragma unroll
    for (int p = 0; p < NP; ++p) part[p] = x[p];
  }
#pragma unroll
  for (int p = 0; p < NP; ++p)
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, part[p]), acc, 0, 0, 0);
}

// A wave's share of a GEMM: steps s0 .. s1 - 1 of K for one 16-row tile of weights and NB column tiles of 16 tokens.  W: the
// expert's weights.  Operand B is the tokens' rows, x_row values apart: bf16 (NP planes `plane` elements apart) or, with X_F32, fp32.
// STREAM: the weights are loaded past the caches.
//
// SEG = 2, 4: a tile is 16 / SEG rows, each SEG times side by side in the MFMA's rows with a SEG-th of K each, and so are up to
// 16 / SEG tokens in its columns: SEG blocks on the diagonal of the result, which the caller adds, for a tile whose products
// the rows of SEG times as many work-groups share.
//
// Row-major weights past the caches go by whole lines, two steps (64 k) at a time, which s0, s1 then count: a load takes the line of 8
// rows (half lines are fetched twice), the first 8 lanes of a 16-lane row its first half and the others its second, and two
// loads (rows 0 to 7 and 8 to 15) make two steps' operands by exchanging halves.  d = 4096, h = 16384, 20 experts: 1 049 us with
// half lines through the caches, 929 so, 923 with the tiles out of step (one expert: 69, 66 and 51).
template <bool PACKED, bool X_F32, int NP, int NB, int SEG, bool STREAM>
__device__ __forceinline__ void few_dot(f32x4 (&acc)[NB], const char* __restrict__ W, const void* __restrict__ X,
                                        size_t plane, int x_row, const int32_t* tok, int n, int tile, int Kdim, int Ndim, int s0,
                                        int s1) {
  constexpr bool LINES = STREAM && !PACKED;
  constexpr int XL = X_F32 ? 2 : NP;  // 16-byte loads of a column tile and step
  constexpr int H = LINES ? 2 : 1, D = few_depth(XL) / H, A = few_ahead(XL, NB), ALL = D * H * NB;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  constexpr int kStep = PACKED ? 16384 : 64 * H, kXStep = X_F32 ? 128 : 64;
  constexpr int R = kFewRowsTile / SEG;
  // (rows past the last repeat it: not stored)
  const int row = min(tile * R + (LINES ? l16 & 7 : l16 % R), Ndim - 1), row1 = min(tile * R + 8 + (l16 & 7), Ndim - 1);
  const int seg = l16 / R, k_seg = Kdim / SEG, chunk = LINES ? q + 4 * (l16 >> 3) : q;
  const char* pw = PACKED ? W + (size_t)(row >> 8) * Kdim * 512 + (row & 255) * 64 + ((q ^ ((row >> 1) & 3)) << 4)
                          : W + (size_t)row * Kdim * 2 + chunk * 16;
  const char* pw1 = W + (size_t)row1 * Kdim * 2 + chunk * 16;  // (LINES)
  pw += (size_t)(seg * (k_seg / 32)) * kStep;
  const char* px[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)  // columns past the group's tokens repeat the last one (not stored)
    px[b] = (const char*)X + ((size_t)tok[min(16 * b + l16 % R, n - 1)] * x_row + seg * k_seg + q * 8) * (X_F32 ? 4 : 2);
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 w[D][H], x[A][XL];
  auto load_w = [&](int u, int s) {
    const u32x4* p = (const u32x4*)(pw + (size_t)s * kStep);
    w[u][0] = STREAM ? __builtin_nontemporal_load(p) : *p;
    if constexpr (LINES) w[u][1] = __builtin_nontemporal_load((const u32x4*)(pw1 + (size_t)s * kStep));
  };
  auto load_x = [&](int at, int s, int b) {
#pragma unroll
    for (int p = 0; p < XL; ++p) x[at][p] = *(const u32x4*)(px[b] + (size_t)s * kXStep + (X_F32 ? p * 16 : p * plane * 2));
  };
  // D steps (or lines) from s on, or fewer: all weights' loads and the first A products' tokens, then the products, the tokens of
  // later ones behind them.  (Tokens behind their step's weights: d = 1600, h = 6400, five experts 46.0 us, behind all weights 47.5.)
  auto turn = [&](int s, auto whole, int count) {
    constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
    for (int u = 0; u < D; ++u)
      if (WHOLE || u < count) {
        load_w(u, s + u);
#pragma unroll
        for (int i = u * H * NB; i < (u + 1) * H * NB && i < A; ++i) load_x(i, s * H + i / NB, i % NB);
      }
#pragma unroll
    for (int i = 0; i < ALL; ++i) {
      const int u = i / (H * NB);
      if (WHOLE || u < count) {
        if constexpr (LINES) {
          if (i % (H * NB) == 0) {  // lanes 8 to 15 of a row take the other lanes' second load, lanes 0 to 7 their first
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t lo = w[u][0][k], hi = w[u][1][k];
              w[u][0][k] = __builtin_amdgcn_update_dpp(lo, hi, kDppRor8, 0xF, 0xC, false);
              w[u][1][k] = __builtin_amdgcn_update_dpp(hi, lo, kDppRor8, 0xF, 0x3, false);
            }
          }
        }
        few_mul<X_F32, NP>(acc[i % NB], w[u][i / NB % H], x[i % A]);
      }
      const int next = i + A;
      if (next < ALL && (WHOLE || next / (H * NB) < count)) load_x(i % A, s * H + next / NB, next % NB);
    }
  };
  // Whole turns in a cycle that begins at a place of its own in neighbouring blocks of packed rows (tiles of row-major lines): in
  // step, all waves read at multiples of a power of two, which are few of the memory's channels (packed, d = 4096, h = 16384, 20
  // experts: 952 -> 890 us).  With fewer turns than places all start together: there, with 17, 18, 21, 22, 25 or 26 experts, where
  // two or eight waves share a tile and have eight turns each (6.5 to 6.6 TB/s, as the others).
  const int full = LINES ? s1 : min(s1, k_seg / 32), turns = max(full - s0, 0) / D;
  int at = s0 + (PACKED ? ((tile >> 4) & 15) * (turns >> 4) : LINES ? (tile & 7) * (turns >> 3) : 0) * D;
  for (int i = 0; i < turns; ++i) {
    turn(at, std::true_type{}, D);
    at += D;
    if (at == s0 + turns * D) at = s0;
  }
  int s = s0 + turns * D;
  if (s < full) turn(s, std::false_type{}, full - s);
  if constexpr (!LINES) {
    s = max(s, full);
    if (s < s1) {  // the step that ends behind K, where both operands are zeros past it
      const bool in = s * 32 + q * 8 < k_seg;
      w[0][0] = u32x4{0u, 0u, 0u, 0u};
      if (in) load_w(0, s);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int p = 0; p < XL; ++p) x[0][p] = u32x4{0u, 0u, 0u, 0u};
        if (in) load_x(0, s, b);
        few_mul<X_F32, NP>(acc[b], w[0][0], x[0]);
      }
    }
  }
}

// All tiles of all groups, over the grid's waves: epilogue(token, first row of weights, 4 sums).  MAXB: column tiles at most (of all
// tokens).  per_wave: 1 / waves of the grid.  red: LDS for the sums of a tile's waves but the first.
constexpr int few_red(int maxb) { return (kFewWaves - 1) * maxb * 64; }
template <bool PACKED, bool X_F32, int NP, int MAXB, int SEG, bool STREAM, class F>
__device__ __forceinline__ void few_gemm(const FewTable* t, const char* W, const void* X, size_t plane, int x_row, int Kdim, int Ndim,
                                         float per_wave, float4* red, F&& epilogue) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  constexpr int R = kFewRowsTile / SEG;
  const unsigned tiles = (unsigned)(Ndim + R - 1) / R, items = t->groups * tiles;
  const int steps = (Kdim / SEG + 31) / 32;
  // 2^lks waves per tile: the fewest k-steps one after another, counting four for a turn of tiles' latency
  int lks = 0;
  float least = 3e38f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float turns = ceilf((float)(items << i) * per_wave);
    const float cost = turns * (float)(((steps - 1) >> i) + 5);
    if (cost < least) { least = cost; lks = i; }
  }
  const int ks = 1 << lks, per = kFewWaves >> lks, sub = wave & (ks - 1), mine = wave >> lks;
  const int units = !PACKED && STREAM ? steps / 2 : steps;  // (row-major weights past the caches go by lines of two steps)
  const int s0 = units * sub >> lks, s1 = units * (sub + 1) >> lks;
  int u = 0;
  unsigned at = blockIdx.x * per + mine;  // number in group u
  for (unsigned i0 = blockIdx.x * per; i0 < items; i0 += gridDim.x * per, at += gridDim.x * per) {
    const bool have = i0 + mine < items;
    if (have)
      while (at >= tiles) { at -= tiles; ++u; }
    const int tile = have ? (int)at : 0;
    const int first = __builtin_amdgcn_readfirstlane(t->start[u]);
    const int32_t* tok = t->token + first;
    const int n = __builtin_amdgcn_readfirstlane(t->start[u + 1]) - first;
    const char* We = W + (size_t)__builtin_amdgcn_readfirstlane(t->expert[u]) * Ndim * Kdim * 2;
    f32x4 acc[MAXB];
    auto dot = [&](auto nb_) {
      constexpr int NB = decltype(nb_)::value;
      f32x4 part[NB];
      few_dot<PACKED, X_F32, NP, NB, SEG, STREAM>(part, We, X, plane, x_row, tok, n, tile, Kdim, Ndim, s0, s1);
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = part[b];
    };
    if (have) {
      if (MAXB == 1 || n <= 16) dot(std::integral_constant<int, 1>{});
      else if constexpr (MAXB > 1) {
        if (n <= 32) dot(std::integral_constant<int, 2>{});
        else dot(std::integral_constant<int, 4>{});
      }
    }
    const int nb = (n + 15) / 16;
    if (ks > 1) {
      float4* sums = red + mine * (ks - 1) * (MAXB * 64) + lane;
      if (have && sub) {
#pragma unroll
        for (int b = 0; b < MAXB; ++b)
          if (b < nb) sums[((sub - 1) * MAXB + b) * 64] = make_float4(acc[b][0], acc[b][1], acc[b][2], acc[b][3]);
      }
      __syncthreads();
      if (have && !sub) {
        for (int j = 0; j < ks - 1; ++j)
#pragma unroll
          for (int b = 0; b < MAXB; ++b)
            if (b < nb) {
              const float4 v = sums[(j * MAXB + b) * 64];
              acc[b][0] += v.x; acc[b][1] += v.y; acc[b][2] += v.z; acc[b][3] += v.w;
            }
      }
    }
    if (have && !sub) {
      if constexpr (SEG > 1) {  // the blocks of the diagonal
        const f32x4 a = acc[0];
#pragma unroll
        for (int i = 1; i < SEG; ++i)
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[0][v] += __shfl(a[v], lane + i * (64 / SEG + R));
      }
#pragma unroll
      for (int b = 0; b < MAXB; ++b) {
        const int c = 16 * b + (lane & 15), r = tile * R + (lane >> 4) * 4;
        // (Ndim is a multiple of 8: the quad is inside or outside)
        if (c < n && (SEG == 1 || (lane < 64 / SEG && (lane & 15) < R)) && r < Ndim) epilogue(tok[c], r, acc[b]);
      }
    }
    if (ks > 1 && i0 + gridDim.x * per < items) __syncthreads();  // (red has been read)
  }
}

// (four waves per SIMD: two work-groups per compute unit)
template <bool BF16, bool PACKED, int MAXB, int SEG, bool STREAM>
__global__ __launch_bounds__(kFewThreads, 4) void few_in_kernel(const void* __restrict__ x, const float* __restrict__ g,
                                                                const float* __restrict__ eps,
                                                                const char* __restrict__ W, int32_t* __restrict__ eid,
                                                                float* __restrict__ w, int32_t* __restrict__ slot,
                                                                FewTable* __restrict__ table, uint16_t* __restrict__ H,
                                                                int T, int d, int E, int h, int C, int relu, FewRoute plan,
                                                                float per_wave) {
  __shared__ int32_t s_eid[kFewTokens], s_slot[kFewTokens];
  __shared__ float s_w[kFewTokens];
  __shared__ FewTable t;
  __shared__ float4 red[few_red(MAXB)];
  const int wave = threadIdx.x >> 6;
  few_route<BF16>(plan, x, g, eps, T, d, E, relu, s_eid, s_w);
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
  const size_t plane = (size_t)T * few_h_row(h);
  few_gemm<PACKED, !BF16, NP, MAXB, SEG, STREAM>(&t, W, x, 0, d, d, h, per_wave, red, [&](int m, int r, const f32x4& a) {
    uint16_t* dst = H + (size_t)m * few_h_row(h) + r;
    if constexpr (BF16) {
      *(uint2*)dst = make_uint2(pack_bf16x2(gelu_bf16(a[0]), gelu_bf16(a[1])), pack_bf16x2(gelu_bf16(a[2]), gelu_bf16(a[3])));
    } else {
      uint32_t lo[3], hi[3];
      split3(gelu_f32(a[0]), gelu_f32(a[1]), lo);
      split3(gelu_f32(a[2]), gelu_f32(a[3]), hi);
#pragma unroll
      for (int p = 0; p < 3; ++p) *(uint2*)(dst + p * plane) = make_uint2(lo[p], hi[p]);
    }
  });
}

template <bool BF16, bool PACKED, int MAXB, int SEG, bool STREAM>
__global__ __launch_bounds__(kFewThreads, 4) void few_out_kernel(const uint16_t* __restrict__ H,
                                                                 const FewTable* __restrict__ table,
                                                                 const int32_t* __restrict__ slot,
                                                                 const float* __restrict__ w,
                                                                 const char* __restrict__ W, void* __restrict__ y, int T,
                                                                 int d, int h, int weighted, float per_wave) {
  __shared__ FewTable t;
  __shared__ float4 red[few_red(MAXB)];
  for (int i = threadIdx.x; i < (int)(sizeof(FewTable) / 4); i += kFewThreads) ((int32_t*)&t)[i] = ((const int32_t*)table)[i];
  __syncthreads();
  if (weighted) {  // dropped tokens
    const int chunks = d / (BF16 ? 8 : 4);
    for (int m = blockIdx.x; m < T; m += gridDim.x)
      if (slot[m] < 0)
        for (int c = threadIdx.x; c < chunks; c += kFewThreads) ((uint4*)y)[(size_t)m * chunks + c] = make_uint4(0, 0, 0, 0);
  }
  few_gemm<PACKED, false, BF16 ? 1 : 3, MAXB, SEG, STREAM>(&t, W, H, (size_t)T * few_h_row(h), few_h_row(h), h, d, per_wave, red, [&](int m, int r, const f32x4& a) {
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
  if (check_desc(desc) != LOCMOE_OK || desc->T > kFewTokens || std::max(desc->d, desc->h) > LOCMOE_FEW_MAX_WIDTH) return 0;
  const size_t planes = desc->x_dtype == LOCMOE_BF16 ? 1 : 3;
  return (kFewHOffset + planes * (size_t)desc->T * (size_t)few_h_row(desc->h) * 2 + 255) & ~(size_t)255;
}

extern "C" int locmoe_layer_few(const locmoe_desc* desc, const void* x, const float* g, const float* eps, const void* W_in,
                                const void* W_out, int32_t weighted, int32_t* eid, float* w, int32_t* slot, void* y,
                                void* ws, size_t ws_bytes, void* stream) {
  using namespace locmoe;
  if (!desc || !x || !W_in || !W_out || !eid || !w || !slot || !y) return LOCMOE_ERR_NULL;
  const int st = check_desc(desc);
  if (st != LOCMOE_OK) return st;
  if (desc->T > kFewTokens || std::max(desc->d, desc->h) > LOCMOE_FEW_MAX_WIDTH) return LOCMOE_ERR_SHAPE;
  if (weighted != 0 && weighted != 1) return LOCMOE_ERR_ARG;
  const bool bf = desc->x_dtype == LOCMOE_BF16;
  if (desc->w_packed && (!bf || locmoe_packed_weights_bytes(desc) == 0)) return LOCMOE_ERR_ARG;
  if (!ws || ws_bytes < locmoe_layer_few_workspace_bytes(desc)) return LOCMOE_ERR_WORKSPACE;
  const int T = desc->T, d = desc->d, E = desc->E, h = desc->h;
  hipStream_t s = as_stream(stream);
  FewTable* table = (FewTable*)ws;
  uint16_t* H = (uint16_t*)((char*)ws + kFewHOffset);
  const FewRoute plan = few_route_plan(T, d, E);
  // Tiles of 16 rows of weights, or of 8 or 4 where those leave compute units without one (one token, d = 1024, h = 4096, second
  // GEMM: 64 tiles of 16 rows 5.5 us, 256 of 4 rows 4.9)
  auto segments = [&](int N, int K) {
    int seg = 1;
    while (seg < 4 && 2 * seg * T <= 16 && K % (64 * seg) == 0 &&
           (long long)std::min(T, E) * ceil_div(N, kFewRowsTile / seg) < cu_count())
      seg *= 2;
    return seg;
  };
  // past the caches? (groups: as many as there can be)
  auto streams = [&](int N, int K, int seg) {
    return seg == 1 && (desc->w_packed || K % 64 == 0) && (long long)std::min(T, E) * N * K * 2 > kFewStreamBytes;
  };
  // two work-groups per compute unit, no more than there can be tiles (of up to eight waves each)
  auto groups = [&](int N, int seg) {
    return (unsigned)std::min<long long>(2 * cu_count(), (long long)std::min(T, E) * ceil_div(N, kFewRowsTile / seg));
  };
  auto launch = [&](auto bf16, auto packed, auto maxb) {
    constexpr bool BF = decltype(bf16)::value, PK = decltype(packed)::value;
    constexpr int MAXB = decltype(maxb)::value;
    const int seg_in = segments(h, d), seg_out = segments(d, h);
    const unsigned in = groups(h, seg_in), out = groups(d, seg_out);
    auto k_in = streams(h, d, seg_in) ? few_in_kernel<BF, PK, MAXB, 1, true> : few_in_kernel<BF, PK, MAXB, 1, false>;
    auto k_out = streams(d, h, seg_out) ? few_out_kernel<BF, PK, MAXB, 1, true> : few_out_kernel<BF, PK, MAXB, 1, false>;
    if constexpr (MAXB == 1) {
      if (seg_in > 1) k_in = seg_in == 2 ? few_in_kernel<BF, PK, 1, 2, false> : few_in_kernel<BF, PK, 1, 4, false>;
      if (seg_out > 1) k_out = seg_out == 2 ? few_out_kernel<BF, PK, 1, 2, false> : few_out_kernel<BF, PK, 1, 4, false>;
    }
    hipLaunchKernelGGL(k_in, dim3(in), dim3(kFewThreads), 0, s, x, g, eps, (const char*)W_in, eid, w, slot, table, H, T, d, E, h,
                       desc->C, desc->relu, plan, 1.0f / (float)(in * kFewWaves));
    hipLaunchKernelGGL(k_out, dim3(out), dim3(kFewThreads), 0, s, H, table, slot, w, (const char*)W_out, y, T, d, h, weighted,
                       1.0f / (float)(out * kFewWaves));
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
