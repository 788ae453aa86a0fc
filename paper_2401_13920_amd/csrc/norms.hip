// The norms of a transformer block around the layer, each in one pass with its neighbour in the path:
//   locmoe_norm_gate          xn = x r gamma, r = 1 / sqrt(mean x^2 + eps), and Eq. 4's gating value of it
//   locmoe_combine_norm       y = res + scale w gamma n, n = out[slot] r (or out[slot] itself): combine, norm, residual
//   locmoe_combine_norm_bwd   its gradients: dout, dw, dgamma
//   locmoe_dispatch_norm_bwd  dxn = dsend[slot] + (E/d) dg, and the norm's backward: dx, dgamma
// Every row is read once, held in registers between the sum over it and its use, and written once.  LPR lanes share a row,
// CPL 16-byte chunks each.  (Backward, rows of more than 32 KiB: gamma and its gradient do not fit beside the row in the 128
// registers of a work-group of 1 024, and spill: bf16, d = 32 768, 4 096 tokens 511 and 745 us, 1.6 and 1.4 TB/s, where d = 16 384
// with 8 192 tokens takes 181 and 208.  fp32 rows, and bf16 ones of 16 to 32 KiB whose blocks are no whole chunks, spill a few
// words: 5.1 and 5.5 TB/s, 4.2 and 4.9.)  All of it is bound by memory, loaded and stored past the caches: with T = 65 536 tokens, d = 4096, E = 64,
// bf16, 31 200 of them kept, norm_gate takes 196 us (1.09 GB, 5.6 TB/s), combine_norm 217 (1.34 GB, 6.2), combine_norm_bwd 158
// (0.79 GB, 5.0) and dispatch_norm_bwd 323 (1.90 GB, 5.9); a plain copy reaches 5.7.  With 64 tokens of d = 1024 each takes 3.4 us,
// less than its launch from the host.
//
// A column's gradient (dgamma) is a sum over tokens: a work-group sums its rows in registers, writes one row of partial
// sums to the workspace, and a second kernel adds those in a fixed order: no atomics, the same bits every time.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "common.h"

namespace locmoe {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormMaxParts = 1024;         // rows of partial sums at most
constexpr int kNormMaxChunks = LOCMOE_NORM_MAX_ROW_BYTES / 16;
constexpr int kMaxNormLds = kNormMaxChunks * 8 * 4;  // every feature of the longest row

template <bool BF16>
struct Vec {
  static constexpr int N = BF16 ? 8 : 4;
};

template <bool BF16>
__device__ __forceinline__ void unpack16(const uint4& v, float (&a)[Vec<BF16>::N]) {
  const uint32_t* p = &v.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      a[2 * i] = bf16_bits_to_f32(p[i] & 0xFFFFu);
      a[2 * i + 1] = __uint_as_float(p[i] & 0xFFFF0000u);
    } else {
      a[i] = __uint_as_float(p[i]);
    }
  }
}
template <bool BF16>
__device__ __forceinline__ uint4 pack16(const float (&a)[Vec<BF16>::N]) {
  uint4 r;
  uint32_t* p = &r.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) p[i] = pack_bf16x2(a[2 * i], a[2 * i + 1]);
    else p[i] = __float_as_uint(a[i]);
  }
  return r;
}
template <bool BF16>
__device__ __forceinline__ float sumsq16(const uint4& v) {
  return BF16 ? sumsq8_bf16(v) : sumsq4_f32(v);
}
// N floats of a vector over the columns (gamma); ones if there is none
template <int N>
__device__ __forceinline__ void load_cols(const float* p, int c, float (&a)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = p ? *(const float4*)(p + (size_t)c * N + i) : make_float4(1.f, 1.f, 1.f, 1.f);
    a[i] = v.x; a[i + 1] = v.y; a[i + 2] = v.z; a[i + 3] = v.w;
  }
}

template <int LPR>
constexpr int threads_of() { return LPR > kNormThreads ? LPR : kNormThreads; }

// The sum over a row's LPR lanes, in every one of them.  Rows of more than a wave go through LDS words of `sm`, which the
// caller alternates between two sets (one barrier per sum).
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* sm) {
  if constexpr (LPR <= kWave) {
    return group_sum<LPR>(v);
  } else {
    constexpr int W = LPR / kWave;
    v = group_sum<kWave>(v);
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0) sm[wave] = v;
    __syncthreads();
    const int w0 = wave / W * W;
    float s = sm[w0];
#pragma unroll
    for (int i = 1; i < W; ++i) s += sm[w0 + i];
    return s;
  }
}
// How the means of the d/E features are formed: kLanes, a block is a power of two of chunks, held by neighbouring lanes of a
// wave; kChunks, whole chunks, whose sums go through LDS; kElements, neither: every feature goes through LDS.
enum GateForm { kLanes, kChunks, kElements };

template <bool BF16, int LPR, int CPL, int GATE>
__global__ __launch_bounds__(threads_of<LPR>()) void norm_gate_kernel(const uint4* x,
                                                                      const float* __restrict__ gamma,
                                                                      uint4* xn, float* __restrict__ rstd,
                                                                      float* __restrict__ g, int T, int chunks, int E,
                                                                      int blk, float inv_d, float eps) {
  constexpr int V = Vec<BF16>::N, THREADS = threads_of<LPR>(), RPB = THREADS / LPR;
  __shared__ float sm[THREADS / kWave];
  extern __shared__ float part[];  // kChunks: [RPB][chunks], kElements: [RPB][chunks V]
  const int rg = threadIdx.x / LPR, l = threadIdx.x % LPR;
  const unsigned m = blockIdx.x * RPB + rg;
  const bool live = m < (unsigned)T;
  const uint4* src = x + (size_t)(live ? m : T - 1) * chunks;
  uint4 v[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    v[i] = c < chunks ? nt_load16(src + c) : make_uint4(0, 0, 0, 0);
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) ss += sumsq16<BF16>(v[i]);
  const float r = 1.0f / sqrtf(row_sum<LPR>(ss, sm) * inv_d + eps);
  const float inv_blk = 1.0f / (float)blk;
  const int L = blk / V;  // (kLanes, kChunks)
  if (live && l == 0 && rstd) rstd[m] = r;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    const bool in = c < chunks;
    float a[V], gm[V];
    unpack16<BF16>(v[i], a);
    load_cols<V>(gamma, in ? c : 0, gm);
#pragma unroll
    for (int k = 0; k < V; ++k) a[k] = a[k] * r * gm[k];
    if (in && live) nt_store16(pack16<BF16>(a), xn + (size_t)m * chunks + c);
    if (!g) continue;
    if constexpr (GATE == kElements) {
      if (in) {
#pragma unroll
        for (int k = 0; k < V; ++k) part[((size_t)rg * chunks + c) * V + k] = a[k];
      }
    } else {
      float s = (a[0] + a[1]) + (a[2] + a[3]);
      if constexpr (V == 8) s += (a[4] + a[5]) + (a[6] + a[7]);
      if constexpr (GATE == kLanes) {
        s = lanes_sum(in ? s : 0.f, L);
        if (in && live && (l & (L - 1)) == 0) g[(size_t)m * E + c / L] = s * inv_blk;
      } else {
        if (in) part[(size_t)rg * chunks + c] = s;
      }
    }
  }
  if constexpr (GATE != kLanes) {
    if (!g) return;
    __syncthreads();
    // P lanes per output
    const int n = GATE == kElements ? blk : L;
    const float* row = part + (size_t)rg * chunks * (GATE == kElements ? V : 1);
    int P = 1;
    while (2 * P * E <= LPR && P < kWave && P < n) P *= 2;
    for (int o0 = 0; o0 < E; o0 += LPR / P) {
      const int o = o0 + l / P;
      float s = 0.f;
      if (o < E)
        for (int k = l % P; k < n; k += P) s += row[o * n + k];
      s = lanes_sum(s, P);
      if (o < E && live && l % P == 0) g[(size_t)m * E + o] = s * inv_blk;
    }
  }
}

// POST: the norm behind the layer.  A dropped token's row is its residual, bit for bit.
template <bool BF16, int LPR, int CPL, bool POST>
__global__ __launch_bounds__(threads_of<LPR>()) void combine_norm_kernel(const uint4* __restrict__ out,
                                                                         const int32_t* __restrict__ slot,
                                                                         const float* __restrict__ w, const uint4* res,
                                                                         const float* __restrict__ gamma, uint4* y,
                                                                         float* __restrict__ rstd, int T, int chunks,
                                                                         float inv_d, float eps, float scale) {
  constexpr int V = Vec<BF16>::N, THREADS = threads_of<LPR>(), RPB = THREADS / LPR;
  __shared__ float sm[THREADS / kWave];
  const int rg = threadIdx.x / LPR, l = threadIdx.x % LPR;
  const unsigned m = blockIdx.x * RPB + rg;
  const bool live = m < (unsigned)T;
  const int s = live ? slot[m] : -1;
  uint4 vo[CPL], vr[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    vr[i] = live && c < chunks ? nt_load16(res + (size_t)m * chunks + c) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    vo[i] = s >= 0 && c < chunks ? nt_load16(out + (size_t)s * chunks + c) : make_uint4(0, 0, 0, 0);
  }
  float r = 1.0f;
  if (POST) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) ss += sumsq16<BF16>(vo[i]);
    r = 1.0f / sqrtf(row_sum<LPR>(ss, sm) * inv_d + eps);
  }
  if (!live) return;
  if (l == 0 && rstd) rstd[m] = s >= 0 ? r : 0.f;
  const float f = s >= 0 ? scale * w[m] * r : 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    if (c >= chunks) continue;
    uint4 o = vr[i];
    if (s >= 0) {
      float a[V], b[V], gm[V];
      unpack16<BF16>(vo[i], a);
      unpack16<BF16>(vr[i], b);
      load_cols<V>(gamma, c, gm);
#pragma unroll
      for (int k = 0; k < V; ++k) b[k] = fmaf(a[k] * f, gm[k], b[k]);
      o = pack16<BF16>(b);
    }
    nt_store16(o, y + (size_t)m * chunks + c);
  }
}

// The partial column sums of a work-group's rows -> row blockIdx.x of `part`.  Row groups are added in order through LDS.
template <int LPR, int CPL, int V>
__device__ __forceinline__ void store_partial(const float (&acc)[CPL][V], float* part, int chunks, float* lds) {
  constexpr int RPB = threads_of<LPR>() / LPR;
  const int rg = threadIdx.x / LPR, l = threadIdx.x % LPR;
  float* dst = part + (size_t)blockIdx.x * chunks * V;
  if constexpr (RPB > 1) {
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int k = 0; k < V; k += 4)
        *(float4*)(lds + ((rg * CPL + i) * LPR + l) * V + k) =
            make_float4(acc[i][k], acc[i][k + 1], acc[i][k + 2], acc[i][k + 3]);
    __syncthreads();
    for (int q = threadIdx.x; q < CPL * LPR * V; q += threads_of<LPR>()) {
      float s = lds[q];
      for (int j = 1; j < RPB; ++j) s += lds[j * CPL * LPR * V + q];
      if (q < chunks * V) dst[q] = s;  // (chunk l + i LPR, value k: the column order)
    }
  } else {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int c = l + i * LPR;
      if (c < chunks) {
#pragma unroll
        for (int k = 0; k < V; k += 4)
          *(float4*)(dst + (size_t)c * V + k) = make_float4(acc[i][k], acc[i][k + 1], acc[i][k + 2], acc[i][k + 3]);
      }
    }
  }
}

// A work-group walks the tokens a stride apart, with the next one's slot in flight; dropped tokens cost that slot alone.  Gathered
// rows, a barrier a row (of more than a wave) and the sums in registers leave 5.0 TB/s; half as many work-groups or twice as many
// take 4 to 11 % longer (both gradients together 497 us, 512 of them 555, 2 048 506), the next row's loads ahead of this one's
// sum 565.
// With n the row that the forward multiplied (out r, or out without the norm) and u = scale gamma dy:
//   dw = <u, n>,   dgamma += scale w dy n,   dout = r w (u - n dw / d), or w u without the norm.
template <bool BF16, int LPR, int CPL, bool POST>
__global__ __launch_bounds__(threads_of<LPR>()) void combine_norm_bwd_kernel(
    const uint4* __restrict__ dy, const uint4* __restrict__ out, const int32_t* __restrict__ slot,
    const float* __restrict__ w, const float* __restrict__ gamma, const float* __restrict__ rstd, uint4* __restrict__ dout,
    float* __restrict__ dw, float* __restrict__ part, int T, int chunks, float inv_d, float scale) {
  constexpr int V = Vec<BF16>::N, THREADS = threads_of<LPR>(), RPB = THREADS / LPR;
  __shared__ float sm[2][THREADS / kWave];
  __shared__ float lds[RPB > 1 ? THREADS * CPL * V : 1];
  const int rg = threadIdx.x / LPR, l = threadIdx.x % LPR;
  float gm[CPL][V], acc[CPL][V];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    load_cols<V>(gamma, c < chunks ? c : 0, gm[i]);
#pragma unroll
    for (int k = 0; k < V; ++k) { gm[i][k] *= scale; acc[i][k] = 0.f; }
  }
  int set = 0;
  int s_next = blockIdx.x * RPB + rg < (unsigned)T ? slot[blockIdx.x * RPB + rg] : -1;
  for (unsigned m0 = blockIdx.x * RPB; m0 < (unsigned)T; m0 += gridDim.x * RPB) {
    const unsigned m = m0 + rg, m_next = m + gridDim.x * RPB;
    const int s = s_next;
    s_next = m_next < (unsigned)T ? slot[m_next] : -1;
    if (s < 0) {  // (rows of more than a wave are a work-group's alone: all of it goes on, past the sum's barrier too)
      if (m < (unsigned)T && l == 0) dw[m] = 0.f;
      continue;
    }
    const float wm = w[m], r = POST ? rstd[m] : 1.f;
    uint4 vd[CPL], vo[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int c = l + i * LPR;
      const bool in = c < chunks;
      vd[i] = in ? nt_load16(dy + (size_t)m * chunks + c) : make_uint4(0, 0, 0, 0);
      vo[i] = in ? nt_load16(out + (size_t)s * chunks + c) : make_uint4(0, 0, 0, 0);
    }
    const float ws = wm * scale;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float a[V], b[V];
      unpack16<BF16>(vd[i], a);
      unpack16<BF16>(vo[i], b);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float n = b[k] * r;
        dot = fmaf(a[k] * gm[i][k], n, dot);
        acc[i][k] = fmaf(a[k] * ws, n, acc[i][k]);
      }
    }
    dot = row_sum<LPR>(dot, sm[set]);
    set ^= 1;
    if (l == 0) dw[m] = dot;
    const float mean = POST ? dot * inv_d : 0.f, wr = wm * r;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int c = l + i * LPR;
      if (c >= chunks) continue;
      float a[V], b[V];
      unpack16<BF16>(vd[i], a);
      unpack16<BF16>(vo[i], b);
#pragma unroll
      for (int k = 0; k < V; ++k) a[k] = wr * (POST ? fmaf(-mean, b[k] * r, a[k] * gm[i][k]) : a[k] * gm[i][k]);
      nt_store16(pack16<BF16>(a), dout + (size_t)s * chunks + c);
    }
  }
  if (part) store_partial<LPR, CPL, V>(acc, part, chunks, lds);
}

// VEC_BLOCK: a chunk lies inside one GrAP block.  With xh = x r, dh = dxn gamma:
//   dgamma += dxn xh,   dx = dres + r (dh - xh mean(dh xh)).
template <bool BF16, int LPR, int CPL, bool VEC_BLOCK>
__global__ __launch_bounds__(threads_of<LPR>()) void dispatch_norm_bwd_kernel(
    const uint4* __restrict__ dsend, const int32_t* __restrict__ slot, const float* __restrict__ dg,
    const uint4* x, const float* __restrict__ gamma, const float* __restrict__ rstd, const uint4* dres, uint4* dx,
    float* __restrict__ part, int T, int chunks, int E, int blk, float inv_d, float dg_scale) {
  constexpr int V = Vec<BF16>::N, THREADS = threads_of<LPR>(), RPB = THREADS / LPR;
  __shared__ float sm[2][THREADS / kWave];
  __shared__ float lds[RPB > 1 ? THREADS * CPL * V : 1];
  const int rg = threadIdx.x / LPR, l = threadIdx.x % LPR;
  float gm[CPL][V], acc[CPL][V];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int c = l + i * LPR;
    load_cols<V>(gamma, c < chunks ? c : 0, gm[i]);
#pragma unroll
    for (int k = 0; k < V; ++k) acc[i][k] = 0.f;
  }
  int set = 0;
  int s_next = blockIdx.x * RPB + rg < (unsigned)T ? slot[blockIdx.x * RPB + rg] : -1;
  for (unsigned m0 = blockIdx.x * RPB; m0 < (unsigned)T; m0 += gridDim.x * RPB, set ^= 1) {
    const unsigned m = m0 + rg, m_next = m + gridDim.x * RPB;
    const int s = s_next;
    s_next = m_next < (unsigned)T ? slot[m_next] : -1;
    const bool live = m < (unsigned)T;
    const float r = live ? rstd[m] : 0.f;
    uint4 vs[CPL], vx[CPL], vr[CPL];
    float t[CPL][VEC_BLOCK ? 1 : V];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int c = l + i * LPR;
      const bool in = live && c < chunks;
      vs[i] = in && s >= 0 ? nt_load16(dsend + (size_t)s * chunks + c) : make_uint4(0, 0, 0, 0);
      vx[i] = in ? nt_load16(x + (size_t)m * chunks + c) : make_uint4(0, 0, 0, 0);
      vr[i] = in && dres ? nt_load16(dres + (size_t)m * chunks + c) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < (VEC_BLOCK ? 1 : V); ++k) t[i][k] = in ? dg_scale * dg[(size_t)m * E + (c * V + k) / blk] : 0.f;
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      float a[V], b[V];
      unpack16<BF16>(vs[i], a);
      unpack16<BF16>(vx[i], b);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float dxn = a[k] + t[i][VEC_BLOCK ? 0 : k], p = dxn * (b[k] * r);
        acc[i][k] += p;
        dot = fmaf(p, gm[i][k], dot);
      }
    }
    const float mean = row_sum<LPR>(dot, sm[set]) * inv_d;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int c = l + i * LPR;
      if (c >= chunks) continue;
      float a[V], b[V], q[V];
      unpack16<BF16>(vs[i], a);
      unpack16<BF16>(vx[i], b);
      unpack16<BF16>(vr[i], q);
#pragma unroll
      for (int k = 0; k < V; ++k)
        a[k] = fmaf(r, fmaf(a[k] + t[i][VEC_BLOCK ? 0 : k], gm[i][k], -(b[k] * r) * mean), q[k]);
      nt_store16(pack16<BF16>(a), dx + (size_t)m * chunks + c);
    }
  }
  if (part) store_partial<LPR, CPL, V>(acc, part, chunks, lds);
}

// dgamma[j] = sum of column j over the rows of partial sums.  A work-group makes 16 columns: four lanes of four columns, 64 row
// groups with up to 16 loads in flight each, whose sums are added in a fixed order through LDS.  1 024 rows of 4 096 columns: 7.0 us
// (64 columns per work-group, which leave most compute units idle, 8.4), of 1 600 columns 4.7.
constexpr int kSumCols = 16;
__global__ __launch_bounds__(256) void column_sum_kernel(const float* __restrict__ part, float* __restrict__ dgamma,
                                                         int rows, int d) {
  __shared__ float4 s[64][4];
  const int j = threadIdx.x & 3, rg = threadIdx.x >> 2, col = blockIdx.x * kSumCols + j * 4;
  const float* p = part + min(col, d - 4);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int U = 16;
  for (int q0 = rg; q0 < rows; q0 += 64 * U) {
    float4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *(const float4*)(p + (size_t)min(q0 + 64 * u, rows - 1) * d);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q0 + 64 * u < rows) { a.x += v[u].x; a.y += v[u].y; a.z += v[u].z; a.w += v[u].w; }
  }
  s[rg][j] = a;
  __syncthreads();
  if (threadIdx.x < 32) {  // eight row groups a lane, then the eight lanes of a column
    a = s[rg * 8][j];
#pragma unroll
    for (int i = 1; i < 8; ++i) { const float4 v = s[rg * 8 + i][j]; a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; }
#pragma unroll
    for (int o = 4; o < 32; o *= 2) {
      a.x += __shfl_xor(a.x, o); a.y += __shfl_xor(a.y, o); a.z += __shfl_xor(a.z, o); a.w += __shfl_xor(a.w, o);
    }
    if (rg == 0 && col < d) *(float4*)(dgamma + col) = a;
  }
}

// The lanes of a row of `chunks` chunks: f(RowShape<lanes, chunks a lane>).  Forward rows are held by a wave or less where eight
// chunks a lane suffice (no barrier); backward rows, which carry gamma and its gradient in registers too, by more lanes.
template <int LPR_, int CPL_>
struct RowShape { static constexpr int LPR = LPR_, CPL = CPL_, kThreads = threads_of<LPR_>(), kRows = kThreads / LPR_; };
template <class F>
int with_forward_row(int chunks, F&& f) {
  if (chunks <= 16) return f(RowShape<16, 1>{});
  if (chunks <= 32) return f(RowShape<16, 2>{});
  if (chunks <= 64) return f(RowShape<64, 1>{});
  if (chunks <= 128) return f(RowShape<64, 2>{});
  if (chunks <= 256) return f(RowShape<64, 4>{});
  if (chunks <= 512) return f(RowShape<256, 2>{});
  if (chunks <= 1024) return f(RowShape<256, 4>{});
  if (chunks <= 2048) return f(RowShape<512, 4>{});
  return f(RowShape<1024, 4>{});
}
template <class F>
int with_backward_row(int chunks, F&& f) {
  if (chunks <= 16) return f(RowShape<16, 1>{});
  if (chunks <= 64) return f(RowShape<64, 1>{});
  if (chunks <= 128) return f(RowShape<64, 2>{});
  if (chunks <= 256) return f(RowShape<256, 1>{});
  if (chunks <= 512) return f(RowShape<256, 2>{});
  if (chunks <= 1024) return f(RowShape<512, 2>{});
  if (chunks <= 2048) return f(RowShape<1024, 2>{});
  return f(RowShape<1024, 4>{});
}

// What the four entry points share: the row in 16-byte chunks
struct NormRow {
  bool bf;
  int chunks, blk;
  float inv_d;
};
int norm_row(const locmoe_desc* p, NormRow* r) {
  const int st = check_desc(p);
  if (st != LOCMOE_OK) return st;
  r->bf = p->x_dtype == LOCMOE_BF16;
  r->chunks = p->d / (r->bf ? 8 : 4);
  r->blk = p->d / p->E;
  r->inv_d = 1.0f / (float)p->d;
  return r->chunks > kNormMaxChunks ? LOCMOE_ERR_SHAPE : LOCMOE_OK;
}
inline bool finite(float v) { return v - v == 0.0f; }

// (T fills 31 bits: no sum with it that may not fit them)
inline int part_rows(int T, int rows_per_group) { return std::min((T - 1) / rows_per_group + 1, kNormMaxParts); }

// The forward kernels have a work-group for every few rows, and a launch takes fewer than 2^32 threads: f(first row, rows) for runs of
// rows of 2^31 threads each.  (2^27 rows of up to 32 chunks, 2^21 of the longest)
template <class S, class F>
int by_runs(int T, F&& f) {
  constexpr long long kRun = (1ll << 31) / S::kThreads * S::kRows;
  for (long long m0 = 0; m0 < T; m0 += kRun) {
    const int st = f((size_t)m0, (int)std::min<long long>(kRun, T - m0));
    if (st != LOCMOE_OK) return st;
  }
  return LOCMOE_OK;
}

template <bool BF>
int norm_gate_impl(const NormRow& row, const locmoe_desc* desc, const void* x, const float* gamma, float eps, void* xn,
                   float* rstd, float* g, hipStream_t s) {
  const int T = desc->T, E = desc->E, V = Vec<BF>::N, L = row.blk / V;
  return with_forward_row(row.chunks, [&](auto shape) {
    using S = decltype(shape);
    const GateForm form = row.blk % V ? kElements : (L & (L - 1)) == 0 && L <= std::min(S::LPR, kWave) ? kLanes : kChunks;
    const size_t lds = !g || form == kLanes ? 0 : (size_t)S::kRows * row.chunks * (form == kElements ? V : 1) * 4;
    auto kern = form == kLanes    ? norm_gate_kernel<BF, S::LPR, S::CPL, kLanes>
                : form == kChunks ? norm_gate_kernel<BF, S::LPR, S::CPL, kChunks>
                                  : norm_gate_kernel<BF, S::LPR, S::CPL, kElements>;
    static std::atomic<uint64_t> allowed[3];
    // (the limit without asking is 64 KiB, some of which are the kernel's own words)
    if (lds > 60000 && !allow_lds((const void*)kern, kMaxNormLds, allowed[form])) return (int)LOCMOE_ERR_HIP;
    return by_runs<S>(T, [&](size_t m0, int n) {
      hipLaunchKernelGGL(kern, dim3(ceil_div(n, S::kRows)), dim3(S::kThreads), lds, s, (const uint4*)x + m0 * row.chunks, gamma,
                         (uint4*)xn + m0 * row.chunks, rstd ? rstd + m0 : nullptr, g ? g + m0 * E : nullptr, n, row.chunks, E,
                         row.blk, row.inv_d, eps);
      return launch_status();
    });
  });
}

template <bool BF>
int combine_norm_impl(const NormRow& row, int T, const void* out, const int32_t* slot, const float* w, const void* res,
                      const float* gamma, bool post, float eps, float scale, void* y, float* rstd, hipStream_t s) {
  return with_forward_row(row.chunks, [&](auto shape) {
    using S = decltype(shape);
    auto kern = post ? combine_norm_kernel<BF, S::LPR, S::CPL, true> : combine_norm_kernel<BF, S::LPR, S::CPL, false>;
    return by_runs<S>(T, [&](size_t m0, int n) {
      hipLaunchKernelGGL(kern, dim3(ceil_div(n, S::kRows)), dim3(S::kThreads), 0, s, (const uint4*)out, slot + m0, w + m0,
                         (const uint4*)res + m0 * row.chunks, gamma, (uint4*)y + m0 * row.chunks, rstd ? rstd + m0 : nullptr, n,
                         row.chunks, row.inv_d, eps, scale);
      return launch_status();
    });
  });
}

void sum_columns(const float* part, float* dgamma, int rows, int d, hipStream_t s) {
  if (dgamma) hipLaunchKernelGGL(column_sum_kernel, dim3(ceil_div(d, kSumCols)), dim3(256), 0, s, part, dgamma, rows, d);
}

template <bool BF>
int combine_norm_bwd_impl(const NormRow& row, const locmoe_desc* desc, const void* dy, const void* out, const int32_t* slot,
                          const float* w, const float* gamma, bool post, float scale, const float* rstd, void* dout,
                          float* dw, float* dgamma, void* ws, hipStream_t s) {
  return with_backward_row(row.chunks, [&](auto shape) {
    using S = decltype(shape);
    const int rows = part_rows(desc->T, S::kRows);
    float* part = dgamma ? (float*)ws : nullptr;
    auto kern = post ? combine_norm_bwd_kernel<BF, S::LPR, S::CPL, true> : combine_norm_bwd_kernel<BF, S::LPR, S::CPL, false>;
    hipLaunchKernelGGL(kern, dim3(rows), dim3(S::kThreads), 0, s, (const uint4*)dy, (const uint4*)out, slot, w, gamma, rstd,
                       (uint4*)dout, dw, part, desc->T, row.chunks, row.inv_d, scale);
    sum_columns(part, dgamma, rows, desc->d, s);
    return launch_status();
  });
}

template <bool BF>
int dispatch_norm_bwd_impl(const NormRow& row, const locmoe_desc* desc, const void* dsend, const int32_t* slot,
                           const float* dg, const void* x, const float* gamma, const float* rstd, const void* dres, void* dx,
                           float* dgamma, void* ws, hipStream_t s) {
  return with_backward_row(row.chunks, [&](auto shape) {
    using S = decltype(shape);
    const int rows = part_rows(desc->T, S::kRows);
    float* part = dgamma ? (float*)ws : nullptr;
    auto kern = row.blk % Vec<BF>::N == 0 ? dispatch_norm_bwd_kernel<BF, S::LPR, S::CPL, true>
                                          : dispatch_norm_bwd_kernel<BF, S::LPR, S::CPL, false>;
    hipLaunchKernelGGL(kern, dim3(rows), dim3(S::kThreads), 0, s, (const uint4*)dsend, slot, dg, (const uint4*)x, gamma, rstd,
                       (const uint4*)dres, (uint4*)dx, part, desc->T, row.chunks, desc->E, row.blk, row.inv_d,
                       (float)desc->E / (float)desc->d);
    sum_columns(part, dgamma, rows, desc->d, s);
    return launch_status();
  });
}

inline bool norm_ws_ok(const locmoe_desc* desc, const float* dgamma, const void* ws, size_t ws_bytes) {
  return !dgamma || (ws && ws_bytes >= locmoe_norm_workspace_bytes(desc));
}

}  // namespace
}  // namespace locmoe

extern "C" size_t locmoe_norm_workspace_bytes(const locmoe_desc* desc) {
  using namespace locmoe;
  NormRow row;
  if (norm_row(desc, &row) != LOCMOE_OK) return 0;
  return (size_t)std::min(desc->T, kNormMaxParts) * (size_t)desc->d * 4;
}

extern "C" int locmoe_norm_gate(const locmoe_desc* desc, const void* x, const float* gamma, float norm_eps, void* xn,
                                float* rstd, float* g, void* stream) {
  using namespace locmoe;
  if (!desc || !x || !xn) return LOCMOE_ERR_NULL;
  NormRow row;
  const int st = norm_row(desc, &row);
  if (st != LOCMOE_OK) return st;
  if (!(norm_eps > 0.0f) || !finite(norm_eps)) return LOCMOE_ERR_ARG;
  return row.bf ? norm_gate_impl<true>(row, desc, x, gamma, norm_eps, xn, rstd, g, as_stream(stream))
                : norm_gate_impl<false>(row, desc, x, gamma, norm_eps, xn, rstd, g, as_stream(stream));
}

extern "C" int locmoe_combine_norm(const locmoe_desc* desc, const void* out, const int32_t* slot, const float* w,
                                   const void* res, const float* gamma, int32_t post_norm, float norm_eps, float scale,
                                   void* y, float* rstd, void* stream) {
  using namespace locmoe;
  if (!desc || !out || !slot || !w || !res || !y) return LOCMOE_ERR_NULL;
  NormRow row;
  const int st = norm_row(desc, &row);
  if (st != LOCMOE_OK) return st;
  if ((post_norm != 0 && post_norm != 1) || !finite(scale)) return LOCMOE_ERR_ARG;
  if (post_norm && (!(norm_eps > 0.0f) || !finite(norm_eps))) return LOCMOE_ERR_ARG;
  auto impl = row.bf ? combine_norm_impl<true> : combine_norm_impl<false>;
  return impl(row, desc->T, out, slot, w, res, gamma, post_norm, norm_eps, scale, y, rstd, as_stream(stream));
}

extern "C" int locmoe_combine_norm_bwd(const locmoe_desc* desc, const void* dy, const void* out, const int32_t* slot,
                                       const float* w, const float* gamma, int32_t post_norm, float scale,
                                       const float* rstd, void* dout, float* dw, float* dgamma, void* ws,
                                       size_t ws_bytes, void* stream) {
  using namespace locmoe;
  if (!desc || !dy || !out || !slot || !w || !dout || !dw || (post_norm && !rstd)) return LOCMOE_ERR_NULL;
  NormRow row;
  const int st = norm_row(desc, &row);
  if (st != LOCMOE_OK) return st;
  if ((post_norm != 0 && post_norm != 1) || !finite(scale)) return LOCMOE_ERR_ARG;
  if (!norm_ws_ok(desc, dgamma, ws, ws_bytes)) return LOCMOE_ERR_WORKSPACE;
  auto impl = row.bf ? combine_norm_bwd_impl<true> : combine_norm_bwd_impl<false>;
  return impl(row, desc, dy, out, slot, w, gamma, post_norm, scale, rstd, dout, dw, dgamma, ws, as_stream(stream));
}

extern "C" int locmoe_dispatch_norm_bwd(const locmoe_desc* desc, const void* dsend, const int32_t* slot, const float* dg,
                                        const void* x, const float* gamma, const float* rstd, const void* dres, void* dx,
                                        float* dgamma, void* ws, size_t ws_bytes, void* stream) {
  using namespace locmoe;
  if (!desc || !dsend || !slot || !dg || !x || !rstd || !dx) return LOCMOE_ERR_NULL;
  NormRow row;
  const int st = norm_row(desc, &row);
  if (st != LOCMOE_OK) return st;
  if (!norm_ws_ok(desc, dgamma, ws, ws_bytes)) return LOCMOE_ERR_WORKSPACE;
  auto impl = row.bf ? dispatch_norm_bwd_impl<true> : dispatch_norm_bwd_impl<false>;
  return impl(row, desc, dsend, slot, dg, x, gamma, rstd, dres, dx, dgamma, ws, as_stream(stream));
}
