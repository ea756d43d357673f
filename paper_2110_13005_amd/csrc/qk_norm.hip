// Norms of queries and keys for each head, with the position rotation in the same pass, on packed rows
// [heads * d | kv * d | kv * d] = [Q | K | V] (the layout attention reads), forward and backward.
//
//   r = 1 / sqrt(mean x^2 + eps),  xh = r x,  z = g xh,   (a, b) -> (a cos - b sin, a sin + b cos) for every rotated pair of z
//   backward: dz = the inverse rotation of dy,  w = g dz,  dx = r (w - xh mean(w xh)),  dg = sum over tokens and heads of dz xh
//
// The angle of pair i is position * inv_freq[i], formed in 64 bits and reduced to a fraction of a turn there, so that far
// positions keep their place on the circle; sine and cosine are computed once per token and pair and shared by the heads
// through LDS.  Sums and the arithmetic are fp32, with one rounding at the end.  HBM-bound: each row is read and written once.
//
// A head belongs to LPH lanes; a lane holds 8 pairs, a[8] and b[8]: of the rotated part, a chunk of the first half and the
// chunk of the second half that it is paired with, or (interleaved) 16 consecutive elements; of the part that is not
// rotated, 16 consecutive elements.  So every pair lies in one lane and all memory operations are chunks of 8 elements.
#include "rows.h"
#include <algorithm>

namespace axonn {

constexpr int QK_THREADS = 256;

struct QkArgs {
  int T, seq, heads, kv, d, rot;
  int items;                       // heads a token has work for: heads + kv, and the kv heads of V if they are copied
  int tokens;                      // of a workgroup's turn
  const elem_t *x, *dy;            // packed rows; upstream gradient (backward)
  elem_t* out;
  int64_t ld_x, ld_dy, ld_out;
  const elem_t *gamma_q, *gamma_k;
  float eps;
  const int* positions;
  const double* inv_freq;
  float* partial;                  // backward: [workgroups][2][d]
};

// What a lane holds of a head.
struct QkLane { int off_a, off_b, n_a, n_b, pair; };       // pair: first rotated pair, or -1
template <bool INTERLEAVED>
__device__ __forceinline__ QkLane qk_lane(int v, int d, int rot) {
  const int turned = (rot / 2 + 7) / 8;                     // lanes of the rotated part
  QkLane l;
  if (v < turned) {
    l.pair = 8 * v;
    l.off_a = INTERLEAVED ? 16 * v : 8 * v;
    l.off_b = INTERLEAVED ? 16 * v + 8 : rot / 2 + 8 * v;
    l.n_a = (INTERLEAVED ? rot : rot / 2) - l.off_a;
    l.n_b = rot - l.off_b;
  } else {
    l.pair = -1;
    l.off_a = rot + 16 * (v - turned);
    l.off_b = l.off_a + 8;
    l.n_a = d - l.off_a;
    l.n_b = d - l.off_b;
  }
  l.n_a = max(0, min(8, l.n_a));
  l.n_b = max(0, min(8, l.n_b));
  return l;
}

// (a, b) of the lane turned by its angles (c, s); INVERSE: back.
template <bool INTERLEAVED, bool INVERSE>
__device__ __forceinline__ void qk_turn(float (&a)[8], float (&b)[8], const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& p = INTERLEAVED ? (i < 4 ? a[2 * i] : b[2 * i - 8]) : a[i];
    float& q = INTERLEAVED ? (i < 4 ? a[2 * i + 1] : b[2 * i - 7]) : b[i];
    const float c = cs[i].x, s = INVERSE ? -cs[i].y : cs[i].y;
    const float np = p * c - q * s, nq = p * s + q * c;
    p = np;
    q = nq;
  }
}

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// cos and sin of the angles of `count` tokens from t0 on, [token][pairs], pairs = rot / 2 rounded up to whole chunks.
__device__ __forceinline__ void qk_angles(const QkArgs& g, int t0, int count, int pairs, float2* cs) {
  for (int i = threadIdx.x; i < count * pairs; i += QK_THREADS) {
    const int k = i / pairs, p = i - k * pairs, t = t0 + k;
    if (p >= g.rot / 2) continue;
    const int pos = g.positions ? g.positions[t] : t % g.seq;
    const double turns = (double)pos * (g.inv_freq[p] * 0.15915494309189533577);       // 1 / (2 pi)
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(c, s);
  }
}

template <int LPH, bool INTERLEAVED, bool BACKWARD>
__global__ __launch_bounds__(QK_THREADS) void qk_norm_rope_kernel(const QkArgs g) {
  extern __shared__ float2 qk_cs[];
  constexpr int GROUPS = QK_THREADS / LPH;
  const int group = threadIdx.x / LPH, v = threadIdx.x % LPH;
  const QkLane l = qk_lane<INTERLEAVED>(v, g.d, g.rot);
  const int pairs = (g.rot / 2 + 7) / 8 * 8;
  const float inv_d = 1.0f / (float)g.d;
  float gq[2][8], gk[2][8], sum_q[2][8], sum_k[2][8];
  {
    const elemx8 qa = load_chunk(g.gamma_q + l.off_a, l.n_a), qb = load_chunk(g.gamma_q + l.off_b, l.n_b);
    const elemx8 ka = load_chunk(g.gamma_k + l.off_a, l.n_a), kb = load_chunk(g.gamma_k + l.off_b, l.n_b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      gq[0][e] = (float)qa[e]; gq[1][e] = (float)qb[e];
      gk[0][e] = (float)ka[e]; gk[1][e] = (float)kb[e];
      sum_q[0][e] = sum_q[1][e] = sum_k[0][e] = sum_k[1][e] = 0.f;
    }
  }
  for (int t0 = blockIdx.x * g.tokens; t0 < g.T; t0 += gridDim.x * g.tokens) {
    const int count = min(g.tokens, g.T - t0);
    __syncthreads();
    qk_angles(g, t0, count, pairs, qk_cs);
    __syncthreads();
    for (int it = blockIdx.y * GROUPS + group; it < count * g.items; it += gridDim.y * GROUPS) {
      const int k = it / g.items, head = it - k * g.items;
      const int64_t t = t0 + k;
      const elem_t* src = (BACKWARD ? g.dy + t * g.ld_dy : g.x + t * g.ld_x) + (int64_t)head * g.d;
      elem_t* dst = g.out + t * g.ld_out + (int64_t)head * g.d;
      const elemx8 va = load_chunk(src + l.off_a, l.n_a), vb = load_chunk(src + l.off_b, l.n_b);
      if (head >= g.heads + g.kv) {                     // V
        store_chunk(dst + l.off_a, va, l.n_a);
        store_chunk(dst + l.off_b, vb, l.n_b);
        continue;
      }
      const bool is_q = head < g.heads;
      const float2* cs = qk_cs + k * pairs + l.pair;
      float a[8], b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { a[e] = (float)va[e]; b[e] = (float)vb[e]; }
      if constexpr (!BACKWARD) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sq += a[e] * a[e] + b[e] * b[e];
        const float r = rsqrtf(head_sum<LPH>(sq) * inv_d + g.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          a[e] *= r * (is_q ? gq[0][e] : gk[0][e]);
          b[e] *= r * (is_q ? gq[1][e] : gk[1][e]);
        }
        if (l.pair >= 0) qk_turn<INTERLEAVED, false>(a, b, cs);
      } else {
        const elem_t* xs = g.x + t * g.ld_x + (int64_t)head * g.d;
        const elemx8 xva = load_chunk(xs + l.off_a, l.n_a), xvb = load_chunk(xs + l.off_b, l.n_b);
        if (l.pair >= 0) qk_turn<INTERLEAVED, true>(a, b, cs);
        float sq = 0.f, dot = 0.f, xa[8], xb[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          xa[e] = (float)xva[e];
          xb[e] = (float)xvb[e];
          sq += xa[e] * xa[e] + xb[e] * xb[e];
          dot += a[e] * (is_q ? gq[0][e] : gk[0][e]) * xa[e] + b[e] * (is_q ? gq[1][e] : gk[1][e]) * xb[e];
        }
        const float r = rsqrtf(head_sum<LPH>(sq) * inv_d + g.eps);
        const float m = head_sum<LPH>(dot) * r * inv_d;                  // mean(w xh)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float ha = r * xa[e], hb = r * xb[e];
          if (is_q) { sum_q[0][e] += a[e] * ha; sum_q[1][e] += b[e] * hb; }
          else { sum_k[0][e] += a[e] * ha; sum_k[1][e] += b[e] * hb; }
          a[e] = r * (a[e] * (is_q ? gq[0][e] : gk[0][e]) - ha * m);
          b[e] = r * (b[e] * (is_q ? gq[1][e] : gk[1][e]) - hb * m);
        }
      }
      elemx8 oa, ob;
#pragma unroll
      for (int e = 0; e < 8; ++e) { oa[e] = (elem_t)a[e]; ob[e] = (elem_t)b[e]; }
      store_chunk(dst + l.off_a, oa, l.n_a);
      store_chunk(dst + l.off_b, ob, l.n_b);
    }
  }
  if constexpr (BACKWARD) {
    // the workgroup's sums of the gains' gradients: over its groups in order
    __shared__ float part[GROUPS][LPH * 16];
    float* const dst = g.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * g.d;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        part[group][v * 16 + e] = which ? sum_k[0][e] : sum_q[0][e];
        part[group][v * 16 + 8 + e] = which ? sum_k[1][e] : sum_q[1][e];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < LPH * 16; i += QK_THREADS) {
        const QkLane o = qk_lane<INTERLEAVED>(i / 16, g.d, g.rot);
        const int e = i % 16, col = e < 8 ? o.off_a + e : o.off_b + e - 8;
        if (e < 8 ? e >= o.n_a : e - 8 >= o.n_b) continue;
        float sum = 0.f;
        for (int q = 0; q < GROUPS; ++q) sum += part[q][i];
        dst[which * g.d + col] = sum;
      }
    }
  }
}

// dgamma_q[c], dgamma_k[c]: the workgroups' sums in order; 16 rows of 16 columns at a time.
__global__ __launch_bounds__(256) void qk_gain_sum_kernel(int blocks, int d, const float* __restrict__ partial, float* __restrict__ dgamma_q,
                                                          float* __restrict__ dgamma_k) {
  __shared__ float red[16][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
  float sum = 0.f;
  if (col < 2 * d)
    for (int r = r0; r < blocks; r += 16) sum += partial[(int64_t)r * 2 * d + col];
  red[r0][threadIdx.x & 15] = sum;
  __syncthreads();
  if (r0 == 0 && col < 2 * d) {
    float total = 0.f;
    for (int q = 0; q < 16; ++q) total += red[q][threadIdx.x];
    if (col < d) dgamma_q[col] = total;
    else dgamma_k[col - d] = total;
  }
}

struct QkPlan { int lph, tokens, grid_x, grid_y; };
static QkPlan qk_plan(int64_t T, int items, int d, int rot, bool backward) {
  QkPlan p;
  const int lanes = (rot / 2 + 7) / 8 + (d - rot + 15) / 16;
  p.lph = lanes <= 4 ? 4 : lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32;
  p.tokens = T >= 2048 ? 4 : 1;
  p.grid_x = (int)std::min<int64_t>((T + p.tokens - 1) / p.tokens, backward ? 512 : 1 << 20);
  p.grid_y = 1;
  return p;
}
// Rows of sums that the backward pass leaves, whatever the rotated part.
uint64_t qk_norm_rope_bwd_ws_bytes(int64_t T, int d) { return 8ull * (uint64_t)d * (uint64_t)std::min<int64_t>(T, 512); }

template <bool BACKWARD>
static hipError_t launch_qk(const QkArgs& g0, bool interleaved, hipStream_t s) {
  QkArgs g = g0;
  const QkPlan p = qk_plan(g.T, g.items, g.d, g.rot, BACKWARD);
  g.tokens = p.tokens;
  const size_t lds = (size_t)p.tokens * ((g.rot / 2 + 7) / 8 * 8) * sizeof(float2);
  auto launch = [&](auto lph) {
    constexpr int LPH = decltype(lph)::value;
    if (interleaved)
      hipLaunchKernelGGL(HIP_KERNEL_NAME(qk_norm_rope_kernel<LPH, true, BACKWARD>), dim3(p.grid_x, p.grid_y), dim3(QK_THREADS), lds, s, g);
    else
      hipLaunchKernelGGL(HIP_KERNEL_NAME(qk_norm_rope_kernel<LPH, false, BACKWARD>), dim3(p.grid_x, p.grid_y), dim3(QK_THREADS), lds, s, g);
  };
  if (p.lph == 4) launch(std::integral_constant<int, 4>{});
  else if (p.lph == 8) launch(std::integral_constant<int, 8>{});
  else if (p.lph == 16) launch(std::integral_constant<int, 16>{});
  else launch(std::integral_constant<int, 32>{});
  return hipGetLastError();
}

hipError_t launch_qk_norm_rope_fwd(const QkShape& q, const void* qkv, int64_t ld_qkv, const void* gamma_q, const void* gamma_k, float eps,
                                   const int* positions, const double* inv_freq, void* out, int64_t ld_out, hipStream_t s) {
  QkArgs g = {};
  g.T = (int)q.T; g.seq = q.seq; g.heads = q.heads; g.kv = q.kv; g.d = q.d; g.rot = q.rot;
  g.items = q.heads + q.kv + (out == qkv ? 0 : q.kv);
  g.x = (const elem_t*)qkv; g.out = (elem_t*)out; g.ld_x = ld_qkv; g.ld_out = ld_out;
  g.gamma_q = (const elem_t*)gamma_q; g.gamma_k = (const elem_t*)gamma_k; g.eps = eps;
  g.positions = positions; g.inv_freq = inv_freq;
  return launch_qk<false>(g, q.interleaved, s);
}

hipError_t launch_qk_norm_rope_bwd(const QkShape& q, const void* dout, int64_t ld_dout, const void* qkv, int64_t ld_qkv, const void* gamma_q,
                                   const void* gamma_k, float eps, const int* positions, const double* inv_freq, void* dqkv,
                                   int64_t ld_dqkv, float* dgamma_q, float* dgamma_k, float* workspace, hipStream_t s) {
  QkArgs g = {};
  g.T = (int)q.T; g.seq = q.seq; g.heads = q.heads; g.kv = q.kv; g.d = q.d; g.rot = q.rot;
  g.items = q.heads + q.kv + (dqkv == dout ? 0 : q.kv);
  g.x = (const elem_t*)qkv; g.dy = (const elem_t*)dout; g.out = (elem_t*)dqkv;
  g.ld_x = ld_qkv; g.ld_dy = ld_dout; g.ld_out = ld_dqkv;
  g.gamma_q = (const elem_t*)gamma_q; g.gamma_k = (const elem_t*)gamma_k; g.eps = eps;
  g.positions = positions; g.inv_freq = inv_freq;
  g.partial = workspace;
  hipError_t e = launch_qk<true>(g, q.interleaved, s);
  if (e != hipSuccess) return e;
  const QkPlan p = qk_plan(q.T, g.items, q.d, q.rot, true);
  hipLaunchKernelGGL(qk_gain_sum_kernel, dim3((2 * q.d + 15) / 16), dim3(256), 0, s, p.grid_x * p.grid_y, q.d, (const float*)workspace,
                     dgamma_q, dgamma_k);
  return hipGetLastError();
}

}  // namespace axonn
