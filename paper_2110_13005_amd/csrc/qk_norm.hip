// Norms of queries and keys for each head, with the position rotation in the same pass, on packed rows
// [heads * d | kv * d | kv * d] = [Q | K | V] (the layout attention reads), forward and backward.
//
//   r = 1 / sqrt(mean x^2 + eps),  xh = r x,  z = g xh,   (a, b) -> (a cos - b sin, a sin + b cos) for every rotated pair of z
//   backward: dz = the inverse rotation of dy,  w = g dz,  dx = r (w - xh mean(w xh)),  dg = sum over tokens and heads of dz xh
//
// The angle of pair i is position * inv_freq[i], formed in 64 bits and reduced to a fraction of a turn there, so that far
// positions keep their place on the circle; sine and cosine are computed once per token and pair and shared by the heads
// through LDS.  Sums and the arithmetic are fp32, with one rounding at the end.  HBM-bound: each row is read and written once;
// 8192 tokens x 40 query and 40 key heads of 128 forward in 96 to 105 us (503 MB, 4.8 to 5.2 TB/s), 4096 x (32, 8) backward in 29 to 32 us
// (143 MB, 4.9) and 4 for the gains' sums.
//
// A head belongs to LPH lanes; a lane holds 8 pairs, a[8] and b[8]: of the rotated part, a chunk of the first half and the
// chunk of the second half that it is paired with, or (interleaved) 16 consecutive elements; of the part that is not
// rotated, 16 consecutive elements.  So every pair lies in one lane and memory operations are chunks of 8 elements.
#include "rows.h"
#include "host_logic.h"
#include <algorithm>

namespace axonn {

constexpr int QK_THREADS = 256, QK_BACKWARD_BLOCKS = 768;

struct QkArgs {
  int T, seq, heads, kv, d, rot;
  int blocks_q;                    // workgroups of the query heads; the others take the key heads (and V)
  int copy_v;                      // not in place
  uint32_t recip_q, recip_k;       // reciprocals of heads and 2 * kv
  int tokens;                      // of a workgroup's turn
  const elem_t *x, *dy;            // packed rows; upstream gradient (backward)
  elem_t* out;
  int64_t ld_x, ld_dy, ld_out;
  const elem_t *gamma_q, *gamma_k;
  float eps;
  const int* positions;
  const double* inv_freq;
  float* partial;                  // backward: [workgroups][d]
};

// How the chunks of a head's parts (rotated halves or pairs, and what is not rotated) come out: all whole; the last one of a part
// shorter, and read as the part's last 8 elements (the ones that the chunk in front has as well are computed twice, to the same
// values, and counted once); or a part has fewer than 8 elements, which are read one by one.
enum QkChunks { QK_WHOLE, QK_OVERLAP, QK_SHORT };

// What a lane holds of a head: chunks at off_a and off_b of n_a and n_b elements (QK_SHORT: up to 8, else 8 or none), the first
// dup of which belong to another lane; first angles of their pairs, or -1.
struct QkLane { int off_a, off_b, n_a, n_b, dup_a, dup_b, pair_a, pair_b; };
template <bool INTERLEAVED, int CHUNKS>
__device__ __forceinline__ QkLane qk_lane(int v, int d, int rot) {
  const int turned = (rot / 2 + 7) / 8;                     // lanes of the rotated part
  const bool rotates = v < turned;
  QkLane l;
  int end_a, end_b;
  if (rotates && !INTERLEAVED) {
    l.off_a = 8 * v;
    l.off_b = rot / 2 + 8 * v;
    end_a = rot / 2;
    end_b = rot;
  } else {
    l.off_a = rotates ? 16 * v : rot + 16 * (v - turned);
    l.off_b = l.off_a + 8;
    end_a = end_b = rotates ? rot : d;
  }
  l.n_a = max(0, min(8, end_a - l.off_a));
  l.n_b = max(0, min(8, end_b - l.off_b));
  l.dup_a = l.dup_b = 0;
  if (CHUNKS == QK_OVERLAP) {
    if (l.n_a) { l.dup_a = 8 - l.n_a; l.off_a -= l.dup_a; l.n_a = 8; }
    if (l.n_b) { l.dup_b = 8 - l.n_b; l.off_b -= l.dup_b; l.n_b = 8; }
  }
  l.pair_a = rotates ? (INTERLEAVED ? l.off_a / 2 : l.off_a) : -1;
  l.pair_b = INTERLEAVED && l.n_b ? l.off_b / 2 : l.pair_a;
  return l;
}

// (a, b) of the lane turned by its angles; INVERSE: back.
template <bool INTERLEAVED, bool INVERSE>
__device__ __forceinline__ void qk_turn(float (&a)[8], float (&b)[8], const float2* cs, const QkLane& l) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& p = INTERLEAVED ? (i < 4 ? a[2 * i] : b[2 * i - 8]) : a[i];
    float& q = INTERLEAVED ? (i < 4 ? a[2 * i + 1] : b[2 * i - 7]) : b[i];
    const float2 t = cs[INTERLEAVED && i >= 4 ? l.pair_b + i - 4 : l.pair_a + i];
    const float c = t.x, s = INVERSE ? -t.y : t.y;
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

// Mean squares plus eps that 32 bits hold with room on both sides.  A head beyond them (bfloat16 values go to 2^128 and down to 2^-133,
// so their squares may overflow or vanish) is multiplied by 2^-70 or 2^70, which is exact, and with it eps by the square:
// x / sqrt(mean x^2 + eps) stays what it is.
constexpr float QK_LEAST = 0x1p-100f, QK_MOST = 0x1p100f;
__device__ __forceinline__ bool qk_out_of_range(float v) { return v < QK_LEAST || v > QK_MOST; }
__device__ __forceinline__ float qk_range_scale(float v) { return v > QK_MOST ? 0x1p-70f : v < QK_LEAST ? 0x1p70f : 1.f; }

// cos and sin of the angles of `count` tokens from t0 on, [token][pairs], pairs = rot / 2 rounded up to whole chunks.  The places behind
// rot / 2 are no pair's, but a lane with fewer than 8 pairs turns zeros by them, and those take part in the head's sums: they
// get no rotation, as what LDS holds may be an infinity or NaN.
__device__ __forceinline__ void qk_angles(const QkArgs& g, int t0, int count, int pairs, float2* cs) {
  for (int i = threadIdx.x; i < count * pairs; i += QK_THREADS) {
    const int k = i / pairs, p = i - k * pairs, t = t0 + k;
    if (p >= g.rot / 2) {
      cs[i] = make_float2(1.f, 0.f);
      continue;
    }
    const int pos = g.positions ? g.positions[t] : t % g.seq;
    const double turns = (double)pos * (g.inv_freq[p] * 0.15915494309189533577);       // 1 / (2 pi)
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(c, s);
  }
}

template <int CHUNKS>
__device__ __forceinline__ elemx8 qk_load(const elem_t* p, int n) {
  if (CHUNKS == QK_SHORT) return load_chunk(p, n);
  return n ? *reinterpret_cast<const elemx8_any*>(p) : elemx8{};
}
template <int CHUNKS>
__device__ __forceinline__ void qk_store(elem_t* p, const elemx8& v, int n) {
  if (CHUNKS == QK_SHORT) store_chunk(p, v, n);
  else if (n) *reinterpret_cast<elemx8_any*>(p) = v;
}

// A workgroup takes the query heads or the key heads (one gain, and backward one set of sums, in registers), the rows of
// the next head are on their way while one is worked on.
template <int LPH, bool INTERLEAVED, int CHUNKS, bool BACKWARD>
__global__ __launch_bounds__(QK_THREADS, BACKWARD ? 3 : 5) void qk_norm_rope_kernel(const QkArgs g) {
  extern __shared__ float2 qk_cs[];
  constexpr int GROUPS = QK_THREADS / LPH;
  const int group = threadIdx.x / LPH, v = threadIdx.x % LPH;
  const bool is_q = (int)blockIdx.x < g.blocks_q;
  const int block = is_q ? blockIdx.x : blockIdx.x - g.blocks_q, blocks = is_q ? g.blocks_q : gridDim.x - g.blocks_q;
  const int items = is_q ? g.heads : 2 * g.kv, normed = is_q ? g.heads : g.kv;
  const uint32_t recip = is_q ? g.recip_q : g.recip_k;
  const int64_t col0 = is_q ? 0 : (int64_t)g.heads * g.d;
  const QkLane l = qk_lane<INTERLEAVED, CHUNKS>(v, g.d, g.rot);
  auto mine_a = [&](int e) { return CHUNKS != QK_OVERLAP || e >= l.dup_a; };
  auto mine_b = [&](int e) { return CHUNKS != QK_OVERLAP || e >= l.dup_b; };
  const int pairs = (g.rot / 2 + 7) / 8 * 8;
  const float inv_d = 1.0f / (float)g.d;
  float gain[2][8], sum[2][8];
  {
    const elem_t* const gamma = is_q ? g.gamma_q : g.gamma_k;
    const elemx8 a = qk_load<CHUNKS>(gamma + l.off_a, l.n_a), b = qk_load<CHUNKS>(gamma + l.off_b, l.n_b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      gain[0][e] = (float)a[e];
      gain[1][e] = (float)b[e];
      sum[0][e] = sum[1][e] = 0.f;
    }
  }
  struct Item { elemx8 va, vb, xa, xb; int k, head; };
  for (int t0 = block * g.tokens; t0 < g.T; t0 += blocks * g.tokens) {
    const int count = min(g.tokens, g.T - t0), n = count * items;
    auto load = [&](Item& w, int it) {
      w.k = (int)host::recip_div((uint32_t)it, (uint32_t)items, recip);
      w.head = it - w.k * items;
      const int64_t t = t0 + w.k, at = col0 + (int64_t)w.head * g.d;
      if (w.head >= normed && !g.copy_v) return;
      const elem_t* const src = (BACKWARD ? g.dy + t * g.ld_dy : g.x + t * g.ld_x) + at;
      w.va = qk_load<CHUNKS>(src + l.off_a, l.n_a);
      w.vb = qk_load<CHUNKS>(src + l.off_b, l.n_b);
      if (BACKWARD && w.head < normed) {
        const elem_t* const xs = g.x + t * g.ld_x + at;
        w.xa = qk_load<CHUNKS>(xs + l.off_a, l.n_a);
        w.xb = qk_load<CHUNKS>(xs + l.off_b, l.n_b);
      }
    };
    Item next;
    if (group < n) load(next, group);
    __syncthreads();
    qk_angles(g, t0, count, pairs, qk_cs);
    __syncthreads();
    for (int it = group; it < n; it += GROUPS) {
      const Item w = next;
      if (it + GROUPS < n) load(next, it + GROUPS);
      elem_t* const dst = g.out + (int64_t)(t0 + w.k) * g.ld_out + col0 + (int64_t)w.head * g.d;
      if (w.head >= normed) {                           // V; in place it is passed over, so that the sums keep their order
        if (!g.copy_v) continue;
        qk_store<CHUNKS>(dst + l.off_a, w.va, l.n_a);
        qk_store<CHUNKS>(dst + l.off_b, w.vb, l.n_b);
        continue;
      }
      const float2* const cs = qk_cs + w.k * pairs;
      float a[8], b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { a[e] = (float)w.va[e]; b[e] = (float)w.vb[e]; }
      if constexpr (!BACKWARD) {
        auto mean_square = [&]() {
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sq += mine_a(e) ? a[e] * a[e] : 0.f;
            sq += mine_b(e) ? b[e] * b[e] : 0.f;
          }
          return head_sum<LPH>(sq) * inv_d;
        };
        float v = mean_square() + g.eps;
        if (__any(qk_out_of_range(v))) {                // (heads of the wave that are in range come out as before)
          const float s = qk_range_scale(v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            a[e] *= s;
            b[e] *= s;
          }
          v = mean_square() + g.eps * s * s;
        }
        const float r = rsqrtf(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          a[e] *= r * gain[0][e];
          b[e] *= r * gain[1][e];
        }
        if (l.pair_a >= 0) qk_turn<INTERLEAVED, false>(a, b, cs, l);
      } else {
        if (l.pair_a >= 0) qk_turn<INTERLEAVED, true>(a, b, cs, l);
        float xa[8], xb[8], s = 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) { xa[e] = (float)w.xa[e]; xb[e] = (float)w.xb[e]; }
        float sq, dot;
        auto sums = [&]() {
          sq = dot = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float ma = mine_a(e) ? xa[e] : 0.f, mb = mine_b(e) ? xb[e] : 0.f;
            sq += ma * ma + mb * mb;
            dot += a[e] * gain[0][e] * ma + b[e] * gain[1][e] * mb;
          }
          sq = head_sum<LPH>(sq) * inv_d;
        };
        sums();
        float v = sq + g.eps;
        if (__any(qk_out_of_range(v))) {
          s = qk_range_scale(v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            xa[e] *= s;
            xb[e] *= s;
          }
          sums();
          v = sq + g.eps * s * s;
        }
        const float r = rsqrtf(v), rs = r * s;          // of the multiplied head; of x
        const float m = head_sum<LPH>(dot) * r * inv_d;                  // mean(w xh)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float ha = r * xa[e], hb = r * xb[e];
          sum[0][e] += a[e] * ha;                       // (of elements that are another lane's as well: not looked at)
          sum[1][e] += b[e] * hb;
          a[e] = rs * (a[e] * gain[0][e] - ha * m);
          b[e] = rs * (b[e] * gain[1][e] - hb * m);
        }
      }
      elemx8 oa, ob;
#pragma unroll
      for (int e = 0; e < 8; ++e) { oa[e] = (elem_t)a[e]; ob[e] = (elem_t)b[e]; }
      qk_store<CHUNKS>(dst + l.off_a, oa, l.n_a);
      qk_store<CHUNKS>(dst + l.off_b, ob, l.n_b);
    }
  }
  if constexpr (BACKWARD) {
    // the workgroup's sums of the gain's gradient: over its groups in order
    __shared__ float part[GROUPS][LPH * 16];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      part[group][v * 16 + e] = sum[0][e];
      part[group][v * 16 + 8 + e] = sum[1][e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < LPH * 16; i += QK_THREADS) {
      const QkLane o = qk_lane<INTERLEAVED, CHUNKS>(i / 16, g.d, g.rot);
      const int e = i & 7, col = (i & 8 ? o.off_b : o.off_a) + e;
      if (e >= (i & 8 ? o.n_b : o.n_a) || e < (i & 8 ? o.dup_b : o.dup_a)) continue;
      float total = 0.f;
      for (int q = 0; q < GROUPS; ++q) total += part[q][i];
      g.partial[(int64_t)blockIdx.x * g.d + col] = total;
    }
  }
}

// dgamma_q (blockIdx.y = 0) and dgamma_k: the workgroups' sums in order, 16 columns and 64 rows of them at a time.
__global__ __launch_bounds__(1024) void qk_gain_sum_kernel(int blocks_q, int blocks_k, int d, const float* __restrict__ partial,
                                                           float* __restrict__ dgamma_q, float* __restrict__ dgamma_k) {
  __shared__ float red[64][17];
  const int c = threadIdx.x & 15, col = blockIdx.x * 16 + c, r0 = threadIdx.x >> 4;
  const float* const p = partial + (blockIdx.y ? (int64_t)blocks_q * d : 0);
  const int rows = blockIdx.y ? blocks_k : blocks_q;
  float sum = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int r = r0; r < rows; r += 64) sum += p[(int64_t)r * d + col];
  }
  red[r0][c] = sum;
  __syncthreads();
  if (r0 == 0 && col < d) {
    float total = 0.f;
#pragma unroll
    for (int q = 0; q < 64; ++q) total += red[q][c];
    (blockIdx.y ? dgamma_k : dgamma_q)[col] = total;
  }
}

struct QkPlan { int lph, tokens, blocks_q, blocks_k; };
static QkPlan qk_plan(int64_t T, int heads, int kv, int d, int rot, bool backward) {
  QkPlan p;
  const int lanes = (rot / 2 + 7) / 8 + (d - rot + 15) / 16;
  p.lph = lanes <= 4 ? 4 : lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32;
  // tokens of a turn: four rounds of heads for every group of lanes, while there are 512 turns.  Measured, us, 1 / 2 / 4 / 8 tokens:
  // 4096 x (32, 8 heads of 128) 28 / 22 / 20 / 20, 16384 x (16, 16 of 64) 75 / 49 / 41 / 39, 8192 x (40, 40 of 128)
  // 103 / 104 / 105 / 110, 512 x (16, 4 of 128) 7.0 / 5.4 / 5.5 / 7.1.
  p.tokens = 1;
  while (p.tokens < 8 && p.tokens * std::min(heads, 2 * kv) < 4 * QK_THREADS / p.lph && T >= (p.tokens == 1 ? 64 : 1024 * p.tokens)) p.tokens *= 2;
  const int64_t turns = (T + p.tokens - 1) / p.tokens;
  int64_t q = std::min<int64_t>(turns, 1 << 20), k = q; // a workgroup takes one turn after the other
  if (backward) {                                       // a row of sums per workgroup: shared out by the heads
    q = std::min<int64_t>(turns, std::max<int64_t>(1, (int64_t)QK_BACKWARD_BLOCKS * heads / (heads + 2 * kv)));
    k = std::min<int64_t>(turns, std::max<int64_t>(1, QK_BACKWARD_BLOCKS - q));
  }
  p.blocks_q = (int)q;
  p.blocks_k = (int)k;
  return p;
}
// Rows of sums that the backward pass leaves, whatever the heads and the rotated part.
uint64_t qk_norm_rope_bwd_ws_bytes(int64_t T, int d) { return 4ull * (uint64_t)d * (uint64_t)std::min<int64_t>(2 * T, QK_BACKWARD_BLOCKS + 1); }

template <bool BACKWARD>
static hipError_t launch_qk(QkArgs g, bool interleaved, const QkPlan& p, hipStream_t s) {
  g.tokens = p.tokens;
  g.blocks_q = p.blocks_q;
  g.recip_q = host::recip_of((uint32_t)g.heads);
  g.recip_k = host::recip_of(2u * (uint32_t)g.kv);
  const size_t lds = (size_t)p.tokens * ((g.rot / 2 + 7) / 8 * 8) * sizeof(float2);
  const dim3 grid((unsigned)(p.blocks_q + p.blocks_k));
  const int part = interleaved ? g.rot : g.rot / 2, rest = g.d - g.rot;
  auto launch_as = [&](auto lph, auto pairwise, auto chunks) {
    constexpr int LPH = decltype(lph)::value, CHUNKS = decltype(chunks)::value;
    constexpr bool PAIRWISE = decltype(pairwise)::value;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(qk_norm_rope_kernel<LPH, PAIRWISE, CHUNKS, BACKWARD>), grid, dim3(QK_THREADS), lds, s, g);
  };
  auto launch_chunks = [&](auto lph, auto pairwise) {
    if ((part > 0 && part < 8) || (rest > 0 && rest < 8)) launch_as(lph, pairwise, std::integral_constant<int, QK_SHORT>{});
    else if (part % 8 || rest % 8) launch_as(lph, pairwise, std::integral_constant<int, QK_OVERLAP>{});
    else launch_as(lph, pairwise, std::integral_constant<int, QK_WHOLE>{});
  };
  auto launch = [&](auto lph) {
    if (interleaved) launch_chunks(lph, std::true_type{});
    else launch_chunks(lph, std::false_type{});
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
  g.copy_v = out != qkv;
  g.x = (const elem_t*)qkv; g.out = (elem_t*)out; g.ld_x = ld_qkv; g.ld_out = ld_out;
  g.gamma_q = (const elem_t*)gamma_q; g.gamma_k = (const elem_t*)gamma_k; g.eps = eps;
  g.positions = positions; g.inv_freq = inv_freq;
  return launch_qk<false>(g, q.interleaved, qk_plan(q.T, q.heads, q.kv, q.d, q.rot, false), s);
}

hipError_t launch_qk_norm_rope_bwd(const QkShape& q, const void* dout, int64_t ld_dout, const void* qkv, int64_t ld_qkv, const void* gamma_q,
                                   const void* gamma_k, float eps, const int* positions, const double* inv_freq, void* dqkv,
                                   int64_t ld_dqkv, float* dgamma_q, float* dgamma_k, float* workspace, hipStream_t s) {
  QkArgs g = {};
  g.T = (int)q.T; g.seq = q.seq; g.heads = q.heads; g.kv = q.kv; g.d = q.d; g.rot = q.rot;
  g.copy_v = dqkv != dout;
  g.x = (const elem_t*)qkv; g.dy = (const elem_t*)dout; g.out = (elem_t*)dqkv;
  g.ld_x = ld_qkv; g.ld_dy = ld_dout; g.ld_out = ld_dqkv;
  g.gamma_q = (const elem_t*)gamma_q; g.gamma_k = (const elem_t*)gamma_k; g.eps = eps;
  g.positions = positions; g.inv_freq = inv_freq;
  g.partial = workspace;
  const QkPlan p = qk_plan(q.T, q.heads, q.kv, q.d, q.rot, true);
  const hipError_t e = launch_qk<true>(g, q.interleaved, p, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(qk_gain_sum_kernel, dim3((q.d + 15) / 16, 2), dim3(1024), 0, s, p.blocks_q, p.blocks_k, q.d, (const float*)workspace,
                     dgamma_q, dgamma_k);
  return hipGetLastError();
}

}  // namespace axonn
