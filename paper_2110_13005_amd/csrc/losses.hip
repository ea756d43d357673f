// Losses over the logits of a vocabulary, beside the cross-entropy of lm_ends.hip: log-probabilities of given tokens with their gradient,
// the clipped policy loss, the preference loss of pairs of sequences, and distillation from a teacher's top logits.
//
// With q = softmax(z), every gradient is a multiple of q plus a few elements of its own:
//   d log q_t / dz = onehot_t - q
// A row's maximum and sum of exponentials come from one sweep with the running-maximum recurrence.  Tokens without a part are not read.
#include "rows.h"

namespace axonn {

constexpr int LOSS_THREADS = 256;

// exp(x c) of the difference of two logits; c = log2(e) / temperature.  (The difference is taken first: the product of a logit of
// the type's lowest value with c alone would be infinite.)
__device__ __forceinline__ float exp_scaled(float x, float c) { return __builtin_amdgcn_exp2f(x * c); }

template <int THREADS, class Op>
__device__ __forceinline__ float block_all(float v, float* shared, Op op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  v = shared[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = op(v, shared[w]);
  return v;
}
struct OpMax { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct OpSum { __device__ float operator()(float a, float b) const { return a + b; } };

// Maximum m of a row's logits and sum of exp((z - m) c) in all threads.
struct RowStats { float m, sum; };
// What exponentials are taken from: the maximum, or 0 where nothing but -inf (or NaN, which has to stay) has been seen.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void stats_add(RowStats& s, const elemx8& v, int n, float c) {
  const float old = s.m;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) top = fmaxf(top, (float)v[i]);
  s.m = fmaxf(s.m, top);
  const float m = reference(s.m);
  float part = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) part += exp_scaled((float)v[i] - m, c);
  s.sum = s.sum * exp_scaled(old - m, c) + part;
}
template <int THREADS>
__device__ __forceinline__ RowStats stats_join(RowStats s, float c, float* shared) {
  const float m = block_all<THREADS>(s.m, shared, OpMax());
  return RowStats{m, block_all<THREADS>(s.sum * exp_scaled(s.m - reference(m), c), shared, OpSum())};
}

constexpr float kLog2e_ = 1.4426950408889634f;

// dlogits[v] = slope (onehot_t - q) for the whole row; slope 0: zeros, and the row is not read.
__device__ __forceinline__ void write_gradient(const elem_t* row, elem_t* out, int V, int target, RowStats s, float slope, int tid) {
  const float f = -slope / s.sum;
  for (int c = tid * 8; c < V; c += LOSS_THREADS * 8) {
    elemx8 r = {};
    if (slope != 0.f) {
      const elemx8 v = load_chunk(row + c, V - c);
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = (elem_t)(exp_scaled((float)v[i] - s.m, kLog2e_) * f + (c + i == target ? slope : 0.f));
    }
    store_chunk(out + c, r, V - c);
  }
}

__global__ __launch_bounds__(LOSS_THREADS) void token_logprobs_fwd_kernel(int V, const elem_t* __restrict__ logits, int64_t ld,
                                                                          const int* __restrict__ targets, float* __restrict__ logp,
                                                                          float* __restrict__ lse) {
  __shared__ float shared[LOSS_THREADS / 64];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, target = targets[t];
  if (target < 0 || target >= V) {
    if (tid == 0) logp[t] = lse[t] = 0.f;
    return;
  }
  const elem_t* row = logits + t * ld;
  RowStats s{-INFINITY, 0.f};
  for (int c = tid * 8; c < V; c += LOSS_THREADS * 8) stats_add(s, load_chunk(row + c, V - c), V - c, kLog2e_);
  s = stats_join<LOSS_THREADS>(s, kLog2e_, shared);
  if (tid == 0) {
    const float log_sum = logf(s.sum);
    logp[t] = ((float)row[target] - s.m) - log_sum;
    lse[t] = s.m + log_sum;
  }
}

__global__ __launch_bounds__(LOSS_THREADS) void token_logprobs_bwd_kernel(int V, const elem_t* logits, int64_t ld,
                                                                          const int* __restrict__ targets, const float* __restrict__ lse,
                                                                          const float* __restrict__ dlogp, elem_t* dlogits, int64_t ld_d) {
  const int64_t t = blockIdx.x;
  const int target = targets[t];
  const float slope = target < 0 || target >= V ? 0.f : dlogp[t];
  write_gradient(logits + t * ld, dlogits + t * ld_d, V, target, RowStats{lse[t], 1.f}, slope, threadIdx.x);
}

// loss and its derivative by logp
__device__ __forceinline__ void policy_token(const PolicyArgs& p, float logp, float old_logp, float ref_logp, float A, float& loss, float& slope) {
  const float ratio = expf(logp - old_logp);
  // min(r A, clip(r) A): what is clipped depends on the sign of A
  const bool clipped = A >= 0.f ? ratio > p.clip_high : ratio < p.clip_low;
  loss = -A * (clipped ? (A >= 0.f ? p.clip_high : p.clip_low) : ratio);
  slope = clipped ? 0.f : -A * ratio;
  if (p.ref_logp) {
    const float d = ref_logp - logp, e = expm1f(d);
    loss += p.kl_coef * (e - d);
    slope -= p.kl_coef * e;
  }
}
__global__ __launch_bounds__(LOSS_THREADS) void policy_loss_kernel(PolicyArgs p) {
  __shared__ float shared[LOSS_THREADS / 64];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, V = p.V, target = p.targets[t];
  const float w = p.weight[t];
  elem_t* out = (elem_t*)p.dlogits + t * p.ld_d;
  if (target < 0 || target >= V || w == 0.f) {
    if (tid == 0) {
      p.token_loss[t] = 0.f;
      if (p.logp) p.logp[t] = 0.f;
    }
    if (p.dlogits) write_gradient(nullptr, out, V, 0, RowStats{0.f, 1.f}, 0.f, tid);
    return;
  }
  const elem_t* row = (const elem_t*)p.logits + t * p.ld;
  const float at_target = (float)row[target];
  RowStats s{-INFINITY, 0.f};
  for (int c = tid * 8; c < V; c += LOSS_THREADS * 8) stats_add(s, load_chunk(row + c, V - c), V - c, kLog2e_);
  s = stats_join<LOSS_THREADS>(s, kLog2e_, shared);
  const float logp = (at_target - s.m) - logf(s.sum);
  float loss, slope;
  policy_token(p, logp, p.old_logp[t], p.ref_logp ? p.ref_logp[t] : 0.f, p.advantage[t], loss, slope);
  if (tid == 0) {
    p.token_loss[t] = loss;
    if (p.logp) p.logp[t] = logp;
  }
  if (p.dlogits) write_gradient(row, out, V, target, s, slope * w * p.loss_scale, tid);
}

// One workgroup per pair; the one behind the last clears dlogp of the rows that belong to no sequence.  The sums are long and their
// difference is what counts: 64 bits.
__global__ __launch_bounds__(LOSS_THREADS) void preference_loss_kernel(PreferenceArgs p) {
  __shared__ double shared[2][LOSS_THREADS / 64];
  const int pair = blockIdx.x, tid = threadIdx.x, T = p.T;
  const auto offset = [&](int i) { return min(max(p.offsets[i], 0), T); };
  if (pair == p.n_pairs) {
    for (int t = tid; t < offset(0); t += LOSS_THREADS) p.dlogp[t] = 0.f;
    for (int t = offset(2 * p.n_pairs) + tid; t < T; t += LOSS_THREADS) p.dlogp[t] = 0.f;
    return;
  }
  const int a = offset(2 * pair), b = max(a, offset(2 * pair + 1)), e = max(b, offset(2 * pair + 2));
  const auto live = [&](int t) { return p.targets[t] >= 0 && p.targets[t] < p.V; };
  double chosen = 0.0, rejected = 0.0;
  for (int t = a + tid; t < e; t += LOSS_THREADS) {
    const double x = live(t) ? (double)p.logp[t] - (p.ref_logp ? (double)p.ref_logp[t] : 0.0) : 0.0;
    (t < b ? chosen : rejected) += x;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    chosen += __shfl_xor(chosen, o, 64);
    rejected += __shfl_xor(rejected, o, 64);
  }
  if ((tid & 63) == 0) { shared[0][tid >> 6] = chosen; shared[1][tid >> 6] = rejected; }
  __syncthreads();
  chosen = rejected = 0.0;
#pragma unroll
  for (int w = 0; w < LOSS_THREADS / 64; ++w) { chosen += shared[0][w]; rejected += shared[1][w]; }
  const float m = (float)((double)p.beta * (chosen - rejected));
  // -log sigma(m) = max(-m, 0) + log(1 + exp(-|m|))
  const float tail = log1pf(expf(-fabsf(m)));
  if (tid == 0) p.pair_loss[pair] = (1.f - p.smoothing) * (fmaxf(-m, 0.f) + tail) + p.smoothing * (fmaxf(m, 0.f) + tail);
  const float dm = p.smoothing / (1.f + expf(-m)) - (1.f - p.smoothing) / (1.f + expf(m));
  const float slope = p.scale * p.loss_scale * p.beta * dm;
  for (int t = a + tid; t < e; t += LOSS_THREADS) p.dlogp[t] = live(t) ? (t < b ? slope : -slope) : 0.f;
}

// The teacher's entries of a row; those without a token (an id outside the vocabulary) have id -1 and probability 0.
struct DistillRow {
  int id[kDistillMax];
  float p[kDistillMax];
};
__global__ __launch_bounds__(LOSS_THREADS) void distill_loss_kernel(DistillArgs a) {
  extern __shared__ uint32_t named[];                 // a bit per token of the vocabulary: the teacher has named it
  __shared__ DistillRow list;
  __shared__ float shared[LOSS_THREADS / 64];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, V = a.V, K = a.K;
  const float w = a.weight[t], c = a.log2e_by_temperature, per = 1.f / a.temperature;
  const elem_t* row = (const elem_t*)a.logits + t * a.ld;
  elem_t* out = (elem_t*)a.dlogits + t * a.ld_d;
  constexpr OpMax op_max;
  constexpr OpSum op_sum;
  int any = 0, twice = 0;
  float top = -INFINITY;
  if (w != 0.f) {
    for (int i = tid; i < (V + 31) / 32; i += LOSS_THREADS) named[i] = 0;
    __syncthreads();
    for (int j = tid; j < K; j += LOSS_THREADS) {
      int id = a.ids[t * a.ld_teacher + j];
      if (id < 0 || id >= V) id = -1;
      list.id[j] = id;
      if (id < 0) continue;
      any = 1;
      const uint32_t bit = 1u << (id & 31);
      if (atomicOr(&named[id >> 5], bit) & bit) twice = 1;
      top = fmaxf(top, a.teacher[t * a.ld_teacher + j]);
    }
    any = __syncthreads_or(any);
    twice = __syncthreads_or(twice);
  }
  if (!any) {
    if (tid == 0) a.token_loss[t] = 0.f;
    if (a.dlogits) write_gradient(nullptr, out, V, 0, RowStats{0.f, 1.f}, 0.f, tid);
    return;
  }
  // log p = (u - lse_u) of the teacher
  float lse_u;
  if (a.teacher_lse) {
    lse_u = a.teacher_lse[t];
  } else {
    top = block_all<LOSS_THREADS>(top, shared, op_max);
    float sum = 0.f;
    for (int j = tid; j < K; j += LOSS_THREADS)
      if (list.id[j] >= 0) sum += exp_scaled(a.teacher[t * a.ld_teacher + j] - top, c);
    lse_u = top * per + logf(block_all<LOSS_THREADS>(sum, shared, op_sum));
  }
  float mass = 0.f;
  for (int j = tid; j < K; j += LOSS_THREADS) {
    const float p = list.id[j] >= 0 ? expf(a.teacher[t * a.ld_teacher + j] * per - lse_u) : 0.f;
    list.p[j] = p;
    mass += p;
  }
  // the student: the named tokens, each once, and all others
  RowStats s{-INFINITY, 0.f}, r{-INFINITY, 0.f};
  __syncthreads();
  const auto first = [&](int j) {                     // of the entries with this token
    if (list.id[j] < 0) return false;
    if (twice)
      for (int i = 0; i < j; ++i)
        if (list.id[i] == list.id[j]) return false;
    return true;
  };
  for (int j = tid; j < K; j += LOSS_THREADS)
    if (first(j)) {
      elemx8 v;
      v[0] = row[list.id[j]];
      stats_add(s, v, 1, c);
    }
  for (int x = tid * 8; x < V; x += LOSS_THREADS * 8) {
    elemx8 v = load_chunk(row + x, V - x);
    const uint32_t bits = named[x >> 5] >> (x & 31) & 0xff;
    if (bits) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (bits >> i & 1) v[i] = (elem_t)-INFINITY;
    }
    stats_add(r, v, V - x, c);
  }
  s = stats_join<LOSS_THREADS>(s, c, shared);
  r = stats_join<LOSS_THREADS>(r, c, shared);
  const float m = fmaxf(s.m, r.m);
  const float others = r.m == -INFINITY ? 0.f : exp_scaled(r.m - m, c), all = s.sum * exp_scaled(s.m - m, c) + r.sum * others;
  const float log_all = logf(all);
  float loss = 0.f;
  for (int j = tid; j < K; j += LOSS_THREADS)
    if (list.p[j] != 0.f)
      loss += list.p[j] * ((a.teacher[t * a.ld_teacher + j] * per - lse_u) - (((float)row[list.id[j]] - m) * per - log_all));
  loss = block_all<LOSS_THREADS>(loss, shared, op_sum);
  float rest = 0.f;
  if (a.teacher_lse) {
    rest = 1.f - block_all<LOSS_THREADS>(mass, shared, op_sum);
    if (rest < 0.f) rest = 0.f;
    if (rest != 0.f) loss += rest * (logf(rest) - ((r.m - m) * per + logf(r.sum) - log_all));
  }
  if (tid == 0) a.token_loss[t] = loss;
  if (!a.dlogits) return;
  // q - p of the named tokens; of the others q (1 - P / Q), by the largest of them
  const float g = w * a.loss_scale * per, f = r.sum != 0.f ? g * (others / all - rest / r.sum) : 0.f, rm = reference(r.m);
  float mine[kDistillMax / LOSS_THREADS];
#pragma unroll
  for (int i = 0; i < kDistillMax / LOSS_THREADS; ++i) {
    const int j = tid + i * LOSS_THREADS;
    mine[i] = 0.f;
    if (j >= K || !first(j)) continue;
    float p = list.p[j];
    if (twice)
      for (int k = j + 1; k < K; ++k)
        if (list.id[k] == list.id[j]) p += list.p[k];
    mine[i] = g * (exp_scaled((float)row[list.id[j]] - m, c) / all - p);
  }
  __syncthreads();                                    // the row may be overwritten by its gradient
  for (int x = tid * 8; x < V; x += LOSS_THREADS * 8) {
    const elemx8 v = load_chunk(row + x, V - x);
    elemx8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (elem_t)(exp_scaled((float)v[i] - rm, c) * f);
    store_chunk(out + x, o, V - x);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kDistillMax / LOSS_THREADS; ++i) {
    const int j = tid + i * LOSS_THREADS;
    if (j < K && first(j)) out[list.id[j]] = (elem_t)mine[i];
  }
}

// out[0] = scale * sum of x[i] * (weight ? weight[i] : 1): one workgroup, fixed order, 64-bit sums.
__global__ __launch_bounds__(1024) void weighted_sum_kernel(int n, const float* __restrict__ x, const float* __restrict__ weight, float scale,
                                                            float* __restrict__ out) {
  __shared__ double shared[16];
  const int tid = threadIdx.x;
  double s = 0.0;
  for (int i = tid; i < n; i += 1024) {
    const float w = weight ? weight[i] : 1.f;
    if (w != 0.f) s += (double)x[i] * w;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((tid & 63) == 0) shared[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 16; ++w) s += shared[w];
    out[0] = (float)(s * scale);
  }
}

// ------------------------------------------------------------------------------------------------------------- launchers
static hipError_t launch_sum(int64_t n, const float* x, const float* weight, float scale, float* out, hipStream_t st) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !out) return e;
  hipLaunchKernelGGL(weighted_sum_kernel, dim3(1), dim3(1024), 0, st, (int)n, x, weight, scale, out);
  return hipGetLastError();
}

hipError_t launch_token_logprobs_fwd(int64_t T, int64_t V, const void* logits, int64_t ld, const int* targets, float* logp, float* lse,
                                     hipStream_t st) {
  hipLaunchKernelGGL(token_logprobs_fwd_kernel, dim3((unsigned)T), dim3(LOSS_THREADS), 0, st, (int)V, (const elem_t*)logits, ld, targets,
                     logp, lse);
  return hipGetLastError();
}
hipError_t launch_token_logprobs_bwd(int64_t T, int64_t V, const void* logits, int64_t ld, const int* targets, const float* lse,
                                     const float* dlogp, void* dlogits, int64_t ld_d, hipStream_t st) {
  hipLaunchKernelGGL(token_logprobs_bwd_kernel, dim3((unsigned)T), dim3(LOSS_THREADS), 0, st, (int)V, (const elem_t*)logits, ld, targets,
                     lse, dlogp, (elem_t*)dlogits, ld_d);
  return hipGetLastError();
}
hipError_t launch_policy_loss(int64_t T, const PolicyArgs& p, float* loss, hipStream_t st) {
  hipLaunchKernelGGL(policy_loss_kernel, dim3((unsigned)T), dim3(LOSS_THREADS), 0, st, p);
  return launch_sum(T, p.token_loss, p.weight, 1.f, loss, st);
}
hipError_t launch_preference_loss(const PreferenceArgs& p, float* loss, hipStream_t st) {
  hipLaunchKernelGGL(preference_loss_kernel, dim3((unsigned)p.n_pairs + 1), dim3(LOSS_THREADS), 0, st, p);
  return launch_sum(p.n_pairs, p.pair_loss, nullptr, p.scale, loss, st);
}
hipError_t launch_distill_loss(int64_t T, const DistillArgs& a, float* loss, hipStream_t st) {
  hipLaunchKernelGGL(distill_loss_kernel, dim3((unsigned)T), dim3(LOSS_THREADS), (unsigned)((a.V + 31) / 32 * 4), st, a);
  return launch_sum(T, a.token_loss, a.weight, 1.f, loss, st);
}

}  // namespace axonn
