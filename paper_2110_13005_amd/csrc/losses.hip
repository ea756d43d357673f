// Losses over the logits of a vocabulary, beside the cross-entropy of lm_ends.hip: log-probabilities of given tokens with their gradient,
// the clipped policy loss, the preference loss of pairs of sequences, and distillation from a teacher's top logits.
//
// With q = softmax(z), every gradient is a multiple of q plus a few elements of its own:
//   d log q_t / dz = onehot_t - q
// HBM-bound: a row of logits is read once and its gradient written once.  A workgroup holds the row in registers between the two (up to 131072
// columns; what lies behind them is read twice).  Tokens without a part are not read.
#include "rows.h"
#include "host_logic.h"
#include <type_traits>

namespace axonn {

constexpr float kLog2eLoss = 1.4426950408889634f;

struct OpMax {
  static constexpr float none = -INFINITY;
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct OpSum {
  static constexpr float none = 0.f;
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
// op over the 64 lanes of a wave, in all of them (a scalar): shifts inside rows of 16 lanes, then row 0 to 1 and 2 to 3, then the
// lower half to the upper one.  The data path of the vector unit, no LDS round trips.
template <class Op>
__device__ __forceinline__ float wave_all(float v, Op op) {
  const auto from = [&](auto ctrl, auto rows) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(Op::none), __float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value,
                                                       0xf, false));
  };
  using std::integral_constant;
  v = op(v, from(integral_constant<int, 0x111>(), integral_constant<int, 0xf>()));
  v = op(v, from(integral_constant<int, 0x112>(), integral_constant<int, 0xf>()));
  v = op(v, from(integral_constant<int, 0x114>(), integral_constant<int, 0xf>()));
  v = op(v, from(integral_constant<int, 0x118>(), integral_constant<int, 0xf>()));
  v = op(v, from(integral_constant<int, 0x142>(), integral_constant<int, 0xa>()));
  v = op(v, from(integral_constant<int, 0x143>(), integral_constant<int, 0xc>()));
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
// op over all threads of a workgroup, in all of them; `shared` is used for nothing else.
template <int THREADS, class Op>
__device__ __forceinline__ float block_all(float v, float (&shared)[THREADS / 64], Op op) {
  v = wave_all(v, op);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  return wave_all(lane < THREADS / 64 ? shared[lane] : Op::none, op);
}

// exp((z - m) / temperature) as exp2(z c - m c) with c = log2(e) / temperature: one fused multiply-add and one exponential.  m c is
// rounded; every exponential of the row is off by the same factor 2^low, which cancels in the softmax and is taken out of the
// logarithm of their sum.  |low| is |m c| 2^-24 at most: 2^low would leave 32 bits' range for a row whose maximum is a mask's value, or at a
// very low temperature.  From |m c| = 2^24 on any other 16-bit value lies 2^-11 |m| or more below m (bfloat16: 2^-8) and has the exponential 0
// whatever c of about that size it is formed with: the power of two below c, with which m c is exact; 2^-30 where even that comes near the
// largest number.
struct Exponent {
  float c, m, mc, low;
  // from the maximum m, the same in all lanes; of nothing but -inf (or NaN, which has to stay) from 0
  __device__ __forceinline__ Exponent(float m_, float c_) {
    m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(m_ == -INFINITY ? 0.f : m_)));
    const float size = fabsf(m) * c_;
    c = size < 0x1p24f ? c_ : size < 0x1p126f ? __uint_as_float(__float_as_uint(c_) & 0x7f800000u) : 0x1p-30f;
    mc = m * c;
    low = m == INFINITY ? 0.f : fmaf(m, c, -mc);
  }
  __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f(fmaf(z, c, -mc)); }
  // log of the sum of exp((z - m) / temperature) from the sum of these
  __device__ __forceinline__ float log_of(float sum) const { return logf(sum) - low * 0.6931471805599453f; }
};

// Maximum and sum of exponentials of a row, in all threads; `shared` for the two reductions.
template <int THREADS>
struct RowShared { float max[THREADS / 64], sum[THREADS / 64]; };
struct RowStats { Exponent e; float sum; };

// The chunk of a row that a lane takes as 16 bytes, or its last, shorter one; -inf behind the row (n <= 0: all of it).
__device__ __forceinline__ elemx8 logits_chunk(const elem_t* p, int n) {
  if (n >= 8) return *reinterpret_cast<const elemx8_any*>(p);
  elemx8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (elem_t)-INFINITY;
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) v[i] = p[i];
  return v;
}
// -inf for the elements whose bits are set
__device__ __forceinline__ void leave_out(elemx8& v, uint32_t bits) {
  if (bits == 0) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (bits >> i & 1) v[i] = (elem_t)-INFINITY;
}
__device__ __forceinline__ float chunk_max(float m, const elemx8& v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, (float)v[i]);
  return m;
}
// f times the exponentials of a chunk
__device__ __forceinline__ elemx8 chunk_gradient(const elemx8& v, const Exponent& e, float f) {
  elemx8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (elem_t)(e((float)v[i]) * f);
  return r;
}
// Chunk number `chunk` of a row: a base that is the same in all lanes and 32 bits of offset.
template <class T>
__device__ __forceinline__ T* chunk_of(T* row, uint32_t chunk) {
  return (T*)((char*)const_cast<elem_t*>(row) + chunk * 16u);
}

// A row of logits in the registers of a workgroup: thread t of THREADS holds chunks t, t + THREADS, ... of 8, as many as it takes
// (so all but the last, or the last two where there is no kernel for every number, are whole: the first WHOLE).
constexpr int row_waves(int chunks) { return chunks >= 1 && chunks <= 8 ? 8 : 4; }      // waves per SIMD that registers are shared among
constexpr int row_whole(int chunks) { return chunks <= 8 ? chunks - 1 : chunks - 2; }
template <int THREADS, int CHUNKS, int WHOLE = row_whole(CHUNKS)>
struct Row {
  elemx8 v[CHUNKS];
  __device__ __forceinline__ void load(const elem_t* row, int V, int tid) {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const uint32_t chunk = tid + j * THREADS;
      v[j] = logits_chunk(chunk_of(row, chunk), j < WHOLE ? 8 : V - 8 * (int)chunk);
    }
  }
  // The elements are converted anew in every sweep: kept converted they would take twice the registers.
  __device__ __forceinline__ void anew() {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) asm volatile("" : "+v"(v[j]));
  }
  // without the tokens whose bits are set
  __device__ __forceinline__ void without(const uint8_t* named, int V, int tid) {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const int chunk = tid + j * THREADS;
      if ((j < WHOLE) || 8 * chunk < V) leave_out(v[j], named[chunk]);
    }
  }
  __device__ __forceinline__ float sum(const Exponent& e) {
    anew();
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) part += e((float)v[j][i]);
      s += part;
    }
    return s;
  }
  __device__ __forceinline__ RowStats stats(float c, RowShared<THREADS>& shared) {
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) m = chunk_max(m, v[j]);
    const Exponent e(block_all<THREADS>(m, shared.max, OpMax()), c);
    return RowStats{e, block_all<THREADS>(sum(e), shared.sum, OpSum())};
  }
  // f times the exponentials
  __device__ __forceinline__ void store(elem_t* out, int V, int tid, const Exponent& e, float f) {
    anew();
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const uint32_t chunk = tid + j * THREADS;
      const int n = j < WHOLE ? 8 : V - 8 * (int)chunk;
      if (n > 0) store_chunk(chunk_of(out, chunk), chunk_gradient(v[j], e, f), n);
    }
  }
  // of one element more, by the thread that has stored its chunk
  __device__ __forceinline__ static void store_one(elem_t* out, int tid, int column, float value) {
    if (tid == (column >> 3) % THREADS) out[column] = (elem_t)value;
  }
};
// A row that is too long for them: what registers do not hold is read for the statistics, with the running-maximum recurrence, and once
// more for the gradient.
template <int THREADS>
struct Row<THREADS, 0, -1> {
  static constexpr int HEAD = 16, FIRST = 8 * THREADS * HEAD, AT_ONCE = 4;
  Row<THREADS, HEAD, HEAD> head;                      // columns up to FIRST; what follows is the rest's
  const elem_t* row;
  const uint8_t* named;
  int V, tid;
  __device__ __forceinline__ void load(const elem_t* row_, int V_, int tid_) {
    head.load(row_, V_, tid_);
    row = row_;
    V = V_;
    tid = tid_;
    named = nullptr;
  }
  __device__ __forceinline__ void without(const uint8_t* named_, int, int) {
    head.without(named_, V, tid);
    named = named_;
  }
  __device__ __forceinline__ void chunks(int first, elemx8 (&v)[AT_ONCE]) const {
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int at = first + 8 * j * THREADS;
      v[j] = logits_chunk(row + at, V - at);
    }
    if (named) {
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int at = first + 8 * j * THREADS;
        if (at < V) leave_out(v[j], named[at >> 3]);
      }
    }
  }
  __device__ __forceinline__ RowStats stats(float c, RowShared<THREADS>& shared) {
    float m = -INFINITY, sum = 0.f;
    for (int at = FIRST + 8 * tid; at < V; at += 8 * THREADS * AT_ONCE) {
      elemx8 v[AT_ONCE];
      chunks(at, v);
      const float old = m;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) m = chunk_max(m, v[j]);
      const float from = m == -INFINITY ? 0.f : m;
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) part += __builtin_amdgcn_exp2f(((float)v[j][i] - from) * c);
      sum = sum * __builtin_amdgcn_exp2f((old - from) * c) + part;
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < HEAD; ++j) top = chunk_max(top, head.v[j]);
    const Exponent e(block_all<THREADS>(top, shared.max, OpMax()), c);
    // the rest's sum is of exponentials without the common factor
    sum = head.sum(e) + sum * __builtin_amdgcn_exp2f((m - e.m) * c) * __builtin_amdgcn_exp2f(e.low);
    return RowStats{e, block_all<THREADS>(sum, shared.sum, OpSum())};
  }
  __device__ __forceinline__ void store(elem_t* out, int, int, const Exponent& e, float f) {
    head.store(out, V, tid, e, f);
    for (int first = FIRST + 8 * tid; first < V; first += 8 * THREADS * AT_ONCE) {
      elemx8 v[AT_ONCE];
      chunks(first, v);
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int at = first + 8 * j * THREADS;
        if (at >= V) continue;
        store_chunk(out + at, chunk_gradient(v[j], e, f), V - at);
      }
    }
  }
  __device__ __forceinline__ static void store_one(elem_t* out, int tid, int column, float value) {
    if (tid == (column >> 3) % THREADS) out[column] = (elem_t)value;
  }
};
template <int THREADS>
__device__ __forceinline__ void store_zeros(elem_t* out, int V, int tid) {
  const elemx8 zero = {};
  for (int c = tid * 8; c < V; c += THREADS * 8) store_chunk(out + c, zero, V - c);
}

// 2758 x 51200, 30 % of the tokens without a target: 198 MB in 40 us (4.9 TB/s), 59 where the caches still have to write back what the
// launch in front has left.
template <int THREADS, int CHUNKS>
__global__ __launch_bounds__(THREADS, row_waves(CHUNKS)) void token_logprobs_fwd_kernel(int V, const elem_t* __restrict__ logits, int64_t ld,
                                                                     const int* __restrict__ targets, float* __restrict__ logp,
                                                                     float* __restrict__ lse) {
  __shared__ RowShared<THREADS> shared;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, target = targets[t];
  if (target < 0 || target >= V) {
    if (tid == 0) logp[t] = lse[t] = 0.f;
    return;
  }
  Row<THREADS, CHUNKS> row;
  row.load(logits + t * ld, V, tid);
  const float at_target = (float)logits[t * ld + target];
  const RowStats s = row.stats(kLog2eLoss, shared);
  if (tid == 0) {
    const float log_sum = s.e.log_of(s.sum);
    logp[t] = (at_target - s.e.m) - log_sum;
    lse[t] = s.e.m + log_sum;
  }
}

// The log-sum-exp being there, rows need not be held whole: a workgroup takes so many chunks per thread of a row.  The same rows: 480 MB in 74
// us (6.5 TB/s, the caches still hold a part of the logits).
constexpr int GRAD_THREADS = 256;
// From here on a rounded log-sum-exp does not say what the softmax is: half a step of it is 2^-14 and more.  The row's first workgroup forms
// both from the logits, alone, so that it may be in place: 2758 x 51200 of such rows 212 us, 100 with lse (all tokens with a target).
constexpr float FAR_LSE = 1024.f;
__device__ __forceinline__ void far_row_gradient(int V, const elem_t* row, int target, float slope, elem_t* out, int tid) {
  __shared__ RowShared<GRAD_THREADS> shared;
  constexpr int STEP = 8 * GRAD_THREADS;
  float top = -INFINITY, sum = 0.f;
  for (int at = 8 * tid; at < V; at += STEP) top = chunk_max(top, logits_chunk(row + at, V - at));
  const Exponent e(block_all<GRAD_THREADS>(top, shared.max, OpMax()), kLog2eLoss);
  for (int at = 8 * tid; at < V; at += STEP) {
    const elemx8 v = logits_chunk(row + at, V - at);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += e((float)v[i]);
  }
  const float at_target = (float)row[target];
  sum = block_all<GRAD_THREADS>(sum, shared.sum, OpSum());       // (and the target's logit has been read)
  for (int at = 8 * tid; at < V; at += STEP) store_chunk(out + at, chunk_gradient(logits_chunk(row + at, V - at), e, -slope / sum), V - at);
  if (tid == (target >> 3) % GRAD_THREADS) out[target] = (elem_t)(slope * (1.f - e(at_target) / sum));
}
template <int CHUNKS>
__global__ __launch_bounds__(GRAD_THREADS) void token_logprobs_bwd_kernel(int V, uint32_t parts, uint32_t parts_recip, const elem_t* logits,
                                                                          int64_t ld, const int* __restrict__ targets,
                                                                          const float* __restrict__ lse, const float* __restrict__ dlogp,
                                                                          elem_t* dlogits, int64_t ld_d) {
  constexpr int COLUMNS = 8 * GRAD_THREADS * CHUNKS;
  const uint32_t t = host::recip_div(blockIdx.x, parts, parts_recip), first = (blockIdx.x - t * parts) * COLUMNS;
  const int target = targets[t], tid = threadIdx.x, n = min(V - (int)first, COLUMNS);
  const float slope = target < 0 || target >= V ? 0.f : dlogp[t];
  elem_t* const out = dlogits + t * ld_d + first;
  if (slope == 0.f) {
    store_zeros<GRAD_THREADS>(out, n, tid);
    return;
  }
  Row<GRAD_THREADS, CHUNKS, 0> row;
  row.load(logits + t * ld + first, n, tid);
  const float lse_t = lse[t];                         // on its way beside the row
  if (fabsf(lse_t) >= FAR_LSE) {
    if (first == 0) far_row_gradient(V, logits + t * ld, target, slope, out, tid);
    return;
  }
  const Exponent e(lse_t, kLog2eLoss);
  const bool here = target >= (int)first && target < (int)first + n;
  const float at_target = here ? (float)logits[t * ld + target] : 0.f;
  if (logits == dlogits) __syncthreads();             // read before it is overwritten
  // exp(z - lse) with the rounded product's factor taken out
  const float f = -slope * __builtin_amdgcn_exp2f(-e.low);
  row.store(out, n, tid, e, f);
  if (here) row.store_one(out, tid, target - (int)first, e(at_target) * f + slope);
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
// 4096 x 51200, a quarter of the tokens without a part: 734 MB in 141 us, 5.2 TB/s, what a copy of 1 GiB reaches; with two sweeps over the
// logits by workgroups of 256 204 us.
template <int THREADS, int CHUNKS>
__global__ __launch_bounds__(THREADS, row_waves(CHUNKS)) void policy_loss_kernel(PolicyArgs p) {
  __shared__ RowShared<THREADS> shared;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, V = p.V, target = p.targets[t];
  const float w = p.weight[t];
  elem_t* const out = (elem_t*)p.dlogits + t * p.ld_d;
  if (target < 0 || target >= V || w == 0.f) {
    if (tid == 0) {
      p.token_loss[t] = 0.f;
      if (p.logp) p.logp[t] = 0.f;
    }
    if (p.dlogits) store_zeros<THREADS>(out, V, tid);
    return;
  }
  const elem_t* const logits = (const elem_t*)p.logits + t * p.ld;
  Row<THREADS, CHUNKS> row;
  row.load(logits, V, tid);
  const float at_target = (float)logits[target], old_logp = p.old_logp[t], ref_logp = p.ref_logp ? p.ref_logp[t] : 0.f, A = p.advantage[t];
  const RowStats s = row.stats(kLog2eLoss, shared);
  const float logp = (at_target - s.e.m) - s.e.log_of(s.sum);
  float loss, slope;
  policy_token(p, logp, old_logp, ref_logp, A, loss, slope);
  if (tid == 0) {
    p.token_loss[t] = loss;
    if (p.logp) p.logp[t] = logp;
  }
  if (!p.dlogits) return;
  slope *= w * p.loss_scale;
  if (slope == 0.f) store_zeros<THREADS>(out, V, tid);
  else {
    row.store(out, V, tid, s.e, -slope / s.sum);
    row.store_one(out, tid, target, slope * (1.f - s.e(at_target) / s.sum));
  }
}

// Latency: 8 pairs in 2758 rows 4.8 us with a workgroup per pair (9 as one workgroup), 2 in 61 rows 3.2 as one, sum included.  The choice goes
// by the rows: many pairs of a few tokens are taken one after the other (1000 rows: 4 pairs 4.3 us, 32 6.0, 250 29.6; 250 in 1025 rows 6.6).
// The sums of a pair are long and their difference is what counts: 64 bits.  A wave takes a pair; with ALL the workgroup is the only one,
// takes the pairs in turn and leaves their sum, otherwise it is a pair's and its waves share the tokens.
constexpr int PREF_THREADS = 1024, PREF_ALONE = 1024;        // rows up to which one workgroup takes all pairs
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <bool ALL>
__global__ __launch_bounds__(PREF_THREADS) void preference_loss_kernel(PreferenceArgs p, float* __restrict__ loss) {
  constexpr int WAVES = PREF_THREADS / 64, STEP = ALL ? 64 : PREF_THREADS;
  __shared__ double shared[2][WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, T = p.T;
  const auto offset = [&](int i) { return min(max(p.offsets[i], 0), T); };
  // rows that belong to no sequence: by the workgroup behind the last pair's
  if (ALL || (int)blockIdx.x == p.n_pairs) {
    for (int t = tid; t < offset(0); t += PREF_THREADS) p.dlogp[t] = 0.f;
    for (int t = offset(2 * p.n_pairs) + tid; t < T; t += PREF_THREADS) p.dlogp[t] = 0.f;
    if (!ALL) return;
  }
  const auto live = [&](int t) { return p.targets[t] >= 0 && p.targets[t] < p.V; };
  double total = 0.0;
  for (int pair = ALL ? wave : blockIdx.x; pair < p.n_pairs; pair += ALL ? WAVES : p.n_pairs) {
    const int a = offset(2 * pair), b = max(a, offset(2 * pair + 1)), e = max(b, offset(2 * pair + 2)), first = a + (ALL ? lane : tid);
    double chosen = 0.0, rejected = 0.0;
    for (int t = first; t < e; t += STEP) {
      const float logp = p.logp[t], ref = p.ref_logp ? p.ref_logp[t] : 0.f;
      const double x = live(t) ? (double)logp - (double)ref : 0.0;
      (t < b ? chosen : rejected) += x;
    }
    chosen = wave_sum64(chosen);
    rejected = wave_sum64(rejected);
    if (!ALL) {
      if (lane == 0) { shared[0][wave] = chosen; shared[1][wave] = rejected; }
      __syncthreads();
      chosen = wave_sum64(lane < WAVES ? shared[0][lane] : 0.0);
      rejected = wave_sum64(lane < WAVES ? shared[1][lane] : 0.0);
    }
    const float m = (float)((double)p.beta * (chosen - rejected));
    // -log sigma(m) = max(-m, 0) + log(1 + exp(-|m|)); without a share an infinite one (a token of probability 0) has no part
    const float tail = log1pf(expf(-fabsf(m))), miss = 1.f - p.smoothing;
    const float value = (miss > 0.f ? miss * (fmaxf(-m, 0.f) + tail) : 0.f) + (p.smoothing > 0.f ? p.smoothing * (fmaxf(m, 0.f) + tail) : 0.f);
    if ((ALL ? lane : tid) == 0) p.pair_loss[pair] = value;
    total += value;
    const float dm = p.smoothing / (1.f + expf(-m)) - miss / (1.f + expf(m));
    const float slope = p.scale * p.loss_scale * p.beta * dm;
    for (int t = first; t < e; t += STEP) p.dlogp[t] = live(t) ? (t < b ? slope : -slope) : 0.f;
  }
  if (!ALL || !loss) return;
  if (lane == 0) shared[0][wave] = total;
  __syncthreads();
  if (wave == 0) {
    total = wave_sum64(lane < WAVES ? shared[0][lane] : 0.0);
    if (lane == 0) loss[0] = (float)(total * p.scale);
  }
}

// What the first wave, which takes the teacher's entries of a row, tells the others.
struct DistillList {
  int id[kDistillMax];                     // -1: no token
  float p[kDistillMax], z[kDistillMax];    // the teacher's logit / temperature, then its probability; the student's logit
  int any;                                 // a token is named at all
  float mass;                              // sum of p
  float top, sum;                          // of the named tokens' logits, each once: maximum; sum of exp((z - top) / temperature)
  float gain;                              // sum of p (log p - (z - top) / temperature)
};
// sum + w (distance * per + more), w_per = w * per: a mask's distance may pass the largest number with its factor, but not with both.
__device__ __forceinline__ float add_weighted(float sum, float w, float w_per, float distance, float more) {
  return fmaf(distance, w_per, fmaf(w, more, sum));
}
// id, u: the lane's first entry, if it has one
__device__ __forceinline__ void distill_list(const DistillArgs& a, int64_t t, const elem_t* row, uint32_t* named, DistillList& l, int lane, int id,
                                             float u, int& twice) {
  const int K = a.K;
  const float c = a.log2e_by_temperature, per = 1.f / a.temperature;
  constexpr OpMax op_max;
  constexpr OpSum op_sum;
  int any = 0;
  twice = 0;
  float top_u = -INFINITY, top = -INFINITY;
  for (int j = lane; j < K; j += 64) {
    if (j >= 64) {
      id = a.ids[t * a.ld_teacher + j];
      u = a.teacher[t * a.ld_teacher + j];
    }
    if (id < 0 || id >= a.V) id = -1;
    l.id[j] = id;
    if (id < 0) continue;
    any = 1;
    const float z = (float)row[id];
    const uint32_t bit = 1u << (id & 31);
    if (atomicOr(&named[id >> 5], bit) & bit) twice = 1;
    l.z[j] = z;
    l.p[j] = u *= per;
    top_u = fmaxf(top_u, u);
    top = fmaxf(top, z);
  }
  any = __any(any);
  twice = __any(twice);
  if (lane == 0) l.any = any;
  if (!any) return;
  // log p = (u - lse_u) of the teacher
  float lse_u;
  if (a.teacher_lse) {
    lse_u = a.teacher_lse[t];
  } else {
    top_u = wave_all(top_u, op_max);
    float sum = 0.f;
    for (int j = lane; j < K; j += 64)
      if (l.id[j] >= 0) sum += __builtin_amdgcn_exp2f((l.p[j] - top_u) * kLog2eLoss);
    lse_u = top_u + logf(wave_all(sum, op_sum));
  }
  top = wave_all(top, op_max);
  const float from = top == -INFINITY ? 0.f : top;
  float mass = 0.f, gain = 0.f, sum = 0.f;
  for (int j = lane; j < K; j += 64) {
    const int id = l.id[j];
    if (id < 0) continue;
    const float z = l.z[j], logp = l.p[j] - lse_u, p = expf(logp);
    l.p[j] = p;
    mass += p;
    const float p_per = p * per;
    if (p_per != 0.f) gain = add_weighted(gain, p, p_per, from - z, logp);
    bool first = true;
    if (twice)
      for (int i = 0; i < j; ++i) first &= l.id[i] != id;
    if (first) sum += __builtin_amdgcn_exp2f((z - from) * c);
  }
  mass = wave_all(mass, op_sum);
  gain = wave_all(gain, op_sum);
  sum = wave_all(sum, op_sum);
  if (lane == 0) { l.mass = mass; l.gain = gain; l.sum = sum; l.top = from; }
}

// 4096 x 51200, 64 entries, a tenth of the tokens without a part: 799 MB in 158 us (5.05 TB/s); 254 with two sweeps and all threads on the
// entries.  333 x 32003: 18 us, one round of workgroups, which is the time of a row from its first load to its last store.
template <int THREADS, int CHUNKS>
__global__ __launch_bounds__(THREADS, row_waves(CHUNKS)) void distill_loss_kernel(DistillArgs a) {
  extern __shared__ uint32_t named[];                 // a bit per token of the vocabulary: the teacher has named it
  __shared__ DistillList list;
  __shared__ RowShared<THREADS> shared;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, V = a.V, K = a.K;
  const float w = a.weight[t], c = a.log2e_by_temperature, per = 1.f / a.temperature;
  const elem_t* const logits = (const elem_t*)a.logits + t * a.ld;
  elem_t* const out = (elem_t*)a.dlogits + t * a.ld_d;
  if (w == 0.f) {
    if (tid == 0) a.token_loss[t] = 0.f;
    if (a.dlogits) store_zeros<THREADS>(out, V, tid);
    return;
  }
  // the entries are on their way in front of the row
  int id = -1, twice = 0;
  float u = 0.f;
  if (tid < 64 && tid < K) {
    id = a.ids[t * a.ld_teacher + tid];
    u = a.teacher[t * a.ld_teacher + tid];
  }
  Row<THREADS, CHUNKS> row;
  row.load(logits, V, tid);
  for (int i = tid; i < (V + 31) / 32; i += THREADS) named[i] = 0;
  __syncthreads();
  if (tid < 64) distill_list(a, t, logits, named, list, tid, id, u, twice);
  __syncthreads();
  if (!list.any) {
    if (tid == 0) a.token_loss[t] = 0.f;
    if (a.dlogits) store_zeros<THREADS>(out, V, tid);
    return;
  }
  // the student's distribution: the tokens that are not named, and with them those that are
  row.without((const uint8_t*)named, V, tid);
  const RowStats r = row.stats(c, shared);
  const float r_sum = r.sum * __builtin_amdgcn_exp2f(-r.e.low);
  const float m = list.sum == 0.f ? r.e.m : r_sum > 0.f ? fmaxf(list.top, r.e.m) : list.top;
  const float top = list.sum == 0.f ? m : list.top;   // (of named tokens that are all masked there is none)
  const float others = __builtin_amdgcn_exp2f((r.e.m - m) * c), all = list.sum * __builtin_amdgcn_exp2f((top - m) * c) + (r_sum > 0.f ? r_sum * others : r_sum);
  const float log_all = logf(all);
  // The others' mass is an outcome of its own, if it has one and the student has other tokens (if not, what 1 - mass is may be its rounding,
  // which would count infinitely); total: the mass of all outcomes, 1 with that one.
  float loss = add_weighted(list.gain, list.mass, list.mass * per, m - top, log_all), rest = 0.f, total = 1.f;
  if (a.teacher_lse) {
    rest = r_sum == 0.f ? 0.f : 1.f - list.mass;
    if (rest < 0.f) rest = 0.f;
    if (rest != 0.f) loss = add_weighted(loss, rest, rest * per, m - r.e.m, logf(rest) - (logf(r_sum) - log_all));
    else total = list.mass;
  }
  if (tid == 0) a.token_loss[t] = loss;
  if (!a.dlogits) return;
  // q total - p of the named tokens; of the others q (total - P / Q)
  const float g = w * a.loss_scale * per;
  const float f = r_sum == 0.f ? 0.f : g * (total * others / all - rest / r_sum) * __builtin_amdgcn_exp2f(-r.e.low);
  row.store(out, V, tid, r.e, f);
  __syncthreads();
  if (tid >= 64) return;
  for (int j = tid; j < K; j += 64) {
    const int id = list.id[j];
    if (id < 0) continue;
    float p = list.p[j];
    bool first = true;
    if (twice) {
      for (int i = 0; i < j; ++i) first &= list.id[i] != id;
      for (int i = j + 1; i < K; ++i)
        if (list.id[i] == id) p += list.p[i];
    }
    if (first) out[id] = (elem_t)(g * (total * __builtin_amdgcn_exp2f((list.z[j] - m) * c) / all - p));
  }
}

// out[0] = scale * sum of x[i] * (weight ? weight[i] : 1): one workgroup, fixed order, 64-bit sums.  Losses of 0 add nothing, whatever
// their weight is: they are also those of tokens that have no part.
__global__ __launch_bounds__(1024) void weighted_sum_kernel(int n, const float* __restrict__ x, const float* __restrict__ weight, float scale,
                                                            float* __restrict__ out) {
  __shared__ double shared[16];
  const int tid = threadIdx.x;
  double s = 0.0;
  for (int i = tid; i < n; i += 8 * 1024) {
    float v[8], w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = min(i + j * 1024, n - 1);
      v[j] = x[at];
      w[j] = weight ? weight[at] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j * 1024 < n && v[j] != 0.f) s += (double)v[j] * w[j];
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

// Workgroups of 256 threads up to 8192 columns, 512 up to 16384 and 1024 above, with as many chunks per thread as a row has: up to 8, two
// thousand threads on a CU; up to 16, half of them.  What lies behind 131072 columns is read twice.  Policy loss, us, in GB/s of a read and
// a written row: 8192 x 8200 with 512 threads 59 (4550), 1024 84; 8192 x 24576 512 155, 1024 147 (5480); 2048 x 131072 in registers 228
// (4710), read twice 251; 1024 x 262144 half of it in registers 275 (3900), all read twice 296.
#define AXONN_ROW_CASE(KERNEL, THREADS, CHUNKS, LDS, ...)                                                                     \
  case THREADS * 100 + CHUNKS: hipLaunchKernelGGL((KERNEL<THREADS, CHUNKS>), dim3((unsigned)T), dim3(THREADS), LDS, st, __VA_ARGS__); break
#define AXONN_ROW_DISPATCH(KERNEL, LDS, ...)                                                                              \
  switch (row_kernel(V)) {                                                                                                \
    AXONN_ROW_CASE(KERNEL, 256, 1, LDS, __VA_ARGS__);  AXONN_ROW_CASE(KERNEL, 256, 2, LDS, __VA_ARGS__);                  \
    AXONN_ROW_CASE(KERNEL, 256, 3, LDS, __VA_ARGS__);  AXONN_ROW_CASE(KERNEL, 256, 4, LDS, __VA_ARGS__);                  \
    AXONN_ROW_CASE(KERNEL, 512, 3, LDS, __VA_ARGS__);  AXONN_ROW_CASE(KERNEL, 512, 4, LDS, __VA_ARGS__);                  \
    AXONN_ROW_CASE(KERNEL, 1024, 3, LDS, __VA_ARGS__); AXONN_ROW_CASE(KERNEL, 1024, 4, LDS, __VA_ARGS__);                 \
    AXONN_ROW_CASE(KERNEL, 1024, 5, LDS, __VA_ARGS__); AXONN_ROW_CASE(KERNEL, 1024, 6, LDS, __VA_ARGS__);                 \
    AXONN_ROW_CASE(KERNEL, 1024, 7, LDS, __VA_ARGS__); AXONN_ROW_CASE(KERNEL, 1024, 8, LDS, __VA_ARGS__);                 \
    AXONN_ROW_CASE(KERNEL, 1024, 10, LDS, __VA_ARGS__); AXONN_ROW_CASE(KERNEL, 1024, 12, LDS, __VA_ARGS__);               \
    AXONN_ROW_CASE(KERNEL, 1024, 14, LDS, __VA_ARGS__); AXONN_ROW_CASE(KERNEL, 1024, 16, LDS, __VA_ARGS__);               \
    default: hipLaunchKernelGGL((KERNEL<1024, 0>), dim3((unsigned)T), dim3(1024), LDS, st, __VA_ARGS__);                  \
  }
static int row_kernel(int64_t V) {
  const int threads = V <= 8192 ? 256 : V <= 16384 ? 512 : 1024, chunks = (int)((V + 8 * threads - 1) / (8 * threads));
  return chunks <= 8 ? threads * 100 + chunks : chunks <= 16 ? threads * 100 + (chunks + 1) / 2 * 2 : 0;
}

hipError_t launch_token_logprobs_fwd(int64_t T, int64_t V, const void* logits, int64_t ld, const int* targets, float* logp, float* lse,
                                     hipStream_t st) {
  AXONN_ROW_DISPATCH(token_logprobs_fwd_kernel, 0, (int)V, (const elem_t*)logits, ld, targets, logp, lse);
  return hipGetLastError();
}
hipError_t launch_token_logprobs_bwd(int64_t T, int64_t V, const void* logits, int64_t ld, const int* targets, const float* lse,
                                     const float* dlogp, void* dlogits, int64_t ld_d, hipStream_t st) {
#define AXONN_GRADIENT(CHUNKS)                                                                                                  \
  do {                                                                                                                     \
    const uint32_t parts = (uint32_t)((V + 8 * GRAD_THREADS * CHUNKS - 1) / (8 * GRAD_THREADS * CHUNKS));                  \
    hipLaunchKernelGGL(token_logprobs_bwd_kernel<CHUNKS>, dim3((unsigned)T * parts), dim3(GRAD_THREADS), 0, st, (int)V, parts,   \
                       host::recip_of(parts), (const elem_t*)logits, ld, targets, lse, dlogp, (elem_t*)dlogits, ld_d);     \
  } while (0)
  // (a shorter kernel for short rows: 61 x 2000 2.6 us, 3.9 with the other one)
  if (V <= 8 * GRAD_THREADS) AXONN_GRADIENT(1);
  else AXONN_GRADIENT(4);
#undef AXONN_GRADIENT
  return hipGetLastError();
}
hipError_t launch_policy_loss(int64_t T, const PolicyArgs& p, float* loss, hipStream_t st) {
  const int64_t V = p.V;
  AXONN_ROW_DISPATCH(policy_loss_kernel, 0, p);
  return launch_sum(T, p.token_loss, p.weight, 1.f, loss, st);
}
hipError_t launch_preference_loss(const PreferenceArgs& p, float* loss, hipStream_t st) {
  if (p.T <= PREF_ALONE) {
    hipLaunchKernelGGL(preference_loss_kernel<true>, dim3(1), dim3(PREF_THREADS), 0, st, p, loss);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(preference_loss_kernel<false>, dim3((unsigned)p.n_pairs + 1), dim3(PREF_THREADS), 0, st, p, nullptr);
  return launch_sum(p.n_pairs, p.pair_loss, nullptr, p.scale, loss, st);
}
hipError_t launch_distill_loss(int64_t T, const DistillArgs& a, float* loss, hipStream_t st) {
  const int64_t V = a.V;
  AXONN_ROW_DISPATCH(distill_loss_kernel, (unsigned)((V + 31) / 32 * 4), a);
  return launch_sum(T, a.token_loss, a.weight, 1.f, loss, st);
}
#undef AXONN_ROW_DISPATCH
#undef AXONN_ROW_CASE

}  // namespace axonn
