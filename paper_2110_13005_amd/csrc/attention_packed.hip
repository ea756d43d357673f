// Causal attention inside sequences of different lengths that lie one behind the other in T rows, with n_kv key / value heads that
// groups of query heads share: forward and backward.  What a workgroup does for a tile of 128 rows is in attention_core.h; here are
// the plan, which says which tiles there are, and the kernels.
//
// Tiles begin at a sequence's first row and end with its last: a descriptor's range keeps what lies behind (another sequence, or
// rows that belong to none and may hold anything) from being read, so that infinities and NaN there reach no result, and from being
// written.  Every row of Q, K and V has one writer in the backward pass, too: a workgroup of the dK / dV kernel walks the query tiles of
// all heads that share its keys and keeps the sums in registers, so that there are no atomics and no partial sums in memory.
#include "attention_core.h"
#include "host_logic.h"

namespace axonn {

// ------------------------------------------------------------------------------------------------------------------- plan
// The tiles of all sequences, those with the most work first: tile t of a sequence walks t + 1 tiles of keys (forward, dQ), or as
// the t-th from the end t + 1 tiles of queries (dK / dV).  One list serves all kernels and layers that see the batch.
struct PlanItem { int start, len, tile, unused; };
struct PackedPlan { int n, unused[3]; PlanItem items[1]; };

int64_t packed_tiles_bound(int64_t T, int64_t n_seq) { return T / 128 + n_seq; }     // sum of ceil(len / 128)
uint64_t attention_packed_plan_size(int64_t T, int64_t n_seq) { return 16u + 16u * (uint64_t)packed_tiles_bound(T, n_seq); }

constexpr int PLAN_THREADS = 1024, PLAN_CLASSES = 4096;      // tiles from the last class on are not ordered among themselves

template <class Op>
__device__ __forceinline__ int plan_scan(int v, int* shared, int tid, Op op, int none) {      // inclusive, over the workgroup
  const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v = op(v, u);
  }
  __syncthreads();
  if (lane == 63) shared[wave] = v;
  __syncthreads();
  int front = none;
  for (int w = 0; w < wave; ++w) front = op(front, shared[w]);
  return op(front, v);
}

// One workgroup.  Offsets that do not ascend or leave [0, T] are taken as the largest so far inside it.  The list's order among tiles
// with the same work is left to the atomics: no result depends on it.
__global__ __launch_bounds__(PLAN_THREADS) void attn_packed_plan_kernel(int T, int n_seq, const int* __restrict__ offsets,
                                                                        PackedPlan* __restrict__ plan) {
  __shared__ int at[PLAN_CLASSES];         // sequences by their number of tiles; then where each class's next tile goes in the list
  __shared__ int scan[PLAN_THREADS / 64], deep;
  const int tid = threadIdx.x, lane = tid & 63;
  const auto larger = [](int a, int b) { return max(a, b); };
  const auto plus = [](int a, int b) { return a + b; };
  for (int i = tid; i < PLAN_CLASSES; i += PLAN_THREADS) at[i] = 0;
  if (tid == 0) deep = 0;
  const int per = (n_seq + PLAN_THREADS - 1) / PLAN_THREADS, first = tid * per;     // sequences of a thread
  const auto offset = [&](int i) { return min(max(offsets[i], 0), T); };
  int top = 0;
  for (int i = first; i < min(first + per, n_seq); ++i) top = max(top, offset(i));
  // a thread's sequences begin at the largest offset up to its first one's
  const int upto = plan_scan(top, scan, tid, larger, 0);
  int before = __shfl_up(upto, 1, 64);
  __syncthreads();
  if (lane == 63) scan[tid >> 6] = upto;
  __syncthreads();
  if (lane == 0) before = tid ? scan[(tid >> 6) - 1] : 0;

  int begin = before;
  for (int i = first; i < min(first + per, n_seq); ++i) {
    begin = max(begin, offset(i));
    const int tiles = (max(offset(i + 1) - begin, 0) + 127) / 128;
    if (tiles > 0) atomicAdd(&at[min(tiles, PLAN_CLASSES) - 1], 1);
    if (tiles > PLAN_CLASSES) atomicAdd(&deep, tiles - PLAN_CLASSES);
  }
  __syncthreads();
  // tiles of class c: of all sequences with more than c of them; their places: behind the classes above
  constexpr int CPT = PLAN_CLASSES / PLAN_THREADS;
  int n[CPT], sum = 0;
  const int base = PLAN_CLASSES - CPT * (tid + 1);          // thread 0 holds the highest classes
#pragma unroll
  for (int j = CPT - 1; j >= 0; --j) sum += n[j] = at[base + j];
  int above = plan_scan(sum, scan, tid, plus, 0) - sum;
  sum = 0;
#pragma unroll
  for (int j = CPT - 1; j >= 0; --j) {
    above += n[j];
    n[j] = above + (base + j == PLAN_CLASSES - 1 ? deep : 0);
    sum += n[j];
  }
  const int upto_here = plan_scan(sum, scan, tid, plus, 0);
  int place = upto_here - sum;
#pragma unroll
  for (int j = CPT - 1; j >= 0; --j) {
    at[base + j] = place;
    place += n[j];
  }
  if (tid == PLAN_THREADS - 1) plan->n = upto_here;
  __syncthreads();
  const int capacity = T / 128 + n_seq;
  const auto put = [&](int start, int len, int tile) {
    const int p = atomicAdd(&at[min(tile, PLAN_CLASSES - 1)], 1);
    if (p < capacity) plan->items[p] = PlanItem{start, len, tile, 0};
  };
  // a thread puts a sequence's first tiles, the wave together those of longer ones
  constexpr int ALONE = 4;
  begin = before;
  for (int e = 0; e < per; ++e) {
    const int i = first + e;
    int len = 0, tiles = 0;
    if (i < n_seq) {
      begin = max(begin, offset(i));
      len = max(offset(i + 1) - begin, 0);
      tiles = (len + 127) / 128;
    }
    for (int t = 0; t < min(tiles, ALONE); ++t) put(begin, len, t);
    unsigned long long more = __ballot(tiles > ALONE);
    while (more) {
      const int l = __ffsll(more) - 1;
      more &= more - 1;
      const int b = __shfl(begin, l, 64), m = __shfl(len, l, 64), k = __shfl(tiles, l, 64);
      for (int t = ALONE + lane; t < k; t += 64) put(b, m, t);
    }
  }
}

// --------------------------------------------------------------------------------------------------------------- kernels
struct PackedArgs {
  int T, heads, kv, group, d;
  float scale;
  uint32_t heads_recip, kv_recip, group_recip;       // reciprocals for the kernels' divisions
  const PackedPlan* plan;
  const elem_t* qkv;
  int64_t ld;
  elem_t* o;
  int64_t ld_o;
  float* lse;                                        // [heads][T], delta too
  const elem_t* dout;
  int64_t ld_do;
  float* delta;
  elem_t* dqkv;
  int64_t ld_dqkv;
};

struct PackedTile { int start, len, tile, unit; };
// Workgroup id -> item of the plan and unit (head) of it; false: there is no such tile.  A list that is not a plan of these rows makes
// no workgroup leave them.
__device__ __forceinline__ bool packed_tile(const PackedArgs& p, uint32_t id, uint32_t units, uint32_t recip, PackedTile& t) {
  const uint32_t i = host::recip_div(id, units, recip);
  if ((int)i >= p.plan->n) return false;
  const PlanItem it = p.plan->items[i];
  t = PackedTile{it.start, it.len, it.tile, (int)(id - i * units)};
  return it.start >= 0 && it.len > 0 && it.len <= p.T && it.start <= p.T - it.len && it.tile >= 0 && it.tile <= (it.len - 1) / 128;
}
// Workgroups are dealt round-robin to the 8 XCDs, each with an L2 of its own: the heads that share keys and values go to as few of
// them as there are heads for (a plan's item has `heads` workgroups, so the XCD is the unit modulo 8 if 8 divides them).
__device__ __forceinline__ int packed_head(const PackedArgs& p, int unit) {
  if (p.heads & 7) return unit;
  const int x = unit & 7, y = unit >> 3;
  if ((p.kv & 7) == 0) {
    const int k = host::recip_div(y, p.group, p.group_recip);
    return (x + 8 * k) * p.group + (y - k * p.group);
  }
  if (p.kv <= 4 && (p.kv & (p.kv - 1)) == 0) {
    const int per = 8 / p.kv;                        // XCDs of a key / value head
    return (x & (p.kv - 1)) * p.group + x / p.kv + per * y;
  }
  return unit;
}
struct PackedHead { const elem_t *q, *k, *v; int64_t row; int head, kv; };
__device__ __forceinline__ PackedHead packed_rows(const PackedArgs& p, int start, int head, int kv) {
  PackedHead h;
  h.row = start;
  h.head = head;
  h.kv = kv;
  const elem_t* row = p.qkv + h.row * p.ld;
  h.q = row + (int64_t)head * p.d;
  h.k = row + (int64_t)(p.heads + kv) * p.d;
  h.v = h.k + (int64_t)p.kv * p.d;
  return h;
}

template <int D>
__global__ __launch_bounds__(256, D > 128 ? 1 : 2) void attn_packed_fwd_kernel(PackedArgs p) {
  __shared__ FwdLds<D> lds;
  PackedTile t;
  if (!packed_tile(p, blockIdx.x, p.heads, p.heads_recip, t)) return;
  const int head = packed_head(p, t.unit);
  const PackedHead h = packed_rows(p, t.start, head, host::recip_div(head, p.group, p.group_recip));
  attn_fwd_tile<D, true>(lds, t.tile, t.len, p.d, p.scale, h.q, h.k, h.v, p.ld, p.o + h.row * p.ld_o + (int64_t)head * p.d, p.ld_o,
                         p.lse + (int64_t)head * p.T + h.row);
}

template <int D>
__device__ __forceinline__ void packed_dkdv(DkdvLds<D>& lds, const PackedArgs& p, uint32_t id) {
  PackedTile t;
  if (!packed_tile(p, id, p.kv, p.kv_recip, t)) return;
  const PackedHead h = packed_rows(p, t.start, t.unit * p.group, t.unit);
  const int64_t stat = (int64_t)h.head * p.T + h.row;
  elem_t* const dk = p.dqkv + h.row * p.ld_dqkv + (int64_t)(p.heads + h.kv) * p.d;
  attn_bwd_dkdv<D, true, true>(lds, (t.len - 1) / 128 - t.tile, t.len, p.d, p.scale, h.q, h.k, h.v, p.ld,
                               p.dout + h.row * p.ld_do + (int64_t)h.head * p.d, p.ld_do, p.lse + stat, p.delta + stat, dk,
                               dk + (int64_t)p.kv * p.d, p.ld_dqkv, p.group, p.T);
}
template <int D, bool FORM_DELTA>
__device__ __forceinline__ void packed_dq(DqLds<D>& lds, const PackedArgs& p, uint32_t id) {
  PackedTile t;
  if (!packed_tile(p, id, p.heads, p.heads_recip, t)) return;
  const int head = packed_head(p, t.unit);
  const PackedHead h = packed_rows(p, t.start, head, host::recip_div(head, p.group, p.group_recip));
  const int64_t stat = (int64_t)head * p.T + h.row, col = (int64_t)head * p.d;
  attn_bwd_dq<D, true, FORM_DELTA>(lds, t.tile, t.len, p.d, p.scale, h.q, h.k, h.v, p.ld, p.o + h.row * p.ld_o + col, p.ld_o,
                                   p.dout + h.row * p.ld_do + col, p.ld_do, p.lse + stat, p.delta + stat,
                                   p.dqkv + h.row * p.ld_dqkv + col, p.ld_dqkv, 0);
}
template <int D>
__global__ __launch_bounds__(256) void attn_packed_bwd_dkdv_kernel(PackedArgs p) {
  __shared__ DkdvLds<D> lds;
  packed_dkdv<D>(lds, p, blockIdx.x);
}
template <int D, bool FORM_DELTA>
__global__ __launch_bounds__(256, D > 128 ? 1 : 2) void attn_packed_bwd_dq_kernel(PackedArgs p) {
  __shared__ DqLds<D> lds;
  packed_dq<D, FORM_DELTA>(lds, p, blockIdx.x);
}
// Both at once, for problems whose tiles do not fill the chip: the first workgroups form dK and dV, the others dQ.
template <int D>
__global__ __launch_bounds__(256) void attn_packed_bwd_both_kernel(PackedArgs p, uint32_t n_dkdv) {
  __shared__ union { DkdvLds<D> dkdv; DqLds<D> dq; } lds;
  if (blockIdx.x < n_dkdv) packed_dkdv<D>(lds.dkdv, p, blockIdx.x);
  else packed_dq<D, false>(lds.dq, p, blockIdx.x - n_dkdv);
}

// delta[head][row] = sum over the head's columns of dO o: 16 lanes per (row, head), 4 elements per lane and step.
__global__ __launch_bounds__(256) void attn_packed_delta_kernel(PackedArgs p) {
  const int64_t pair = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int j = threadIdx.x & 15;
  const int64_t row = pair / p.heads;
  const int head = (int)(pair - row * p.heads);
  float sum = 0.f;
  if (row < p.T) {
    const elem_t* o = p.o + row * p.ld_o + (int64_t)head * p.d;
    const elem_t* dout = p.dout + row * p.ld_do + (int64_t)head * p.d;
    for (int c = 4 * j; c < p.d; c += 64)
      sum = delta_add<4, true>(sum, *reinterpret_cast<const elemx4*>(o + c), *reinterpret_cast<const elemx4*>(dout + c), 0);
  }
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
  if (row < p.T && j == 0) p.delta[(int64_t)head * p.T + row] = sum;
}

// ------------------------------------------------------------------------------------------------------------- launchers
hipError_t launch_attention_packed_plan(int64_t T, int64_t n_seq, const int* offsets, void* plan, hipStream_t st) {
  hipLaunchKernelGGL(attn_packed_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, (int)T, (int)n_seq, offsets, (PackedPlan*)plan);
  return hipGetLastError();
}

static PackedArgs packed_args(const PackedShape& s, const void* plan) {
  PackedArgs p = {};
  p.T = (int)s.T; p.heads = s.heads; p.kv = s.kv; p.group = s.heads / s.kv; p.d = s.d;
  p.scale = s.scale;
  p.heads_recip = host::recip_of(p.heads); p.kv_recip = host::recip_of(p.kv); p.group_recip = host::recip_of(p.group);
  p.plan = (const PackedPlan*)plan;
  return p;
}

hipError_t launch_attention_packed_fwd(const PackedShape& s, const void* plan, const void* qkv, int64_t ld, void* o, int64_t ld_o, float* lse,
                                       hipStream_t st) {
  PackedArgs p = packed_args(s, plan);
  p.qkv = (const elem_t*)qkv; p.ld = ld;
  p.o = (elem_t*)o; p.ld_o = ld_o; p.lse = lse;
  const dim3 grid((unsigned)(packed_tiles_bound(s.T, s.n_seq) * s.heads));
  if (s.d <= 64) hipLaunchKernelGGL(attn_packed_fwd_kernel<64>, grid, dim3(256), 0, st, p);
  else if (s.d <= 128) hipLaunchKernelGGL(attn_packed_fwd_kernel<128>, grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(attn_packed_fwd_kernel<192>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

uint64_t attention_packed_bwd_ws_bytes(const PackedShape& s) { return 4u * (uint64_t)s.T * (uint64_t)s.heads; }

hipError_t launch_attention_packed_bwd(const PackedShape& s, const void* plan, const void* qkv, int64_t ld, const void* o, int64_t ld_o,
                                       const float* lse, const void* dout, int64_t ld_do, void* dqkv, int64_t ld_dqkv, void* workspace,
                                       hipStream_t st) {
  PackedArgs p = packed_args(s, plan);
  p.qkv = (const elem_t*)qkv; p.ld = ld;
  p.o = (elem_t*)const_cast<void*>(o); p.ld_o = ld_o; p.lse = const_cast<float*>(lse);
  p.dout = (const elem_t*)dout; p.ld_do = ld_do;
  p.dqkv = (elem_t*)dqkv; p.ld_dqkv = ld_dqkv;
  p.delta = (float*)workspace;
  const int64_t tiles = packed_tiles_bound(s.T, s.n_seq);
  const unsigned n_dq = (unsigned)(tiles * s.heads), n_dkdv = (unsigned)(tiles * s.kv);
  const bool both = n_dq <= 256;
  if (both || (s.d != 64 && s.d != 128)) {
    hipLaunchKernelGGL(attn_packed_delta_kernel, dim3((unsigned)((s.T * s.heads + 15) / 16)), dim3(256), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (both) {
    const dim3 grid(n_dq + n_dkdv);
    if (s.d <= 64) hipLaunchKernelGGL(attn_packed_bwd_both_kernel<64>, grid, dim3(256), 0, st, p, n_dkdv);
    else if (s.d <= 128) hipLaunchKernelGGL(attn_packed_bwd_both_kernel<128>, grid, dim3(256), 0, st, p, n_dkdv);
    else hipLaunchKernelGGL(attn_packed_bwd_both_kernel<192>, grid, dim3(256), 0, st, p, n_dkdv);
    return hipGetLastError();
  }
  // where the dQ kernel forms delta it has to be the first
  if (s.d == 64) hipLaunchKernelGGL((attn_packed_bwd_dq_kernel<64, true>), dim3(n_dq), dim3(256), 0, st, p);
  else if (s.d < 64) hipLaunchKernelGGL((attn_packed_bwd_dq_kernel<64, false>), dim3(n_dq), dim3(256), 0, st, p);
  else if (s.d == 128) hipLaunchKernelGGL((attn_packed_bwd_dq_kernel<128, true>), dim3(n_dq), dim3(256), 0, st, p);
  else if (s.d < 128) hipLaunchKernelGGL((attn_packed_bwd_dq_kernel<128, false>), dim3(n_dq), dim3(256), 0, st, p);
  else hipLaunchKernelGGL((attn_packed_bwd_dq_kernel<192, false>), dim3(n_dq), dim3(256), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (s.d <= 64) hipLaunchKernelGGL(attn_packed_bwd_dkdv_kernel<64>, dim3(n_dkdv), dim3(256), 0, st, p);
  else if (s.d <= 128) hipLaunchKernelGGL(attn_packed_bwd_dkdv_kernel<128>, dim3(n_dkdv), dim3(256), 0, st, p);
  else hipLaunchKernelGGL(attn_packed_bwd_dkdv_kernel<192>, dim3(n_dkdv), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace axonn
