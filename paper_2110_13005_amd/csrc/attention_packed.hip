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

// Offsets that do not ascend or leave [0, T] are taken as the largest so far inside it, in both kernels.
//
// Few sequences: every wave holds them all, a lane SEQS of them, and lists the tiles of one range of classes by itself: how many tiles
// lie in the classes above is a sum over the sequences, a tile's place among its class a count of the lanes in front.  No barriers; 15
// documents in 8192 rows in 2.9 us (by the other kernel 6.1).
constexpr int PLAN_FEW = 256;
template <int SEQS>
__global__ __launch_bounds__(PLAN_THREADS) void attn_packed_plan_few_kernel(int T, int n_seq, const int* __restrict__ offsets,
                                                                            PackedPlan* __restrict__ plan) {
  constexpr int WAVES = PLAN_THREADS / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int start[SEQS], len[SEQS], tiles[SEQS];
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    const int at = 64 * i + lane;
    start[i] = offsets[min(at, n_seq)];
    len[i] = offsets[min(at + 1, n_seq)];
  }
  int upto = 0, most = 0, total = 0;
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    int top = min(max(start[i], 0), T);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(top, o, 64);
      if (lane >= o) top = max(top, u);
    }
    start[i] = max(top, upto);
    upto = __shfl(start[i], 63, 64);
    len[i] = 64 * i + lane < n_seq ? max(min(max(len[i], 0), T) - start[i], 0) : 0;
    tiles[i] = (len[i] + 127) / 128;
    most = max(most, tiles[i]);
    total += tiles[i];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    most = max(most, __shfl_xor(most, o, 64));
    total += __shfl_xor(total, o, 64);
  }
  if (threadIdx.x == 0) plan->n = total;
  // this wave's classes, from the highest down
  const int per = (most + WAVES - 1) / WAVES, high = most - wave * per, low = max(high - per, 0);
  int place = 0;
#pragma unroll
  for (int i = 0; i < SEQS; ++i) place += max(tiles[i] - max(high, 0), 0);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) place += __shfl_xor(place, o, 64);
  for (int c = high - 1; c >= low; --c) {
#pragma unroll
    for (int i = 0; i < SEQS; ++i) {
      const unsigned long long mine = __ballot(tiles[i] > c);
      if (tiles[i] > c) plan->items[place + __popcll(mine & ((1ull << lane) - 1))] = PlanItem{start[i], len[i], c, 0};
      place += __popcll(mine);
    }
  }
}

// Any number: one workgroup sorts by counting.  The list's order among tiles with the same work is left to the atomics: no result
// depends on it.
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
  // dK / dV: workgroups that share a tile of keys, each with group / parts of its heads; above 1 they leave their sums in `partial`
  int parts;
  uint32_t units_recip, parts_recip;               // reciprocals of kv * parts and of parts
  floatx4* partial;
};

// A workgroup's item of the plan, on its way, and the unit (head) of it that the workgroup takes.  Grids have as many workgroups as a plan
// has places, so that the item can be read beside the number of items.
struct PackedTile {
  int start, len, tile, unit, item, n;
  // Is there such a tile?  A list that is not a plan of these rows makes no workgroup leave them.
  __device__ __forceinline__ bool exists(int T) const {
    return (item < n) & (len > 0) & (len <= T) & ((uint32_t)start <= (uint32_t)(T - len)) & ((uint32_t)tile <= (uint32_t)(len - 1) / 128u);
  }
};
__device__ __forceinline__ PackedTile packed_tile(const PackedArgs& p, uint32_t id, uint32_t units, uint32_t recip) {
  const uint32_t i = host::recip_div(id, units, recip);
  const int n = p.plan->n;
  const int4 it = *reinterpret_cast<const int4*>(&p.plan->items[i]);
  return PackedTile{it.x, it.y, it.z, (int)(id - i * units), (int)i, n};
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

// MFMA-bound on long sequences: one of 8192, 16 heads of 128 on 4, 267 us (1030 TFLOP/s of algorithmic work; the matrix units are busy 64 %
// of the time, at the clock that the power limit leaves).  On shorter ones the tiles' beginnings and ends count: of 40 heads of 128 over
// sequences of 80 to 1023 rows (4003 in all, 53 us, 600 TFLOP/s) the matrix units are busy 35 %; a workgroup walks 7 tiles of keys on
// average, about 1 us each, and takes 5 to get its rows, to leave its results and to give way to the next.
template <int D>
__global__ __launch_bounds__(256, 2) void attn_packed_fwd_kernel(PackedArgs p) {
  constexpr int KEYS = D > 128 ? 32 : 64;
  __shared__ FwdLds<D, KEYS> lds;
  const PackedTile t = packed_tile(p, blockIdx.x, p.heads, p.heads_recip);
  const int head = packed_head(p, t.unit), kv = host::recip_div(head, p.group, p.group_recip);
  if (!t.exists(p.T)) return;
  const PackedHead h = packed_rows(p, t.start, head, kv);
  attn_fwd_tile<D, true, KEYS>(lds, t.tile, t.len, p.d, p.scale, h.q, h.k, h.v, p.ld, p.o + h.row * p.ld_o + (int64_t)head * p.d, p.ld_o,
                         p.lse + (int64_t)head * p.T + h.row);
}

template <int D>
__device__ __forceinline__ void packed_dkdv(DkdvLds<D>& lds, const PackedArgs& p, uint32_t id) {
  const PackedTile t = packed_tile(p, id, p.kv * p.parts, p.units_recip);
  const int kv = host::recip_div(t.unit, p.parts, p.parts_recip), part = t.unit - kv * p.parts, heads = host::recip_div(p.group, p.parts, p.parts_recip);
  if (!t.exists(p.T)) return;
  const PackedHead h = packed_rows(p, t.start, kv * p.group + part * heads, kv);
  const int64_t stat = (int64_t)h.head * p.T + h.row;
  elem_t* const dk = p.dqkv + h.row * p.ld_dqkv + (int64_t)(p.heads + kv) * p.d;
  attn_bwd_dkdv<D, true, true>(lds, (t.len - 1) / 128 - t.tile, t.len, p.d, p.scale, h.q, h.k, h.v, p.ld,
                               p.dout + h.row * p.ld_do + (int64_t)h.head * p.d, p.ld_do, p.lse + stat, p.delta + stat, dk,
                               dk + (int64_t)p.kv * p.d, p.ld_dqkv, heads, p.T,
                               p.parts > 1 ? p.partial + (int64_t)id * partial_size<D>() : nullptr);
}
// The parts' sums, in order: a workgroup per tile, key / value head, dK or dV and 32 columns; a lane has 32 columns' half of a row.  What
// it takes is the latency of its reads and HBM: 2 parts of 64 tiles x 4 heads of 128 columns, 67 MB, 17 us.
template <int D>
__global__ __launch_bounds__(256) void attn_packed_dkdv_join_kernel(PackedArgs p) {
  constexpr int DT = D / 32, AT_ONCE = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t id = blockIdx.x / (2 * DT), rest = blockIdx.x - id * (2 * DT), which = rest / DT, dt = rest - which * DT;
  const PackedTile t = packed_tile(p, id, p.kv, p.kv_recip);
  if (!t.exists(p.T)) return;
  const int k = 128 * ((t.len - 1) / 128 - t.tile) + 32 * wave + (lane & 31);
  if (k >= t.len) return;
  const floatx4* const from = p.partial + (int64_t)id * p.parts * partial_size<D>() + partial_at<D>(wave, which, dt, 0, lane);
  floatx4 acc[4] = {};
  for (int first = 0; first < p.parts; first += AT_ONCE) {
    floatx4 v[AT_ONCE][4];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = from[(int64_t)min(first + i, p.parts - 1) * partial_size<D>() + 64 * j];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] += first + i < p.parts ? v[i][j][e] : 0.f;
  }
  const float mul = which ? 1.f : p.scale;
  elem_t* const out = p.dqkv + (t.start + (int64_t)k) * p.ld_dqkv + (int64_t)(p.heads + which * p.kv + t.unit) * p.d;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int col = 32 * dt + 8 * j + 4 * (lane >> 5);
    if (col >= p.d) continue;
    elemx4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (elem_t)(acc[j][e] * mul);
    *reinterpret_cast<elemx4*>(out + col) = v;
  }
}
template <int D, int FORM_DELTA, bool PINNED>
__device__ __forceinline__ void packed_dq(DqLds<D>& lds, const PackedArgs& p, uint32_t id) {
  const PackedTile t = packed_tile(p, id, p.heads, p.heads_recip);
  const int head = packed_head(p, t.unit), kv = host::recip_div(head, p.group, p.group_recip);
  if (!t.exists(p.T)) return;
  const PackedHead h = packed_rows(p, t.start, head, kv);
  const int64_t stat = (int64_t)head * p.T + h.row, col = (int64_t)head * p.d;
  attn_bwd_dq<D, true, FORM_DELTA, PINNED>(lds, t.tile, t.len, p.d, p.scale, h.q, h.k, h.v, p.ld, p.o + h.row * p.ld_o + col, p.ld_o,
                                   p.dout + h.row * p.ld_do + col, p.ld_do, p.lse + stat, p.delta + stat,
                                   p.dqkv + h.row * p.ld_dqkv + col, p.ld_dqkv, 0);
}
// dK / dV in a launch of its own behind dQ (up to 128 columns).  One sequence of 8192, 16 heads of 128 on 4: dQ 375, dK / dV 500, the parts' sums
// 17 us, 850 together (810 TFLOP/s; matrix units busy 65 % in both); the 40 heads above 73, 112 and none, busy 37 %: of a workgroup's 20 us
// 6.5 go to its beginning and end, which nothing hides (one workgroup per CU: 362 registers, 130 KB of LDS).
template <int D>
__global__ __launch_bounds__(256) void attn_packed_bwd_dkdv_kernel(PackedArgs p) {
  __shared__ DkdvLds<D> lds;
  packed_dkdv<D>(lds, p, blockIdx.x);
}
template <int D>
__global__ __launch_bounds__(256, 2) void attn_packed_bwd_dq_kernel(PackedArgs p) {
  __shared__ DqLds<D> lds;
  packed_dq<D, FORM_DELTA_ANY, false>(lds, p, blockIdx.x);
}
// Both at once (host::packed_one_launch): the first workgroups form dK and dV, the others dQ.  24 heads of 188 over seven sequences of about
// 512: 110 us where the two launches took 63 and 72.
template <int D>
__global__ __launch_bounds__(256) void attn_packed_bwd_both_kernel(PackedArgs p, uint32_t n_dkdv) {
  __shared__ union { DkdvLds<D> dkdv; DqLds<D> dq; } lds;
  if (blockIdx.x < n_dkdv) packed_dkdv<D>(lds.dkdv, p, blockIdx.x);
  else packed_dq<D, READ_DELTA, (D > 128)>(lds.dq, p, blockIdx.x - n_dkdv);
}

// delta[head][row] = sum over the head's columns of dO o, for the one-launch backward: LANES lanes per (row, head), 8 elements each,
// DELTA_PAIRS pairs on their way at once.  HBM-bound: 3064 rows of 24 heads of 188, 55 MB, 12 us.
constexpr int DELTA_PAIRS = 4;
template <int D>
__global__ __launch_bounds__(256) void attn_packed_delta_kernel(PackedArgs p) {
  constexpr int LANES = D == 192 ? 32 : D / 8;
  const int ch = threadIdx.x % LANES, n = p.d - 8 * ch;
  const uint32_t group = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, pairs = (uint32_t)p.T * p.heads;      // at most 2^27
  elemx8 o[DELTA_PAIRS], g[DELTA_PAIRS];
  uint32_t row[DELTA_PAIRS], head[DELTA_PAIRS];
  const auto chunk = [&](const elem_t* q) {
    union { elemx8 v; u32x4 w; u32x2 h[2]; } u;
    u.w = u32x4{0, 0, 0, 0};
    if (n >= 8) u.v = *reinterpret_cast<const elemx8*>(q);
    else if (n >= 4) u.h[0] = *reinterpret_cast<const u32x2*>(q);
    return u.v;
  };
#pragma unroll
  for (int i = 0; i < DELTA_PAIRS; ++i) {
    const uint32_t pair = min(group * DELTA_PAIRS + i, pairs - 1);
    row[i] = host::recip_div(pair, p.heads, p.heads_recip);
    head[i] = pair - row[i] * p.heads;
    const int64_t col = (int64_t)head[i] * p.d + 8 * ch;
    o[i] = chunk(p.o + row[i] * p.ld_o + col);
    g[i] = chunk(p.dout + row[i] * p.ld_do + col);
  }
#pragma unroll
  for (int i = 0; i < DELTA_PAIRS; ++i) {
    float sum = delta_add<8, false>(0.f, o[i], g[i], 0);
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (ch == 0 && group * DELTA_PAIRS + i < pairs) p.delta[(int64_t)head[i] * p.T + row[i]] = sum;
  }
}

// ------------------------------------------------------------------------------------------------------------- launchers
hipError_t launch_attention_packed_plan(int64_t T, int64_t n_seq, const int* offsets, void* plan, hipStream_t st) {
  if (n_seq <= 64)
    hipLaunchKernelGGL(attn_packed_plan_few_kernel<1>, dim3(1), dim3(PLAN_THREADS), 0, st, (int)T, (int)n_seq, offsets, (PackedPlan*)plan);
  else if (n_seq <= PLAN_FEW)
    hipLaunchKernelGGL(attn_packed_plan_few_kernel<PLAN_FEW / 64>, dim3(1), dim3(PLAN_THREADS), 0, st, (int)T, (int)n_seq, offsets, (PackedPlan*)plan);
  else
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

static int packed_columns(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 192; }
static int packed_parts(const PackedShape& s) { return host::packed_parts(s.T, s.n_seq, s.heads, s.kv, packed_columns(s.d)); }
static uint64_t delta_bytes(const PackedShape& s) { return ((uint64_t)s.T * (uint64_t)s.heads * 4 + 255) / 256 * 256; }
uint64_t attention_packed_bwd_ws_bytes(const PackedShape& s) {
  const int parts = packed_parts(s);
  return delta_bytes(s) + (parts > 1 ? (uint64_t)packed_tiles_bound(s.T, s.n_seq) * s.kv * parts * 128 * 2 * packed_columns(s.d) * 4 : 0);
}

#define AXONN_PACKED_128(KERNEL, GRID, ...)                                                                 \
  do {                                                                                                 \
    if (s.d <= 64) hipLaunchKernelGGL(KERNEL<64>, dim3(GRID), dim3(256), 0, st, __VA_ARGS__);          \
    else hipLaunchKernelGGL(KERNEL<128>, dim3(GRID), dim3(256), 0, st, __VA_ARGS__);                   \
    const hipError_t e = hipGetLastError();                                                            \
    if (e != hipSuccess) return e;                                                                     \
  } while (0)
#define AXONN_PACKED(KERNEL, GRID, ...)                                                                     \
  do {                                                                                                 \
    if (s.d <= 128) {                                                                                  \
      AXONN_PACKED_128(KERNEL, GRID, __VA_ARGS__);                                                     \
      break;                                                                                           \
    }                                                                                                  \
    hipLaunchKernelGGL(KERNEL<192>, dim3(GRID), dim3(256), 0, st, __VA_ARGS__);                        \
    const hipError_t e = hipGetLastError();                                                            \
    if (e != hipSuccess) return e;                                                                     \
  } while (0)

hipError_t launch_attention_packed_fwd(const PackedShape& s, const void* plan, const void* qkv, int64_t ld, void* o, int64_t ld_o, float* lse,
                                       hipStream_t st) {
  PackedArgs p = packed_args(s, plan);
  p.qkv = (const elem_t*)qkv; p.ld = ld;
  p.o = (elem_t*)o; p.ld_o = ld_o; p.lse = lse;
  AXONN_PACKED(attn_packed_fwd_kernel, (unsigned)(packed_tiles_bound(s.T, s.n_seq) * s.heads), p);
  return hipSuccess;
}

hipError_t launch_attention_packed_bwd(const PackedShape& s, const void* plan, const void* qkv, int64_t ld, const void* o, int64_t ld_o,
                                       const float* lse, const void* dout, int64_t ld_do, void* dqkv, int64_t ld_dqkv, void* workspace,
                                       hipStream_t st) {
  PackedArgs p = packed_args(s, plan);
  p.qkv = (const elem_t*)qkv; p.ld = ld;
  p.o = (elem_t*)const_cast<void*>(o); p.ld_o = ld_o; p.lse = const_cast<float*>(lse);
  p.dout = (const elem_t*)dout; p.ld_do = ld_do;
  p.dqkv = (elem_t*)dqkv; p.ld_dqkv = ld_dqkv;
  p.delta = (float*)workspace;
  p.parts = packed_parts(s);
  p.parts_recip = host::recip_of(p.parts); p.units_recip = host::recip_of(p.kv * p.parts);
  p.partial = (floatx4*)((char*)workspace + delta_bytes(s));
  const int64_t tiles = packed_tiles_bound(s.T, s.n_seq);
  const unsigned n_dq = (unsigned)(tiles * s.heads), n_join = (unsigned)(tiles * s.kv), n_dkdv = n_join * p.parts;
  if (host::packed_one_launch(n_dq, packed_columns(s.d))) {
    const int per_block = 256 * DELTA_PAIRS / (s.d > 128 ? 32 : packed_columns(s.d) / 8);
    AXONN_PACKED(attn_packed_delta_kernel, (unsigned)((s.T * s.heads + per_block - 1) / per_block), p);
    AXONN_PACKED(attn_packed_bwd_both_kernel, n_dq + n_dkdv, p, n_dkdv);
  } else {
    AXONN_PACKED_128(attn_packed_bwd_dq_kernel, n_dq, p);   // forms delta
    AXONN_PACKED_128(attn_packed_bwd_dkdv_kernel, n_dkdv, p);
  }
  if (p.parts > 1) AXONN_PACKED(attn_packed_dkdv_join_kernel, n_join * (packed_columns(s.d) / 16), p);
  return hipSuccess;
}
#undef AXONN_PACKED
#undef AXONN_PACKED_128

}  // namespace axonn
