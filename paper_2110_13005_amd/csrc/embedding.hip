// Embedding lookup with a scale, and the gradient of its table by sorted tokens.
//
//   out[t, :] = scale * table[id_t, :]            dtable[v, :] (+)= scale * sum over the tokens t with id_t = v of dout[t, :]
//
// Both are bound by HBM.  The gradient's sums are formed in fp32 in the order of the tokens (a stable sort of the ids, then
// fixed pieces of the sorted list, then the pieces of one id in order): no atomics on values, the same bits every run.
// Ids outside [0, vocab) are clamped into range, as everywhere in the library.
#include "rows.h"
#include <algorithm>

namespace axonn {

__device__ __forceinline__ int clamp_token(int id, int vocab) { return id < 0 ? 0 : (id >= vocab ? vocab - 1 : id); }

// ------------------------------------------------------------------------------------------------------------- lookup
// A row belongs to LPR lanes (a power of two that covers it, at most a workgroup; grid.y where it is wider); every lane has
// EMB_ROWS rows in flight.
constexpr int EMB_THREADS = 256, EMB_ROWS = 4;

template <int LPR>
__global__ __launch_bounds__(EMB_THREADS) void embedding_fwd_kernel(int T, int h, int vocab, const int* __restrict__ tokens,
                                                                    const elem_t* __restrict__ table, float scale,
                                                                    elem_t* __restrict__ out, int64_t ld_out) {
  constexpr int PAR = EMB_THREADS / LPR;
  const int64_t t0 = (int64_t)blockIdx.x * (PAR * EMB_ROWS) + threadIdx.x / LPR;
  const int c = 8 * (blockIdx.y * LPR + threadIdx.x % LPR), n = h - c;
  if (n <= 0) return;
  elemx8 v[EMB_ROWS];
#pragma unroll
  for (int i = 0; i < EMB_ROWS; ++i) {
    const int64_t t = t0 + i * PAR;
    if (t < T) v[i] = load_chunk(table + (int64_t)clamp_token(tokens[t], vocab) * h + c, n);
  }
#pragma unroll
  for (int i = 0; i < EMB_ROWS; ++i) {
    const int64_t t = t0 + i * PAR;
    if (t >= T) break;
    elemx8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (elem_t)((float)v[i][e] * scale);
    store_chunk(out + t * ld_out + c, o, n);
  }
}

hipError_t launch_embedding_fwd(int64_t T, int64_t h, int64_t vocab, const int* tokens, const void* table, float scale, void* out,
                                int64_t ld_out, hipStream_t s) {
  const int chunks = (int)((h + 7) / 8);
  auto launch = [&](auto lpr) {
    constexpr int LPR = decltype(lpr)::value, ROWS = EMB_THREADS / LPR * EMB_ROWS;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_fwd_kernel<LPR>), dim3((unsigned)((T + ROWS - 1) / ROWS), (chunks + LPR - 1) / LPR),
                       dim3(EMB_THREADS), 0, s, (int)T, (int)h, (int)vocab, tokens, (const elem_t*)table, scale, (elem_t*)out, ld_out);
  };
  if (chunks <= 16) launch(std::integral_constant<int, 16>{});
  else if (chunks <= 32) launch(std::integral_constant<int, 32>{});
  else if (chunks <= 64) launch(std::integral_constant<int, 64>{});
  else if (chunks <= 128) launch(std::integral_constant<int, 128>{});
  else launch(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

// --------------------------------------------------------------------------------------------------------------- sort
// Least-significant-digit radix sort of (id, token index): one pass per digit, a histogram kernel and a scatter kernel each.
// A workgroup owns a contiguous range of the list; the scatter kernel forms its own bases from the histograms of all ranges
// (at most SORT_MAX_BLOCKS of them), so that no workgroup ever waits for another.
constexpr int SORT_THREADS = 512, SORT_WAVES = SORT_THREADS / 64, SORT_ITEMS = 4, SORT_TILE = SORT_THREADS * SORT_ITEMS;
constexpr int SORT_MAX_BLOCKS = 128, SORT_MAX_BITS = 10;

struct SortPass {
  int T, per_block, vocab;       // per_block: a multiple of SORT_TILE
  int shift, bits;
  const int* keys_in;            // the first pass: the tokens themselves
  const int* index_in;           // null: the position
  int *keys_out, *index_out;
  uint32_t* hist;                // [blocks][bins]
};

__global__ __launch_bounds__(SORT_THREADS) void embedding_sort_hist_kernel(const SortPass p) {
  extern __shared__ uint32_t sort_lds[];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += SORT_THREADS) sort_lds[b] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * p.per_block, hi = min((int64_t)p.T, lo + p.per_block);
  for (int64_t i = lo + threadIdx.x; i < hi; i += SORT_THREADS)
    atomicAdd(&sort_lds[(clamp_token(p.keys_in[i], p.vocab) >> p.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += SORT_THREADS) p.hist[(int64_t)blockIdx.x * bins + b] = sort_lds[b];
}

// Stable: an item's place is the base of its digit, plus the items of that digit in front of it: in earlier ranges and tiles,
// in earlier waves of the tile (a wave owns 64 * SORT_ITEMS consecutive items), in earlier rounds of the wave, in lower lanes.
// LDS: counters [SORT_WAVES][bins], bases [bins], sums of 8 waves.
__global__ __launch_bounds__(SORT_THREADS) void embedding_sort_scatter_kernel(const SortPass p, int blocks) {
  extern __shared__ uint32_t sort_lds[];
  const int bins = 1 << p.bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t* const base = sort_lds + SORT_WAVES * bins;
  uint32_t* const wave_total = base + bins;
  // bases: exclusive sums of the digits' totals, SORT_THREADS digits at a time, plus what earlier ranges hold
  uint32_t carry = 0;
  for (int b0 = 0; b0 < bins; b0 += SORT_THREADS) {
    const int b = b0 + tid;
    uint32_t total = 0, before = 0;
    if (b < bins)
      for (int q = 0; q < blocks; ++q) {
        const uint32_t v = p.hist[(int64_t)q * bins + b];
        total += v;
        before += q < (int)blockIdx.x ? v : 0;
      }
    uint32_t scan = total;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(scan, o, 64);
      if (lane >= o) scan += up;
    }
    if (lane == 63) wave_total[wave] = scan;
    __syncthreads();
    uint32_t front = carry, all = carry;
    for (int w = 0; w < SORT_WAVES; ++w) {
      if (w < wave) front += wave_total[w];
      all += wave_total[w];
    }
    if (b < bins) base[b] = front + scan - total + before;
    carry = all;
    __syncthreads();
  }
  const int64_t lo = (int64_t)blockIdx.x * p.per_block, hi = min((int64_t)p.T, lo + p.per_block);
  for (int64_t t0 = lo; t0 < hi; t0 += SORT_TILE) {
    for (int b = tid; b < SORT_WAVES * bins; b += SORT_THREADS) sort_lds[b] = 0;
    __syncthreads();
    int key[SORT_ITEMS], index[SORT_ITEMS];
    uint32_t rank[SORT_ITEMS];
    volatile uint32_t* const mine = sort_lds + wave * bins;
#pragma unroll
    for (int k = 0; k < SORT_ITEMS; ++k) {
      const int64_t i = t0 + wave * (64 * SORT_ITEMS) + k * 64 + lane;
      const bool live = i < hi;
      key[k] = live ? clamp_token(p.keys_in[i], p.vocab) : 0;
      index[k] = live ? (p.index_in ? p.index_in[i] : (int)i) : -1;
      const int digit = (key[k] >> p.shift) & (bins - 1);
      unsigned long long peers = __ballot(live);
      for (int bit = 0; bit < p.bits; ++bit) {
        const unsigned long long set = __ballot((digit >> bit) & 1);
        peers &= (digit >> bit) & 1 ? set : ~set;
      }
      const unsigned long long below = peers & ((1ull << lane) - 1);
      const uint32_t old = live ? mine[digit] : 0;
      rank[k] = old + __popcll(below);
      __builtin_amdgcn_wave_barrier();                 // every lane has read before the first of a digit's lanes writes
      if (live && below == 0) mine[digit] = old + __popcll(peers);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // counters -> places: exclusive over the waves, on top of the digit's base, which moves past this tile
    for (int b = tid; b < bins; b += SORT_THREADS) {
      uint32_t at = base[b];
      for (int w = 0; w < SORT_WAVES; ++w) {
        const uint32_t c = sort_lds[w * bins + b];
        sort_lds[w * bins + b] = at;
        at += c;
      }
      base[b] = at;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_ITEMS; ++k)
      if (index[k] >= 0) {
        const uint32_t at = mine[(key[k] >> p.shift) & (bins - 1)] + rank[k];
        p.keys_out[at] = key[k];
        p.index_out[at] = index[k];
      }
    __syncthreads();
  }
}

// --------------------------------------------------------------------------------------------------------------- sums
// The sorted list is cut into pieces of PIECE tokens; a wave adds the rows of one piece over 512 columns (8 per lane), a
// batch of 8 rows in flight.  A run of equal ids that lies within the piece is finished here; one that crosses the piece's
// start leaves its sum in partial[piece][0], one that begins in the piece and crosses its end in partial[piece][1], and
// embedding_bwd_join_kernel adds them up.
constexpr int PIECE = 32, SUM_BATCH = 8, SUM_COLS = 512;

struct TableGrad {
  int T, h, vocab, pieces, col_chunks;
  const int *ids, *order;            // sorted
  const elem_t* dout;
  int64_t ld_dout;
  float scale;
  int accumulate;
  void* dtable;
  float* partial;                    // [pieces][2][h]
};

template <bool FP32>
__device__ __forceinline__ void store_table_row(const TableGrad& g, int id, int c, int n, const float (&acc)[8]) {
  if constexpr (FP32) {
    float* p = (float*)g.dtable + (int64_t)id * g.h + c;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = acc[e] * g.scale + (g.accumulate ? p[e] : 0.f);
  } else {
    elem_t* p = (elem_t*)g.dtable + (int64_t)id * g.h + c;
    elemx8 o, old = {};
    if (g.accumulate) old = load_chunk(p, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (elem_t)(acc[e] * g.scale + (float)old[e]);
    store_chunk(p, o, n);
  }
}

template <bool FP32>
__global__ __launch_bounds__(256) void embedding_bwd_sum_kernel(const TableGrad g) {
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int piece = (int)(w / g.col_chunks), c = (int)(w - (int64_t)piece * g.col_chunks) * SUM_COLS + 8 * lane, n = g.h - c;
  if (piece >= g.pieces) return;
  const int first = piece * PIECE, count = min(PIECE, g.T - first);
  const int id = lane < count ? g.ids[first + lane] : -1, row = lane < count ? g.order[first + lane] : 0;
  const int before = first > 0 ? g.ids[first - 1] : -1, behind = first + count < g.T ? g.ids[first + count] : -1;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  bool from_start = true;                               // the run at hand began with the piece
  for (int i0 = 0; i0 < count; i0 += SUM_BATCH) {
    elemx8 v[SUM_BATCH];
#pragma unroll
    for (int k = 0; k < SUM_BATCH; ++k) {
      const int r = __builtin_amdgcn_readlane(row, min(i0 + k, count - 1));
      if (n > 0) v[k] = load_chunk(g.dout + (int64_t)r * g.ld_dout + c, n);
    }
#pragma unroll
    for (int k = 0; k < SUM_BATCH; ++k) {
      const int i = i0 + k;
      if (i >= count) break;
      const int cur = __builtin_amdgcn_readlane(id, i);
      const int next = i + 1 < count ? __builtin_amdgcn_readlane(id, min(i + 1, 63)) : behind;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += (float)v[k][e];
      if (next == cur && i + 1 < count) continue;
      const bool head = from_start && before == cur, tail = next == cur;
      if (n > 0) {
        if (!head && !tail) store_table_row<FP32>(g, cur, c, n, acc);
        else {
          float* p = g.partial + ((int64_t)piece * 2 + (head ? 0 : 1)) * g.h + c;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = acc[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      from_start = false;
    }
  }
}

// Runs that cross pieces.  One workgroup per piece and 512 columns; it has work if a run begins in its piece and crosses the
// end.  The run's parts in the following pieces are shared out to the four waves in order, and the waves' sums added in order.
template <bool FP32>
__global__ __launch_bounds__(256) void embedding_bwd_join_kernel(const TableGrad g) {
  __shared__ float sums[3][64][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = blockIdx.x;
  const int c = blockIdx.y * SUM_COLS + 8 * lane, n = g.h - c;
  const int first = piece * PIECE, last = first + PIECE - 1;
  if (last + 1 >= g.T) return;
  const int id = g.ids[last];
  if (g.ids[last + 1] != id || (first > 0 && g.ids[first - 1] == id && g.ids[first] == id)) return;
  // the last piece that begins with this id: ids at the pieces' starts are sorted
  int lo = piece + 1, hi = g.pieces - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (g.ids[mid * PIECE] == id) lo = mid;
    else hi = mid - 1;
  }
  const int parts = lo - piece + 1;                     // partial[piece][1], then partial[piece + 1 .. lo][0]
  const int share = (parts + 3) / 4, p0 = wave * share, p1 = min(parts, p0 + share);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  if (n > 0)
    for (int q = p0; q < p1; ++q) {
      const float* p = g.partial + ((int64_t)(piece + q) * 2 + (q == 0 ? 1 : 0)) * g.h + c;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) acc[e] += p[e];
    }
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave - 1][lane][e] = acc[e];
  }
  __syncthreads();
  if (wave > 0 || n <= 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += sums[w][lane][e];
  store_table_row<FP32>(g, id, c, n, acc);
}

// bytes of zeros at p (any 2-byte aligned address).
__global__ __launch_bounds__(256) void embedding_clear_kernel(uint16_t* p, int64_t halves) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i < halves) store_chunk((elem_t*)(p + i), elemx8{}, (int)min((int64_t)8, halves - i));
}

// Workspace, in this order, each part at a multiple of 256 bytes.
struct EmbeddingWs {
  int blocks, per_block, bits, pieces;
  uint64_t keys[2], index[2], hist, partial, bytes;
};
static EmbeddingWs embedding_ws(int64_t T, int64_t h, int64_t vocab) {
  EmbeddingWs w;
  w.bits = 1;
  while (((int64_t)1 << w.bits) < vocab) ++w.bits;
  const int64_t tiles = (T + SORT_TILE - 1) / SORT_TILE;
  const int64_t per = (tiles + SORT_MAX_BLOCKS - 1) / SORT_MAX_BLOCKS;
  w.per_block = (int)(per * SORT_TILE);
  w.blocks = (int)((tiles + per - 1) / per);
  w.pieces = (int)((T + PIECE - 1) / PIECE);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t r = at; at += (bytes + 255) / 256 * 256; return r; };
  for (int i = 0; i < 2; ++i) { w.keys[i] = take(4 * (uint64_t)T); w.index[i] = take(4 * (uint64_t)T); }
  w.hist = take(4ull * w.blocks << SORT_MAX_BITS);
  w.partial = take(8ull * w.pieces * (uint64_t)h);
  w.bytes = at;
  return w;
}
uint64_t embedding_bwd_ws_bytes(int64_t T, int64_t h, int64_t vocab) { return embedding_ws(T, h, vocab).bytes; }

hipError_t launch_embedding_bwd(int64_t T, int64_t h, int64_t vocab, const int* tokens, const void* dout, int64_t ld_dout, float scale,
                                void* dtable, bool fp32, bool accumulate, void* workspace, hipStream_t s) {
  const EmbeddingWs w = embedding_ws(T, h, vocab);
  char* const ws = (char*)workspace;
  if (!accumulate) {
    const int64_t halves = vocab * h * (fp32 ? 2 : 1);
    hipLaunchKernelGGL(embedding_clear_kernel, dim3((unsigned)((halves + 2047) / 2048)), dim3(256), 0, s, (uint16_t*)dtable, halves);
  }
  const int passes = (w.bits + SORT_MAX_BITS - 1) / SORT_MAX_BITS;
  for (int i = 0, shift = 0; i < passes; ++i) {
    SortPass p;
    p.T = (int)T; p.per_block = w.per_block; p.vocab = (int)vocab;
    p.bits = (w.bits - shift + passes - i - 1) / (passes - i);
    p.shift = shift;
    const int to = i & 1, from = to ^ 1;
    p.keys_in = i == 0 ? tokens : (const int*)(ws + w.keys[from]);
    p.index_in = i == 0 ? nullptr : (const int*)(ws + w.index[from]);
    p.keys_out = (int*)(ws + w.keys[to]); p.index_out = (int*)(ws + w.index[to]);
    p.hist = (uint32_t*)(ws + w.hist);
    const int bins = 1 << p.bits;
    hipLaunchKernelGGL(embedding_sort_hist_kernel, dim3(w.blocks), dim3(SORT_THREADS), bins * 4, s, p);
    hipLaunchKernelGGL(embedding_sort_scatter_kernel, dim3(w.blocks), dim3(SORT_THREADS), ((SORT_WAVES + 1) * bins + SORT_WAVES) * 4, s, p,
                       w.blocks);
    shift += p.bits;
  }
  TableGrad g;
  g.T = (int)T; g.h = (int)h; g.vocab = (int)vocab; g.pieces = w.pieces; g.col_chunks = (int)((h + SUM_COLS - 1) / SUM_COLS);
  g.ids = (const int*)(ws + w.keys[(passes - 1) & 1]); g.order = (const int*)(ws + w.index[(passes - 1) & 1]);
  g.dout = (const elem_t*)dout; g.ld_dout = ld_dout; g.scale = scale; g.accumulate = accumulate; g.dtable = dtable;
  g.partial = (float*)(ws + w.partial);
  const unsigned blocks = (unsigned)(((int64_t)g.pieces * g.col_chunks + 3) / 4);
  const dim3 join(g.pieces, g.col_chunks);
  if (fp32) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_sum_kernel<true>), dim3(blocks), dim3(256), 0, s, g);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_join_kernel<true>), join, dim3(256), 0, s, g);
  } else {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_sum_kernel<false>), dim3(blocks), dim3(256), 0, s, g);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_join_kernel<false>), join, dim3(256), 0, s, g);
  }
  return hipGetLastError();
}

}  // namespace axonn
