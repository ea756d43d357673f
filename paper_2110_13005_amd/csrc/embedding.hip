// Embedding lookup with a scale, and the gradient of its table by sorted tokens.
//
//   out[t, :] = scale * table[id_t, :]            dtable[v, :] (+)= scale * sum over the tokens t with id_t = v of dout[t, :]
//
// Both are bound by HBM.  The gradient's sums are formed in fp32 in the order of the tokens (equal ids brought together in the
// tokens' order, then fixed pieces of the list, then the pieces of one id in order): no atomics on values, the same bits every run.
// Ids outside [0, vocab) are clamped into range, as everywhere in the library.
#include "rows.h"
#include <algorithm>

namespace axonn {

__device__ __forceinline__ int clamp_token(int id, int vocab) { return id < 0 ? 0 : (id >= vocab ? vocab - 1 : id); }

// ------------------------------------------------------------------------------------------------------------- lookup
// A row belongs to LPR lanes (a power of two that covers it, at most a workgroup; grid.y where it is wider); every lane has
// EMB_ROWS rows in flight.  HBM-bound: 16384 tokens x 5120 of a table of 51200 in 46 us (4.8 TB/s of the rows that differ and the
// result; a device copy reaches 5.1).
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
#pragma unroll 8
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

// Up to SORT_SHARE_MAX tokens in one launch, and equal ids only brought together: a workgroup per residue of the ids modulo
// SORT_SHARES looks at all tokens, counts those of smaller residues (its place in the list) and sorts its own, in LDS: quotient
// and token index as one 32-bit key, one pass per digit as in the scatter kernel, none if they are all the same.  The launch's
// other workgroups clear the table meanwhile: 15 us and, for 51200 x 2048, 39 (5.3 TB/s of writes).  A workgroup that sorted all
// ids by itself was bound by its ballots: 30 us for 16384 tokens; with ranges of consecutive ids the one of a text's most
// frequent words had most of them.
constexpr int SORT_SHARE_THREADS = 1024, SORT_SHARE_WAVES = SORT_SHARE_THREADS / 64, SORT_SHARE_ITEMS = 16;
constexpr int SORT_SHARE_MAX = SORT_SHARE_THREADS * SORT_SHARE_ITEMS, SORT_SHARE_BITS = 8;
constexpr int SORT_SHARES_LOG = 5, SORT_SHARES = 1 << SORT_SHARES_LOG;

// Zeros to `halves` 16-bit numbers from p on, by workgroup `block` of `blocks`: four chunks per thread and round.
template <int THREADS>
__device__ __forceinline__ void clear_table(uint16_t* p, int64_t halves, int64_t block, int64_t blocks) {
  constexpr int64_t ROUND = THREADS * 8 * 4;
  for (int64_t i0 = block * ROUND; i0 < halves; i0 += blocks * ROUND) {
    const int64_t i = i0 + threadIdx.x * 8;
    if (i0 + ROUND <= halves) {
#pragma unroll
      for (int k = 0; k < 4; ++k) *reinterpret_cast<elemx8_any*>(p + i + k * (THREADS * 8)) = elemx8{};
    } else {
#pragma unroll 1
      for (int k = 0; k < 4; ++k) {
        const int64_t at = i + k * (THREADS * 8);
        if (at < halves) store_chunk((elem_t*)(p + at), elemx8{}, (int)min((int64_t)8, halves - at));
      }
    }
  }
}

__global__ __launch_bounds__(SORT_SHARE_THREADS) void embedding_sort_share_kernel(int T, int vocab, int key_bits, int shares, int t_bits,
                                                                                  const int* __restrict__ tokens, int* __restrict__ ids,
                                                                                  int* __restrict__ order, uint16_t* clear, int64_t halves) {
  constexpr int BINS = 1 << SORT_SHARE_BITS;
  __shared__ uint32_t list[SORT_SHARE_MAX];
  __shared__ uint32_t counter[SORT_SHARE_WAVES][BINS];
  __shared__ uint32_t wave_sum[SORT_SHARE_WAVES], wave_below[SORT_SHARE_WAVES];
  if ((int)blockIdx.x >= shares) {
    clear_table<SORT_SHARE_THREADS>(clear, halves, blockIdx.x - shares, gridDim.x - shares);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int share = blockIdx.x;
  auto share_of = [](int id) { return id & (SORT_SHARES - 1); };
  // the tokens of this share, in order: wave w looks at 64 * looks consecutive ones
  const int looks = (T + SORT_SHARE_THREADS - 1) / SORT_SHARE_THREADS;
  int id[SORT_SHARE_ITEMS];
  uint32_t taken = 0, below = 0;
#pragma unroll
  for (int k = 0; k < SORT_SHARE_ITEMS; ++k) {
    const int i = (wave * looks + k) * 64 + lane;
    id[k] = k < looks && i < T ? clamp_token(tokens[i], vocab) : -1;
  }
#pragma unroll
  for (int k = 0; k < SORT_SHARE_ITEMS; ++k) {
    taken += __popcll(__ballot(id[k] >= 0 && share_of(id[k]) == share));
    below += __popcll(__ballot(id[k] >= 0 && share_of(id[k]) < share));
  }
  if (lane == 0) {
    wave_sum[wave] = taken;
    wave_below[wave] = below;
  }
  __syncthreads();
  uint32_t at = 0, n = 0, base = 0;
  for (int w = 0; w < SORT_SHARE_WAVES; ++w) {
    if (w < wave) at += wave_sum[w];
    n += wave_sum[w];
    base += wave_below[w];
  }
  if (n == 0) return;
#pragma unroll
  for (int k = 0; k < SORT_SHARE_ITEMS; ++k) {
    const bool in = id[k] >= 0 && share_of(id[k]) == share;
    const unsigned long long m = __ballot(in);
    if (in) list[at + __popcll(m & ((1ull << lane) - 1))] = (uint32_t)id[k] >> SORT_SHARES_LOG << t_bits | (uint32_t)((wave * looks + k) * 64 + lane);
    at += __popcll(m);
  }
  __syncthreads();
  // sort list[0 .. n): wave w owns 64 * items consecutive places
  const int items = ((int)n + SORT_SHARE_THREADS - 1) / SORT_SHARE_THREADS, first = wave * 64 * items + lane;
  uint32_t key[SORT_SHARE_ITEMS], rank[SORT_SHARE_ITEMS];
  bool other = false;
  const uint32_t some = list[0] >> t_bits;
#pragma unroll
  for (int k = 0; k < SORT_SHARE_ITEMS; ++k) {
    const int i = first + 64 * k;
    key[k] = k < items && i < (int)n ? list[i] : 0;
    other |= k < items && i < (int)n && key[k] >> t_bits != some;
  }
  const bool unsorted = __syncthreads_or(other);
  for (int shift = 0; unsorted && shift < key_bits; shift += SORT_SHARE_BITS) {
    const int digit_bits = min(SORT_SHARE_BITS, key_bits - shift), low = t_bits + shift;
    for (int b = tid; b < SORT_SHARE_WAVES * BINS; b += SORT_SHARE_THREADS) (&counter[0][0])[b] = 0;
    __syncthreads();
    volatile uint32_t* const mine = counter[wave];
#pragma unroll
    for (int k = 0; k < SORT_SHARE_ITEMS; ++k) {
      if (k >= items) continue;
      const bool live = first + 64 * k < (int)n;
      const uint32_t digit = key[k] >> low & ((1u << digit_bits) - 1);
      unsigned long long peers = __ballot(live);
      for (int bit = 0; bit < digit_bits; ++bit) {
        const unsigned long long set = __ballot(digit >> bit & 1);
        peers &= digit >> bit & 1 ? set : ~set;
      }
      const unsigned long long in_front = peers & ((1ull << lane) - 1);
      const uint32_t old = live ? mine[digit] : 0;
      rank[k] = old + __popcll(in_front);
      __builtin_amdgcn_wave_barrier();                 // every lane has read before the first of a digit's lanes writes
      if (live && in_front == 0) mine[digit] = old + __popcll(peers);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // counters -> places: exclusive over the digits, then over the waves
    uint32_t total = 0, scan = 0;
    if (wave < BINS / 64) {
      for (int w = 0; w < SORT_SHARE_WAVES; ++w) total += counter[w][tid];
      scan = total;
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(scan, o, 64);
        if (lane >= o) scan += up;
      }
      if (lane == 63) wave_sum[wave] = scan;
    }
    __syncthreads();
    if (wave < BINS / 64) {
      uint32_t place = scan - total;
      for (int w = 0; w < wave; ++w) place += wave_sum[w];
      for (int w = 0; w < SORT_SHARE_WAVES; ++w) {
        const uint32_t c = counter[w][tid];
        counter[w][tid] = place;
        place += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_SHARE_ITEMS; ++k)
      if (k < items && first + 64 * k < (int)n) list[mine[key[k] >> low & ((1u << digit_bits) - 1)] + rank[k]] = key[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_SHARE_ITEMS; ++k)
      if (k < items && first + 64 * k < (int)n) key[k] = list[first + 64 * k];
  }
#pragma unroll
  for (int k = 0; k < SORT_SHARE_ITEMS; ++k)
    if (k < items && first + 64 * k < (int)n) {
      ids[base + first + 64 * k] = (int)(key[k] >> t_bits << SORT_SHARES_LOG) | share;
      order[base + first + 64 * k] = (int)(key[k] & ((1u << t_bits) - 1));
    }
}

// --------------------------------------------------------------------------------------------------------------- sums
// The sorted list is cut into pieces; a wave adds the rows of one piece over 512 columns (8 per lane), SUM_BATCH of them in
// flight: 16384 x 2048 in 24 us, 3.2 TB/s with what a run's end writes.  Pieces are one batch, or four where there are many tokens:
// fewer sums of runs that cross pieces (accumulating, text / one id, in all: 131072 x 1024 109 / 135 us, with pieces of one batch
// 150 / 346; 32768 x 2048 72 / 93 and 74 / 150).  A run of equal ids
// that lies within the piece is finished here; one that crosses the piece's start leaves its sum in partial[piece][0], one that
// begins in the piece and crosses its end in partial[piece][1], and embedding_bwd_join_kernel adds them up.
constexpr int SUM_BATCH = 16, SUM_COLS = 512;
constexpr int PIECE_FEW = SUM_BATCH, PIECE_MANY = 4 * SUM_BATCH, MANY_TOKENS = 32768;
typedef floatx4 floatx4_any __attribute__((aligned(4)));

struct TableGrad {
  int T, h, vocab, pieces, col_chunks;
  const int *ids, *order;            // sorted (few tokens: ids are the tokens as they are)
  const elem_t* dout;
  int64_t ld_dout;
  float scale;
  int accumulate;
  void* dtable;
  float* partial;                    // [pieces][2][h]
};

// Columns c .. c + n of row id, n of 8 (8 or more: all).
template <bool FP32>
__device__ __forceinline__ void store_table_row(const TableGrad& g, int id, int c, int n, const float (&acc)[8], float scale) {
  const bool accumulate = g.accumulate;
  if constexpr (FP32) {
    float* p = (float*)g.dtable + (int64_t)id * g.h + c;
    if (n >= 8) {
      floatx4_any* const v = (floatx4_any*)p;
      floatx4 lo = {acc[0], acc[1], acc[2], acc[3]}, hi = {acc[4], acc[5], acc[6], acc[7]};
      lo *= scale;
      hi *= scale;
      if (accumulate) { lo += v[0]; hi += v[1]; }
      v[0] = lo;
      v[1] = hi;
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < n) p[e] = acc[e] * scale + (accumulate ? p[e] : 0.f);
    }
  } else {
    elem_t* p = (elem_t*)g.dtable + (int64_t)id * g.h + c;
    elemx8 o, old = {};
    if (accumulate) old = load_chunk(p, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (elem_t)(acc[e] * scale + (float)old[e]);
    store_chunk(p, o, n);
  }
}
__device__ __forceinline__ void add_chunk(float (&acc)[8], const elemx8& v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] += (float)v[e];
}

template <bool FP32, int PIECE>
__global__ __launch_bounds__(256) void embedding_bwd_sum_kernel(const TableGrad g) {
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = (int)(w / g.col_chunks), c = (int)(w - (int64_t)piece * g.col_chunks) * SUM_COLS + 8 * lane, n = g.h - c;
  if (piece >= g.pieces) return;
  const int first = piece * PIECE, count = min(PIECE, g.T - first);
  const int mine = first + min(lane, count - 1);
  const int lane_id = g.ids[mine], lane_row = g.order[mine];
  const int before = first > 0 ? g.ids[first - 1] : -1, behind = first + count < g.T ? g.ids[first + count] : -1;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  bool from_start = true;                               // the run at hand began with the piece
#pragma unroll 1
  for (int b = 0; b < count; b += SUM_BATCH) {
    // Ids and rows as scalars, in front of every branch that lanes take differently: in such a branch the registers of lanes that
    // are not in it may hold anything.  Places past the last token repeat it, and are not added.
    int id[SUM_BATCH + 1], row[SUM_BATCH];
#pragma unroll
    for (int k = 0; k < SUM_BATCH; ++k) {
      id[k] = __builtin_amdgcn_readlane(lane_id, b + k);
      row[k] = __builtin_amdgcn_readlane(lane_row, b + k);
    }
    id[SUM_BATCH] = b + SUM_BATCH < count ? __builtin_amdgcn_readlane(lane_id, min(b + SUM_BATCH, 63)) : behind;
    elemx8 v[SUM_BATCH];
    if (n >= 8) {
#pragma unroll
      for (int k = 0; k < SUM_BATCH; ++k) v[k] = *reinterpret_cast<const elemx8_any*>(g.dout + (int64_t)row[k] * g.ld_dout + c);
    } else if (n > 0) {
      // the lane of the last, shorter chunk, element by element
#pragma unroll
      for (int k = 0; k < SUM_BATCH; ++k) v[k] = load_chunk(g.dout + (int64_t)row[k] * g.ld_dout + c, n);
    }
#pragma unroll
    for (int i = 0; i < SUM_BATCH; ++i) {
      if (b + i < count) {
        const bool final = b + i + 1 == count;
        const int cur = id[i], next = final ? behind : id[i + 1];
        add_chunk(acc, v[i]);
        if (next != cur || final) {
          const bool head = from_start && before == cur, tail = next == cur;
          if (n > 0) {
            if (!head && !tail) store_table_row<FP32>(g, cur, c, n, acc, g.scale);
            else {
              float* p = g.partial + ((int64_t)piece * 2 + (head ? 0 : 1)) * g.h + c;
              if (n >= 8) {
                ((floatx4_any*)p)[0] = floatx4{acc[0], acc[1], acc[2], acc[3]};
                ((floatx4_any*)p)[1] = floatx4{acc[4], acc[5], acc[6], acc[7]};
              } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                  if (e < n) p[e] = acc[e];
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = 0.f;
          from_start = false;
        }
      }
    }
  }
}

// Runs that cross pieces.  One workgroup per piece and 512 columns; it has work if a run begins in its piece and crosses the
// end.  The run's parts in the following pieces are shared out to the four waves in order, and the waves' sums added in order.
template <bool FP32, int PIECE>
__global__ __launch_bounds__(256) void embedding_bwd_join_kernel(const TableGrad g) {
  __shared__ float sums[3][64][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), piece = blockIdx.x;
  const int c = blockIdx.y * SUM_COLS + 8 * lane, n = g.h - c;
  const int first = piece * PIECE, last = first + PIECE - 1;
  if (last + 1 >= g.T) return;
  const int id = g.ids[last];
  if (g.ids[last + 1] != id || (first > 0 && g.ids[first - 1] == id && g.ids[first] == id)) return;
  // pieces that begin with this id, 64 at a time
  int parts = 1;                                        // partial[piece][1], then partial[piece + 1 ..][0]
  for (int p = piece + 1;; p += 64) {
    const unsigned long long same = __ballot(p + lane < g.pieces && g.ids[min(p + lane, g.pieces - 1) * PIECE] == id);
    parts += ~same ? __ffsll(~same) - 1 : 64;
    if (~same) break;
  }
  const int share = (parts + 3) / 4, p0 = wave * share, p1 = min(parts, p0 + share);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  auto part = [&](int q) { return g.partial + ((int64_t)(piece + q) * 2 + (q == 0 ? 1 : 0)) * g.h + c; };
  if (n >= 8) {
    int q = p0;
    for (; q + 8 <= p1; q += 8) {
      floatx4 v[8][2];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const floatx4_any* const p = (const floatx4_any*)part(q + k);
        v[k][0] = p[0];
        v[k][1] = p[1];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += v[k][e >> 2][e & 3];
    }
    for (; q < p1; ++q) {
      const floatx4_any* const p = (const floatx4_any*)part(q);
      const floatx4 lo = p[0], hi = p[1];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += e < 4 ? lo[e] : hi[e - 4];
    }
  } else if (n > 0) {
    for (int q = p0; q < p1; ++q) {
      const float* const p = part(q);
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < n) acc[e] += p[e];
    }
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
  store_table_row<FP32>(g, id, c, n, acc, g.scale);
}

// Up to FEW_MAX tokens: no sort, and every row of the result has one writer.  A workgroup takes ROWS rows and 512 columns, marks
// in bit masks which tokens name them, and its waves add the marked rows of dout in token order, eight in flight; the tokens
// of a row with many are shared out to the four waves.  The rows are those of the table in turn (`all`: rows without tokens are
// cleared, so this is the only launch), or the ids of ROWS tokens that no earlier token has.  200 x 384 of 1000 rows takes
// 5.2 to 5.7 us in the kernel trace, a pass with its host part 12.5 (sorted, in seven launches, 58); 512 x 1024 of 51200 rows 30 us
// (65 if all are one id), sorted 26 (23).  A table of 51200 x 4096 row by row took 179 us, cleared by streaming stores and then one
// token 77.
constexpr int FEW_MAX = 256, FEW_SHARED = 32;
template <bool FP32, int ROWS>
__global__ __launch_bounds__(256) void embedding_bwd_few_kernel(const TableGrad g, int all) {
  __shared__ unsigned long long mask[ROWS][FEW_MAX / 64];
  __shared__ float sums[3][64][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = blockIdx.x * ROWS, c = blockIdx.y * SUM_COLS + 8 * lane, n = g.h - c, words = (g.T + 63) / 64;
  auto row_id = [&](int r) {                            // -1: none
    const int i = r0 + r;
    if (all) return i < g.vocab ? i : -1;
    return i < g.T ? clamp_token(g.ids[i], g.vocab) : -1;
  };
  int want[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) want[r] = row_id(r);
  for (int w = wave; w < words; w += 4) {
    const int t = w * 64 + lane, id = t < g.T ? clamp_token(g.ids[t], g.vocab) : -2;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const unsigned long long m = __ballot(id == want[r]);
      if (lane == 0) mask[r][w] = m;
    }
  }
  __syncthreads();
  // adds the tokens marked in words [w0, w1)
  auto add = [&](int r, int w0, int w1, float (&acc)[8]) {
    int rows[8], k = 0;
    auto flush = [&]() {
      elemx8 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < k && n > 0) v[i] = load_chunk(g.dout + (int64_t)rows[i] * g.ld_dout + c, n);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < k) add_chunk(acc, v[i]);
      k = 0;
    };
    for (int w = w0; w < w1; ++w) {
      unsigned long long m = mask[r][w];
      m = (unsigned long long)__builtin_amdgcn_readfirstlane((int)(m >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
      while (m) {
        const int t = w * 64 + __ffsll(m) - 1;
        m &= m - 1;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i == k) rows[i] = t;
        if (++k == 8) flush();
      }
    }
    if (k) flush();
  };
#pragma unroll 1
  for (int r = 0; r < ROWS; ++r) {
    const int id = row_id(r);
    if (id < 0) break;
    int tokens = 0, earlier = 0;
    for (int w = 0; w < words; ++w) {
      const unsigned long long m = mask[r][w];
      tokens += __popcll(m);
      if (!all && w * 64 < r0 + r) earlier |= (w * 64 + 64 <= r0 + r ? m : m & ((1ull << ((r0 + r) & 63)) - 1)) != 0;
    }
    if (earlier) continue;
    const bool shared = tokens > FEW_SHARED;            // the same for the whole workgroup
    if (!shared && (r & 3) != wave) continue;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    if (!shared) add(r, 0, words, acc);
    else {
      const int part = (words + 3) / 4;
      add(r, min(words, wave * part), min(words, (wave + 1) * part), acc);
      __syncthreads();
      if (wave > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave - 1][lane][e] = acc[e];
      }
      __syncthreads();
      if (wave > 0) continue;
#pragma unroll
      for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += sums[w][lane][e];
    }
    if (n > 0) store_table_row<FP32>(g, id, c, n, acc, tokens ? g.scale : 0.f);      // no tokens: zeros, whatever the scale
  }
}

__global__ __launch_bounds__(256) void embedding_clear_kernel(uint16_t* p, int64_t halves) {
  clear_table<256>(p, halves, blockIdx.x, gridDim.x);
}

// Workspace, in this order, each part at a multiple of 256 bytes.
struct EmbeddingWs {
  int blocks, per_block, bits, pieces;
  uint64_t keys[2], index[2], hist, partial, bytes;
};
static EmbeddingWs embedding_ws(int64_t T, int64_t h, int64_t vocab) {
  EmbeddingWs w = {};
  w.bits = 1;
  while (((int64_t)1 << w.bits) < vocab) ++w.bits;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t r = at; at += (bytes + 255) / 256 * 256; return r; };
  if (T > FEW_MAX) {
    const int64_t tiles = (T + SORT_TILE - 1) / SORT_TILE;
    const int64_t per = (tiles + SORT_MAX_BLOCKS - 1) / SORT_MAX_BLOCKS;
    const int piece = T >= MANY_TOKENS ? PIECE_MANY : PIECE_FEW;
    w.per_block = (int)(per * SORT_TILE);
    w.blocks = (int)((tiles + per - 1) / per);
    w.pieces = (int)((T + piece - 1) / piece);
    for (int i = 0; i < 2; ++i) { w.keys[i] = take(4 * (uint64_t)T); w.index[i] = take(4 * (uint64_t)T); }
    w.hist = take(4ull * w.blocks << SORT_MAX_BITS);
    w.partial = take(8ull * w.pieces * (uint64_t)h);
  }
  w.bytes = std::max<uint64_t>(at, 16);
  return w;
}
uint64_t embedding_bwd_ws_bytes(int64_t T, int64_t h, int64_t vocab) { return embedding_ws(T, h, vocab).bytes; }

template <bool FP32, int PIECE>
static void launch_embedding_sums(const TableGrad& g, hipStream_t s) {
  hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_sum_kernel<FP32, PIECE>), dim3((unsigned)(((int64_t)g.pieces * g.col_chunks + 3) / 4)),
                     dim3(256), 0, s, g);
  hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_join_kernel<FP32, PIECE>), dim3(g.pieces, g.col_chunks), dim3(256), 0, s, g);
}

template <bool FP32>
static hipError_t launch_embedding_bwd_t(TableGrad g, const EmbeddingWs& w, const int* tokens, char* ws, hipStream_t s) {
  const int64_t T = g.T, halves = (int64_t)g.vocab * g.h * (FP32 ? 2 : 1);
  auto clear = [&]() {
    hipLaunchKernelGGL(embedding_clear_kernel, dim3((unsigned)std::min<int64_t>(1 << 20, (halves + 8191) / 8192)), dim3(256), 0, s,
                       (uint16_t*)g.dtable, halves);
  };
  if (T <= FEW_MAX) {
    g.ids = tokens;
    // rows of a small table one by one (every workgroup looks at every token), else the table cleared by a launch of its own
    const bool all = !g.accumulate && g.vocab <= 2048;
    if (!g.accumulate && !all) clear();
    hipLaunchKernelGGL(HIP_KERNEL_NAME(embedding_bwd_few_kernel<FP32, 4>), dim3((unsigned)(((all ? g.vocab : T) + 3) / 4), g.col_chunks), dim3(256),
                       0, s, g, (int)all);
    return hipGetLastError();
  }
  int t_bits = 1;
  while (((int64_t)1 << t_bits) < T) ++t_bits;
  const int key_bits = std::max(0, w.bits - SORT_SHARES_LOG);
  if (T <= SORT_SHARE_MAX && key_bits + t_bits <= 32) {
    const int shares = std::min(SORT_SHARES, g.vocab);
    const int64_t clearing = g.accumulate ? 0 : std::min<int64_t>(1 << 20, (halves + 32767) / 32768);
    hipLaunchKernelGGL(embedding_sort_share_kernel, dim3((unsigned)(shares + clearing)), dim3(SORT_SHARE_THREADS), 0, s, g.T, g.vocab, key_bits,
                       shares, t_bits, tokens, (int*)(ws + w.keys[0]), (int*)(ws + w.index[0]), (uint16_t*)g.dtable, halves);
    g.ids = (const int*)(ws + w.keys[0]); g.order = (const int*)(ws + w.index[0]);
  } else {
    if (!g.accumulate) clear();
    const int passes = (w.bits + SORT_MAX_BITS - 1) / SORT_MAX_BITS;
    for (int i = 0, shift = 0; i < passes; ++i) {
      SortPass p;
      p.T = g.T; p.per_block = w.per_block; p.vocab = g.vocab;
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
    g.ids = (const int*)(ws + w.keys[(passes - 1) & 1]); g.order = (const int*)(ws + w.index[(passes - 1) & 1]);
  }
  g.partial = (float*)(ws + w.partial);
  if (T >= MANY_TOKENS) launch_embedding_sums<FP32, PIECE_MANY>(g, s);
  else launch_embedding_sums<FP32, PIECE_FEW>(g, s);
  return hipGetLastError();
}

hipError_t launch_embedding_bwd(int64_t T, int64_t h, int64_t vocab, const int* tokens, const void* dout, int64_t ld_dout, float scale,
                                void* dtable, bool fp32, bool accumulate, void* workspace, hipStream_t s) {
  const EmbeddingWs w = embedding_ws(T, h, vocab);
  TableGrad g = {};
  g.T = (int)T; g.h = (int)h; g.vocab = (int)vocab; g.pieces = w.pieces; g.col_chunks = (int)((h + SUM_COLS - 1) / SUM_COLS);
  g.dout = (const elem_t*)dout; g.ld_dout = ld_dout; g.scale = scale; g.accumulate = accumulate; g.dtable = dtable;
  return fp32 ? launch_embedding_bwd_t<true>(g, w, tokens, (char*)workspace, s) : launch_embedding_bwd_t<false>(g, w, tokens, (char*)workspace, s);
}

}  // namespace axonn
