// Fused causal self-attention of sequences of one length for gfx950: forward (online softmax, never materialises the
// s x s matrix in HBM) and backward (probabilities recomputed from the stored log-sum-exp).  What a workgroup does is in
// attention_core.h; here are which tile it takes, the kernels and their launches.
#include "attention_core.h"
#include "host_logic.h"

namespace axonn {

// Work assignment of the attention kernels: block id of a 1-D grid of n_tiles * n_bh blocks -> (rank of
// the tile, batch*head index).  Workgroups are dealt round-robin to the 8 XCDs, each with an L2 of its
// own, so XCD x gets ids x, x+8, ...: those are mapped to a contiguous range of (batch, head) pairs, so
// that the K/V (or Q/dO) rows of a head are fetched into one L2 instead of all eight; inside the range
// the tiles of rank 0 (the longest-running ones under causal masking) of every head come first.
// The divisions are by numbers whose reciprocals come with the arguments: of the instructions in front of the first copy, which
// the smallest launches feel, they were half.  2 x 4 heads of 64 x 128 forward 5.20 -> 5.12 us, of 64 x 64 4.34 -> 4.14.
struct AttnWalk { uint32_t xcds, block, heads; };   // blocks are dealt by XCD (1) or not (0); reciprocals of a block row's length and of a
__device__ __forceinline__ void attn_block(uint32_t id, uint32_t n_bh, uint32_t a, AttnWalk w, int& rank, int& bi, int& hd) {
  const uint32_t len = w.xcds ? n_bh >> 3 : n_bh, j = w.xcds ? id >> 3 : id;     // j-th block of XCD id % 8
  rank = host::recip_div(j, len, w.block);
  const uint32_t bh = j - rank * len + (w.xcds ? (id & 7) * len : 0);
  bi = host::recip_div(bh, a, w.heads);
  hd = bh - bi * a;
}

// One head of one sequence in the packed qkv [b * s, 3h] and in o / dO [b * s, h]: first row, first column.
struct DenseHead {
  int h;
  int64_t ld;
  const elem_t* q;
  int64_t row, stat;       // of the sequence in [b * s, .], of the head's first query in lse and delta
  int col;
};
__device__ __forceinline__ DenseHead dense_head(const elem_t* qkv, int s, int a, int d, int bi, int hd) {
  DenseHead r;
  r.h = a * d;
  r.ld = 3 * (int64_t)r.h;
  r.row = (int64_t)bi * s;
  r.col = hd * d;
  r.q = qkv + r.row * r.ld + r.col;
  r.stat = ((int64_t)bi * a + hd) * s;
  return r;
}

// grid: ceil(s/128) * b * a workgroups
template <int D, bool FITS>
__global__ __launch_bounds__(256, D > 128 ? 1 : 2) void attn_fwd_kernel(int s, int a, int n_bh, AttnWalk walk, int d,
                                                                        const elem_t* __restrict__ qkv,
                                                                        elem_t* __restrict__ o,
                                                                        float* __restrict__ lse) {
  __shared__ FwdLds<D> lds;
  int rank, bi, hd;
  attn_block(blockIdx.x, n_bh, a, walk, rank, bi, hd);
  const DenseHead t = dense_head(qkv, s, a, d, bi, hd);
  // longest rows first
  attn_fwd_tile<D, FITS>(lds, (s + 127) / 128 - 1 - rank, s, d, rsqrtf((float)d), t.q, t.q + t.h, t.q + 2 * t.h, t.ld,
                         o + t.row * t.h + t.col, t.h, lse + t.stat);
}

// For any head dimension d that is a multiple of 4: 16 lanes per (row, head), 4 elements per lane and step.
// (Launched in front of the one-launch backward and where d is not 64 or 128; at those the dQ kernel in a launch of its own forms
// delta itself.)
__global__ __launch_bounds__(256) void attn_delta_general_kernel(int64_t n_pairs, int s, int a, int d,
                                                                 const elem_t* __restrict__ o,
                                                                 const elem_t* __restrict__ dout,
                                                                 float* __restrict__ delta) {
  const int64_t pair = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);   // (row, head)
  const int j = threadIdx.x & 15;
  float p = 0.f;
  if (pair < n_pairs) {
    const elem_t* op = o + pair * d;          // rows are a * d long: pair * d = row * a * d + head * d
    const elem_t* dp = dout + pair * d;
    for (int c = 4 * j; c < d; c += 64) {
      p = delta_add<4, true>(p, *reinterpret_cast<const elemx4*>(op + c), *reinterpret_cast<const elemx4*>(dp + c), 0);
    }
  }
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) p += __shfl_xor(p, off, 64);
  if (pair < n_pairs && j == 0) {
    const int64_t row = pair / a;
    const int hd = (int)(pair % a);
    const int64_t bi = row / s, i = row % s;
    delta[(bi * a + hd) * s + i] = p;
  }
}

// ------------------------------------------------------------------- backward kernels
template <int D, bool FITS>
__device__ __forceinline__ void dense_dkdv(DkdvLds<D>& lds, int id, int s, int a, int n_bh, AttnWalk walk, int d,
                                           const elem_t* __restrict__ qkv, const elem_t* __restrict__ dout,
                                           const float* __restrict__ lse, const float* __restrict__ delta,
                                           elem_t* __restrict__ dqkv) {
  int rank, bi, hd;
  attn_block(id, n_bh, a, walk, rank, bi, hd);    // key tile `rank` walks n_tiles - rank query tiles: longest first
  const DenseHead t = dense_head(qkv, s, a, d, bi, hd);
  elem_t* const dk = dqkv + t.row * t.ld + t.h + t.col;
  attn_bwd_dkdv<D, FITS>(lds, rank, s, d, rsqrtf((float)d), t.q, t.q + t.h, t.q + 2 * t.h, t.ld, dout + t.row * t.h + t.col, t.h,
                         lse + t.stat, delta + t.stat, dk, dk + t.h, t.ld);
}
template <int D, bool FITS, int FORM_DELTA>
__device__ __forceinline__ void dense_dq(DqLds<D>& lds, int id, int s, int a, int n_bh, AttnWalk walk, int d,
                                         const elem_t* __restrict__ qkv, const elem_t* __restrict__ o,
                                         const elem_t* __restrict__ dout, const float* __restrict__ lse, float* delta,
                                         elem_t* __restrict__ dqkv, int by_4) {
  int rank, bi, hd;
  attn_block(id, n_bh, a, walk, rank, bi, hd);
  const DenseHead t = dense_head(qkv, s, a, d, bi, hd);
  const int64_t at = t.row * t.h + t.col;
  attn_bwd_dq<D, FITS, FORM_DELTA>(lds, (s + 127) / 128 - 1 - rank, s, d, rsqrtf((float)d), t.q, t.q + t.h, t.q + 2 * t.h, t.ld,
                                   o + at, t.h, dout + at, t.h, lse + t.stat, delta + t.stat, dqkv + t.row * t.ld + t.col, t.ld, by_4);
}
// At D = 64 two workgroups share a CU, with 160 ordinary and 96 accumulation registers per lane: at four more 8 x 16 heads of
// 64 x 1024 take 55 us for dK / dV instead of 44.  (A second argument to __launch_bounds__ does not keep it so: it makes the compiler
// halve the 256 between the two kinds and move accumulators about between the MFMAs, at distances that it does not know.)
template <int D, bool FITS>
__global__ __launch_bounds__(256) void attn_bwd_dkdv_kernel(
    int s, int a, int n_bh, AttnWalk walk, int d, const elem_t* __restrict__ qkv, const elem_t* __restrict__ dout,
    const float* __restrict__ lse, const float* __restrict__ delta, elem_t* __restrict__ dqkv) {
  __shared__ DkdvLds<D> lds;
  dense_dkdv<D, FITS>(lds, blockIdx.x, s, a, n_bh, walk, d, qkv, dout, lse, delta, dqkv);
}
template <int D, bool FITS, bool FORM_DELTA = false>
__global__ __launch_bounds__(256, D > 128 ? 1 : 2) void attn_bwd_dq_kernel(
    int s, int a, int n_bh, AttnWalk walk, int d, const elem_t* __restrict__ qkv, const elem_t* __restrict__ o,
    const elem_t* __restrict__ dout, const float* __restrict__ lse, float* __restrict__ delta,
    elem_t* __restrict__ dqkv, int by_4) {
  __shared__ DqLds<D> lds;
  dense_dq<D, FITS, FORM_DELTA ? FORM_DELTA_EXACT : READ_DELTA>(lds, blockIdx.x, s, a, n_bh, walk, d, qkv, o, dout, lse, delta, dqkv, by_4);
}
// Both at once, for problems whose tiles do not fill the chip: the first half of the workgroups forms dK and dV, the second
// dQ; delta is there already.  Each half alone is a chain of up to s / 128 (s / 64) tiles per workgroup on a part of the
// CUs; side by side they take the longer of the two times.
template <int D, bool FITS>
__global__ __launch_bounds__(256) void attn_bwd_both_kernel(
    int s, int a, int n_bh, AttnWalk walk, int d, const elem_t* __restrict__ qkv, const elem_t* __restrict__ dout,
    const float* __restrict__ lse, float* delta, elem_t* __restrict__ dqkv) {
  __shared__ union { DkdvLds<D> dkdv; DqLds<D> dq; } lds;
  const int n = gridDim.x >> 1, id = blockIdx.x;
  if (id < n) dense_dkdv<D, FITS>(lds.dkdv, id, s, a, n_bh, walk, d, qkv, dout, lse, delta, dqkv);
  else dense_dq<D, FITS, READ_DELTA>(lds.dq, id - n, s, a, n_bh, walk, d, qkv, nullptr, dout, lse, delta, dqkv, 0);
}

// ------------------------------------------------------------------------- launchers
// Head dimensions up to 64, 128 and 192 run in tiles of that many columns.  The copies into LDS and the stores take 32-bit byte
// offsets within 128 rows (FITS); longer rows, of 2.8 million columns and more, go through registers, a chunk after the other.
// Matrices start at any element.  16 heads of 128 x 2048 at a multiple of 16 bytes, 8 bytes behind one and 2 bytes behind one, us:
// forward 39.4, 39.6 and 52.2, dQ 54.0, 49.8 and 60.8, dK / dV 57.1, 53.7 and 65.9 (through registers 147, 158 and 120).
#define AXONN_ATTN_DISPATCH(KERNEL, ...)                                                                  \
  do {                                                                                                    \
    if (d <= 64) { if (fits) hipLaunchKernelGGL((KERNEL<64, true>), grid, dim3(256), 0, st, __VA_ARGS__);       \
                   else hipLaunchKernelGGL((KERNEL<64, false>), grid, dim3(256), 0, st, __VA_ARGS__); }           \
    else if (d <= 128) { if (fits) hipLaunchKernelGGL((KERNEL<128, true>), grid, dim3(256), 0, st, __VA_ARGS__); \
                         else hipLaunchKernelGGL((KERNEL<128, false>), grid, dim3(256), 0, st, __VA_ARGS__); }    \
    else { if (fits) hipLaunchKernelGGL((KERNEL<192, true>), grid, dim3(256), 0, st, __VA_ARGS__);              \
           else hipLaunchKernelGGL((KERNEL<192, false>), grid, dim3(256), 0, st, __VA_ARGS__); }                  \
  } while (0)
static bool offsets_fit(int64_t h) { return 128 * 3 * h * 2 < (int64_t(1) << 31); }

// dK / dV and dQ as one launch while the workgroups of both find a CU each (above 64 columns the dK / dV one leaves no room for a
// second in registers and LDS).  delta then has a launch of its own, which the dQ kernel spares at 64 and 128 columns.  Backward in
// separate launches / in one, us: 16 heads of 64 x 1024 (128 tiles) 37.2 / 26.5, of 128 x 1024 53.5 / 34.4; 16 of 188 x 512 49.2 / 27.4; 3 of
// 128 x 200, 2 sequences 22.8 / 14.0; 4 of 64 x 128, 2 sequences 12.7 / 9.0.  Beyond the line one launch is the faster one, too:
// 24 heads of 64 x 1024 (192 tiles) 37.7 / 29.2, of 128 x 1024 55.4 / 40.9, of 188 x 1024 88.3 / 57.7; 16 of 64 x 2048 (256) 64.8 / 58.8.  The line
// also says in which order delta is summed (by_4), which these shapes keep.
constexpr int kBothMaxTiles = 128;

static AttnWalk attn_walk(int n_bh, int a) {
  const bool xcds = n_bh % 8 == 0;             // and with it the number of blocks
  return {xcds ? 1u : 0u, host::recip_of(xcds ? n_bh / 8 : n_bh), host::recip_of(a)};
}
static bool head_dim_supported(int d) { return d >= 4 && d <= 192 && d % 4 == 0; }

hipError_t launch_attention_fwd(int b, int s, int a, int d, const void* qkv, void* o, float* lse,
                                hipStream_t st) {
  if (!head_dim_supported(d)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(((s + 127) / 128) * b * a));
  const bool fits = offsets_fit((int64_t)a * d);
  const AttnWalk walk = attn_walk(b * a, a);
  AXONN_ATTN_DISPATCH(attn_fwd_kernel, s, a, b * a, walk, d, (const elem_t*)qkv, (elem_t*)o, lse);
  return hipGetLastError();
}

hipError_t launch_attention_bwd(int b, int s, int a, int d, const void* qkv, const void* o,
                                const float* lse, const void* dout, void* dqkv, float* delta,
                                hipStream_t st, int rule_b) {
  if (!head_dim_supported(d)) return hipErrorInvalidValue;
  const int n_tiles = ((s + 127) / 128) * b * a;
  const bool both = n_tiles <= kBothMaxTiles;
  const bool fits = offsets_fit((int64_t)a * d);
  const AttnWalk walk = attn_walk(b * a, a);
  // for d = 64 and 128 the dQ kernel forms delta itself and runs first; sequences that run together get the sums in the order
  // that rule_b of them have
  const bool dq_forms_delta = !both && (d == 64 || d == 128);
  const int by_4 = ((s + 127) / 128) * (rule_b > 0 ? rule_b : b) * a <= kBothMaxTiles;
  hipError_t e;
  dim3 grid((unsigned)n_tiles);
  if (dq_forms_delta) {
#define AXONN_ATTN_DQ(D, FITS)                                                                                                 \
  hipLaunchKernelGGL((attn_bwd_dq_kernel<D, FITS, true>), grid, dim3(256), 0, st, s, a, b * a, walk, d, (const elem_t*)qkv,          \
                     (const elem_t*)o, (const elem_t*)dout, lse, delta, (elem_t*)dqkv, by_4)
    if (d == 64) { if (fits) AXONN_ATTN_DQ(64, true); else AXONN_ATTN_DQ(64, false); }
    else { if (fits) AXONN_ATTN_DQ(128, true); else AXONN_ATTN_DQ(128, false); }
#undef AXONN_ATTN_DQ
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    AXONN_ATTN_DISPATCH(attn_bwd_dkdv_kernel, s, a, b * a, walk, d, (const elem_t*)qkv, (const elem_t*)dout, lse, (const float*)delta, (elem_t*)dqkv);
    return hipGetLastError();
  }
  const int64_t n_pairs = (int64_t)b * s * a;
  hipLaunchKernelGGL(attn_delta_general_kernel, dim3((unsigned)((n_pairs + 15) / 16)), dim3(256), 0, st, n_pairs, s, a, d,
                     (const elem_t*)o, (const elem_t*)dout, delta);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (both) {
    grid = dim3(2u * (unsigned)n_tiles);
    AXONN_ATTN_DISPATCH(attn_bwd_both_kernel, s, a, b * a, walk, d, (const elem_t*)qkv, (const elem_t*)dout, lse, delta, (elem_t*)dqkv);
    return hipGetLastError();
  }
  AXONN_ATTN_DISPATCH(attn_bwd_dkdv_kernel, s, a, b * a, walk, d, (const elem_t*)qkv, (const elem_t*)dout, lse, (const float*)delta, (elem_t*)dqkv);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  AXONN_ATTN_DISPATCH(attn_bwd_dq_kernel, s, a, b * a, walk, d, (const elem_t*)qkv, (const elem_t*)o, (const elem_t*)dout, lse, delta, (elem_t*)dqkv, 0);
  return hipGetLastError();
}
#undef AXONN_ATTN_DISPATCH

}  // namespace axonn
