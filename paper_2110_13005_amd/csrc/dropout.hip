// Dropout from a counter-based generator.  Whether an element is kept is a function of (seed, offset, row, column): the
// mask is never stored, and the backward pass and a regenerated forward pass form it again.
//
// Columns 8g..8g+7 of row r take the eight 16-bit halves of the four words
//   Philox4x32-10(key = seed, counter = (g, r, offset low, offset high)),      low half of word 0 first
// (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), and an element is kept if its half is at
// least thr = round(65536 p).  Kept elements are multiplied by 65536 / (65536 - thr), the reciprocal of the probability with
// which they are kept, so the rounding of p leaves the expectation as it is.  32 bits per element would be twice the generator's
// work, which then bounds the kernel; this way HBM does: 16384 x 5120 with a residual in 89 to 93 us (5.4 to 5.7 TB/s), 4096 x 4512
// without in 15.
#include "rows.h"
#include "host_logic.h"
#include <type_traits>

namespace axonn {

constexpr int DO_THREADS = 256;

struct DropoutArgs {
  int64_t n_chunks;                 // of all rows
  uint32_t row_chunks, row_recip;   // chunks of one row, and their reciprocal
  int h;
  const elem_t *x, *res;
  elem_t* out;
  int64_t ld_x, ld_res, ld_out;
  uint32_t threshold, key0, key1;
  float scale;
  uint64_t offset;
  const uint64_t* offset_dev;
};

__device__ __forceinline__ void philox4x32_10(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c[0], p1 = (uint64_t)0xCD9E8D57u * c[2];
    const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(p0 >> 32) ^ c[3] ^ k1;
    c[0] = n0; c[1] = (uint32_t)p1; c[2] = n2; c[3] = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// DO_CHUNKS: chunks of 8 elements per lane.
template <bool RES, int DO_CHUNKS>
__global__ __launch_bounds__(DO_THREADS) void dropout_kernel(const DropoutArgs g) {
  const int64_t base = (int64_t)blockIdx.x * (DO_THREADS * DO_CHUNKS);
  const int64_t row0 = base / g.row_chunks;
  const uint32_t col0 = (uint32_t)(base - row0 * g.row_chunks);
  const uint64_t offset = g.offset + (g.offset_dev ? *g.offset_dev : 0);
  elemx8 xv[DO_CHUNKS], rv[DO_CHUNKS];
  int64_t row[DO_CHUNKS];
  uint32_t col[DO_CHUNKS];
  int n[DO_CHUNKS];                                   // elements of the chunk; none behind the last
#pragma unroll
  for (int u = 0; u < DO_CHUNKS; ++u) {
    const uint32_t i = u * DO_THREADS + threadIdx.x, t = col0 + i, q = host::recip_div(t, g.row_chunks, g.row_recip);
    row[u] = row0 + q;
    col[u] = t - q * g.row_chunks;
    n[u] = base + i < g.n_chunks ? g.h - (int)(8 * col[u]) : 0;
    if (n[u] > 0) {
      xv[u] = load_chunk(g.x + row[u] * g.ld_x + 8 * col[u], n[u]);
      if (RES) rv[u] = load_chunk(g.res + row[u] * g.ld_res + 8 * col[u], n[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < DO_CHUNKS; ++u) {
    if (n[u] <= 0) continue;
    uint32_t w[4] = {col[u], (uint32_t)row[u], (uint32_t)offset, (uint32_t)(offset >> 32)};
    philox4x32_10(w, g.key0, g.key1);
    elemx8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t half = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
      // a dropped element is zero whatever it was, an infinity or NaN too
      float y = half >= g.threshold ? (float)xv[u][e] * g.scale : 0.f;
      if (RES) y += (float)rv[u][e];
      o[e] = (elem_t)y;
    }
    store_chunk(g.out + row[u] * g.ld_out + 8 * col[u], o, n[u]);
  }
}

hipError_t launch_dropout(int64_t T, int64_t h, const void* x, int64_t ld_x, const void* res, int64_t ld_res, uint32_t threshold,
                          uint64_t seed, uint64_t offset, const uint64_t* offset_dev, void* out, int64_t ld_out, hipStream_t s) {
  DropoutArgs g;
  g.row_chunks = (uint32_t)((h + 7) / 8);
  g.row_recip = host::recip_of(g.row_chunks);
  g.n_chunks = T * (int64_t)g.row_chunks;
  g.h = (int)h;
  g.x = (const elem_t*)x; g.res = (const elem_t*)res; g.out = (elem_t*)out;
  g.ld_x = ld_x; g.ld_res = ld_res; g.ld_out = ld_out;
  g.threshold = threshold;
  g.key0 = (uint32_t)seed; g.key1 = (uint32_t)(seed >> 32);
  g.scale = threshold < 65536u ? (float)(65536.0 / (65536.0 - threshold)) : 0.f;
  g.offset = offset; g.offset_dev = offset_dev;
  // four chunks per lane (their loads in flight together) where that leaves every CU two workgroups; else one: 7 x 1001 takes 2.9 us
  // in the kernel trace, with four 6.3
  const auto launch = [&](auto chunks) {
    constexpr int CHUNKS = decltype(chunks)::value;
    const dim3 blocks((unsigned)((g.n_chunks + DO_THREADS * CHUNKS - 1) / (DO_THREADS * CHUNKS)));
    if (res) hipLaunchKernelGGL(HIP_KERNEL_NAME(dropout_kernel<true, CHUNKS>), blocks, dim3(DO_THREADS), 0, s, g);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(dropout_kernel<false, CHUNKS>), blocks, dim3(DO_THREADS), 0, s, g);
  };
  if (g.n_chunks >= 512 * DO_THREADS * 4) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

}  // namespace axonn
