// Linear maps in 8-bit floating point (e4m3: 4 bits of exponent, 3 of significand, largest 448) with a scale for each block of
// 128 elements along the contraction.
//
// The scale is a power of two, 2^e with the least e for which the block's largest magnitude is at most 448 * 2^e, stored as the
// byte e + 127: the form in which gfx950's scaled MFMA takes it as an operand, so the product's loop has no vector
// instruction for it.  x * 2^-e is exact, so a code is one rounding of x (to nearest, ties to even), however it is formed.
//
// Quantised matrices: codes [rows][Kp], Kp = K rounded up to 128, zeros behind K; scales [rows][S], S = Kp / 128 rounded up to
// 4: a row's scales of four blocks are one 32-bit word, of which the MFMA picks a byte by an immediate.
#include "rows.h"
#include "host_logic.h"
#include <algorithm>

namespace axonn {

constexpr int FB = 128;                      // elements of a block

// ---------------------------------------------------------------------------------------------------------- quantiser
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
#ifdef AXONN_ELEM_FP16
typedef _Float16 elem_pair __attribute__((ext_vector_type(2)));
#define AXONN_CVT_PK_FP8 __builtin_amdgcn_cvt_scalef32_pk_fp8_f16
constexpr uint32_t kInfinity16 = 0x7c00;
#else
typedef __bf16 elem_pair __attribute__((ext_vector_type(2)));
#define AXONN_CVT_PK_FP8 __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16
constexpr uint32_t kInfinity16 = 0x7f80;
#endif

// Largest magnitude of both halves of a word and m's, as bit patterns (of non-negative numbers their order is the integers').
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t m, uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
}
// The same without what is not finite.
__device__ __forceinline__ uint32_t finite_magnitudes(uint32_t m, uint32_t w) {
  w &= 0x7fff7fffu;
  if ((w & 0xffffu) >= kInfinity16) w &= 0xffff0000u;
  if ((w >> 16) >= kInfinity16) w &= 0xffffu;
  return max_magnitudes(m, w);
}
// e of a block from the bit pattern of its largest finite magnitude.
__device__ __forceinline__ int block_exponent(uint32_t pattern) {
  const float amax = (float)__builtin_bit_cast(elem_t, (uint16_t)pattern);
  const uint32_t b = __float_as_uint(amax);
  return max(-127, (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0));       // 448 = 1.75 * 2^8
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(e == -127 ? 0x400000u : (uint32_t)(e + 127) << 23); }   // -127 <= e <= 127
// Codes of the four elements of two words, the first in the low byte: one rounding of x / scale to nearest, ties to even
// (v_cvt_scalef32_pk_fp8_*, compared with the definition for every 16-bit pattern).
__device__ __forceinline__ uint32_t encode4(uint32_t lo, uint32_t hi, float scale) {
  s16x2 r = {0, 0};
  r = AXONN_CVT_PK_FP8(r, __builtin_bit_cast(elem_pair, lo), scale, false);
  r = AXONN_CVT_PK_FP8(r, __builtin_bit_cast(elem_pair, hi), scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// Puts 0x7f in the codes `c` of the infinities and NaN among the four elements.
__device__ __forceinline__ uint32_t mark_not_finite(uint32_t c, uint32_t lo, uint32_t hi) {
  if ((lo & 0x7fffu) >= kInfinity16) c = (c & 0xffffff00u) | 0x7fu;
  if ((lo >> 16 & 0x7fffu) >= kInfinity16) c = (c & 0xffff00ffu) | 0x7f00u;
  if ((hi & 0x7fffu) >= kInfinity16) c = (c & 0xff00ffffu) | 0x7f0000u;
  if ((hi >> 16 & 0x7fffu) >= kInfinity16) c = (c & 0x00ffffffu) | 0x7f000000u;
  return c;
}

struct QuantArgs {
  int R, C;                 // rows and columns of x
  const elem_t* x;
  int64_t ld_x;
  uint8_t *q, *scale;       // [R][Cp], [R][S]
  uint8_t *q_t, *scale_t;   // [C][Rp], [C][S_t]
  int64_t Cp, S, Rp, S_t;
};

// The codes of a lane's chunk of 8 elements, one of the 16 lanes that share a block; e: the block's exponent.
__device__ __forceinline__ u32x2 encode_chunk(u32x4 w, int& e) {
  uint32_t m = max_magnitudes(max_magnitudes(max_magnitudes(w[0] & 0x7fff7fffu, w[1]), w[2]), w[3]);
  m = max(m & 0xffffu, m >> 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  if (!__any(m >= kInfinity16)) {
    e = block_exponent(m);
    const float s = exp2_int(e);
    return u32x2{encode4(w[0], w[1], s), encode4(w[2], w[3], s)};
  }
  m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = finite_magnitudes(m, w[i]);
  m = max(m & 0xffffu, m >> 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  e = block_exponent(m);
  const float s = exp2_int(e);
  return u32x2{mark_not_finite(encode4(w[0], w[1], s), w[0], w[1]), mark_not_finite(encode4(w[2], w[3], s), w[2], w[3])};
}

// Rows alone: a wave takes 512 columns (four blocks, one word of scales) of QR_ROWS rows.  HBM-bound: 8192 x 5120 in 21.4 us
// (5.9 TB/s), 8192 x 20480 83 (6.0), 2047 x 8192 10.5, 200 x 392 4.5 by launches one behind the other; 1, 4 and 8 rows per wave
// 23.5, 22.2, 24.0 for the first, 4.7, 5.3, 4.9 for the last.
constexpr int QR_ROWS = 2;
__global__ __launch_bounds__(256) void fp8_quantize_rows_kernel(const QuantArgs g) {
  const int lane = threadIdx.x & 63, quads = (int)(g.S / 4);
  const int group = blockIdx.x / quads, quad = blockIdx.x - group * quads;
  const int row0 = (group * 4 + (threadIdx.x >> 6)) * QR_ROWS, c = quad * 512 + 8 * lane, n = g.C - c;
  u32x4 w[QR_ROWS];
#pragma unroll
  for (int i = 0; i < QR_ROWS; ++i) {
    w[i] = u32x4{0, 0, 0, 0};
    if (row0 + i < g.R && n > 0) w[i] = __builtin_bit_cast(u32x4, load_chunk(g.x + (int64_t)(row0 + i) * g.ld_x + c, n));
  }
#pragma unroll
  for (int i = 0; i < QR_ROWS; ++i) {
    if (row0 + i >= g.R) return;
    int e;
    const u32x2 codes = encode_chunk(w[i], e);
    // blocks behind the last hold zeros: byte 0
    const uint32_t b = (uint32_t)(e + 127);
    const uint32_t word = __builtin_amdgcn_readlane(b, 0) | __builtin_amdgcn_readlane(b, 16) << 8 | __builtin_amdgcn_readlane(b, 32) << 16 |
                          __builtin_amdgcn_readlane(b, 48) << 24;
    if (c < g.Cp) *reinterpret_cast<u32x2*>(g.q + (int64_t)(row0 + i) * g.Cp + c) = codes;
    if (lane == 0) *reinterpret_cast<uint32_t*>(g.scale + (int64_t)(row0 + i) * g.S + 4 * quad) = word;
  }
}

// The transpose, and with ROWS the rows too, of a block of 128 x 128 elements per workgroup, read once.  The rows' codes come
// straight from the registers; the columns go through LDS: a thread has two adjacent columns (one word per row) of a quarter of
// the rows.  Their codes lie in LDS with 16-byte chunk k of column c at k ^ (c / 2 % 8), without bank conflicts both ways.
// Scale bytes behind the last block are cleared by the workgroup of that block.  HBM-bound: 16384 x 5120 in 71 us (4.7 TB/s)
// with the rows, 47 (5.3) without; 2047 x 8192 17.7 and 12.4.
constexpr int QT_LD = FB + 8;                // elements of an LDS row
template <bool ROWS>
__global__ __launch_bounds__(256, 4) void fp8_quantize_tile_kernel(const QuantArgs g) {
  __shared__ __align__(16) char smem[FB * QT_LD * 2];
  __shared__ uint32_t col_max[4][FB / 2];
  elem_t* const tile = (elem_t*)smem;
  const int tid = threadIdx.x;
  const int blocks_c = (int)(g.Cp / FB), by = blockIdx.x / blocks_c, bx = blockIdx.x - by * blocks_c;
  const int c0 = bx * FB, r0 = by * FB, ch = tid & 15, n = g.C - (c0 + 8 * ch);
  u32x4 w[8];
  const elem_t* const from = g.x + (int64_t)(r0 + (tid >> 4)) * g.ld_x + c0 + 8 * ch;
  elem_t* const mine = tile + (tid >> 4) * QT_LD + 8 * ch;
  if (r0 + FB <= g.R && c0 + FB <= g.C) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const elemx8_any*>(from + (int64_t)(16 * i) * g.ld_x));
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(mine + 16 * i * QT_LD) = w[i];
  } else {
    // at the edges chunk by chunk: element-wise loads of all eight at once take more registers than there are
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      elemx8 v = {};
      if (r0 + 16 * i + (tid >> 4) < g.R && n > 0) v = load_chunk(from + (int64_t)(16 * i) * g.ld_x, n);
      *reinterpret_cast<elemx8*>(mine + 16 * i * QT_LD) = v;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const u32x4*>(mine + 16 * i * QT_LD);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = r0 + 16 * i + (tid >> 4);
    if (ROWS) {
      int e;
      const u32x2 codes = encode_chunk(w[i], e);
      if (row < g.R) {
        *reinterpret_cast<u32x2*>(g.q + (int64_t)row * g.Cp + c0 + 8 * ch) = codes;
        if (ch == 0) g.scale[(int64_t)row * g.S + bx] = (uint8_t)(e + 127);
        else if (bx == blocks_c - 1 && bx + ch < g.S) g.scale[(int64_t)row * g.S + bx + ch] = 0;
      }
    }
  }
  __syncthreads();
  const int pair = tid & 63, quarter = tid >> 6;
  uint32_t v[32], m = 0;
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    v[r] = *reinterpret_cast<const uint32_t*>(tile + (quarter * 32 + r) * QT_LD + 2 * pair);
    m = max_magnitudes(m, v[r]);
  }
  const bool odd_values = __syncthreads_or((m & 0xffffu) >= kInfinity16 || m >> 16 >= kInfinity16);
  if (odd_values) {
    m = 0;
#pragma unroll
    for (int r = 0; r < 32; ++r) m = finite_magnitudes(m, v[r]);
  }
  col_max[quarter][pair] = m;
  __syncthreads();                                       // everyone is done with the tile as well
  m = max_magnitudes(max_magnitudes(max_magnitudes(col_max[0][pair], col_max[1][pair]), col_max[2][pair]), col_max[3][pair]);
  const int e0 = block_exponent(m & 0xffffu), e1 = block_exponent(m >> 16);
  const float s0 = exp2_int(e0), s1 = exp2_int(e1);
  uint8_t* const codes_t = (uint8_t*)smem;
  auto low = [&](int i) { return __builtin_amdgcn_perm(v[i + 1], v[i], 0x05040100); };      // the left column's two rows
  auto high = [&](int i) { return __builtin_amdgcn_perm(v[i + 1], v[i], 0x07060302); };
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    u32x4 a, b;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = encode4(low(16 * k + 4 * j), low(16 * k + 4 * j + 2), s0);
      b[j] = encode4(high(16 * k + 4 * j), high(16 * k + 4 * j + 2), s1);
    }
    if (odd_values) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = mark_not_finite(a[j], low(16 * k + 4 * j), low(16 * k + 4 * j + 2));
        b[j] = mark_not_finite(b[j], high(16 * k + 4 * j), high(16 * k + 4 * j + 2));
      }
    }
    const int at = 16 * ((2 * quarter + k) ^ (pair & 7));
    *reinterpret_cast<u32x4*>(codes_t + (2 * pair) * FB + at) = a;
    *reinterpret_cast<u32x4*>(codes_t + (2 * pair + 1) * FB + at) = b;
  }
  if (quarter == 0) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int col = c0 + 2 * pair + k;
      if (col >= g.C) continue;
      g.scale_t[(int64_t)col * g.S_t + by] = (uint8_t)((k ? e1 : e0) + 127);
      if (by == (int)(g.Rp / FB) - 1)
        for (int b = by + 1; b < g.S_t; ++b) g.scale_t[(int64_t)col * g.S_t + b] = 0;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = i * 32 + (tid >> 3);
    if (c0 + col < g.C)
      *reinterpret_cast<u32x4*>(g.q_t + (int64_t)(c0 + col) * g.Rp + r0 + 16 * (tid & 7)) =
          *reinterpret_cast<const u32x4*>(codes_t + col * FB + 16 * ((tid & 7) ^ (col >> 1 & 7)));
  }
}

hipError_t launch_fp8_quantize(int64_t R, int64_t C, const void* x, int64_t ld_x, void* q, void* scale, void* q_t, void* scale_t,
                               hipStream_t s) {
  QuantArgs g;
  g.R = (int)R; g.C = (int)C; g.x = (const elem_t*)x; g.ld_x = ld_x;
  g.q = (uint8_t*)q; g.scale = (uint8_t*)scale; g.q_t = (uint8_t*)q_t; g.scale_t = (uint8_t*)scale_t;
  g.Cp = (C + FB - 1) / FB * FB; g.Rp = (R + FB - 1) / FB * FB;
  g.S = (g.Cp / FB + 3) / 4 * 4; g.S_t = (g.Rp / FB + 3) / 4 * 4;
  const unsigned tiles = (unsigned)(g.Cp / FB * (g.Rp / FB));
  if (q_t) {
    if (q) hipLaunchKernelGGL(HIP_KERNEL_NAME(fp8_quantize_tile_kernel<true>), dim3(tiles), dim3(256), 0, s, g);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(fp8_quantize_tile_kernel<false>), dim3(tiles), dim3(256), 0, s, g);
  } else {
    const int64_t quads = g.S / 4;
    hipLaunchKernelGGL(fp8_quantize_rows_kernel, dim3((unsigned)((R + 4 * QR_ROWS - 1) / (4 * QR_ROWS) * quads)), dim3(256), 0, s, g);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------------------ product
// C[M, N] = epilogue(sum_k A[m, k] B[n, k]) with v_mfma_scale_f32_16x16x128_f8f6f4: one instruction covers a block of 128, so an
// operand's scale is one byte per row of a fragment, the same in the four lanes that share the row.  Which 32 of the 128 k a
// lane holds is the same for A and B and does not matter otherwise.
// The B fragment goes first: lane l then holds row l % 16 of C and columns 4 * (l / 16) + 0..3.
//
// How exact it is: within groups of 8 k the matrix unit drops what lies more than 13 binary places below the group's largest
// product (measured: 2^16 + 2^2 gives 2^16, 2^16 + 2^3 is exact; the groups, and the instructions, are added in fp32).  Each of seven
// products loses less than 2^-13 of the largest, so a sum is off by at most 7 * 2^-13 of its products' magnitudes: on random data 1.5e-5
// of a result, but with cancellation any part of it.  16-bit results are formed this way by choice: on random data the distance from the
// exact result stays that of the rounding (bf16 1.66e-3 of the result in the root mean square with either kind of sum, fp16 2.08e-4; 1 %
// and 6 % of the elements differ, by one step), a code itself is off by up to 2^-4 of its number, and the exact way is half as fast
// (8192^3 733 to 756 us, this way 382).  Who needs the sums themselves takes 32-bit results (EPI_ACC_F32): those are formed with the bf16 MFMA,
// whose sums are exact to fp32, from codes converted in registers with their scale.
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
struct WideFrag { bf16x8 v[4]; };            // a fragment's 32 values per lane

struct Fp8Args {
  int M, N, nk;                    // nk: blocks of the contraction
  int tiles_m, tiles_n;
  int64_t Kp, S;
  const uint8_t *A, *B;
  const uint8_t *sa, *sb;
  void* C;
  int64_t ldc, ld_side;            // ld_side: of res or aux
  const elem_t *bias, *res;
  elem_t* aux;
  int accumulate;
};

template <int J>
__device__ __forceinline__ floatx4 mfma_fp8(intx8 b, intx8 a, floatx4 c, int sb, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, J, sb, J, sa);
}

// Byte J of a word of scales as the power of two it stands for.
template <int J>
__device__ __forceinline__ float scale_value(int word) { return __uint_as_float((uint32_t)(word >> 8 * J & 255) << 23); }
__device__ __forceinline__ WideFrag widen(intx8 f, float scale) {
  WideFrag w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    union { bf16x8 v; bf16x2 h[4]; } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i], scale, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i], scale, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i + 1], scale, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i + 1], scale, true);
    w.v[i] = u.v;
  }
  return w;
}

// Columns n .. n + count of row m, count <= 8: v = the sums, bv = their bias.
template <int EPI>
__device__ __forceinline__ void fp8_epilogue8(const Fp8Args& g, float (&v)[8], const float (&bv)[8], int m, int n, int count) {
  elem_t* const c = (elem_t*)g.C + (int64_t)m * g.ldc + n;
  elemx8 x = {}, out;
  if (EPI == EPI_BIAS_RES) x = load_chunk(g.res + (int64_t)m * g.ld_side + n, count);
  if (EPI == EPI_DGELU) x = load_chunk(g.aux + (int64_t)m * g.ld_side + n, count);
  if (EPI == EPI_ACC_BF16 && g.accumulate) x = load_chunk(c, count);
  if (EPI == EPI_BIAS || EPI == EPI_BIAS_RES || EPI == EPI_BIAS_GELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += bv[e];
  }
  if (EPI == EPI_BIAS_GELU) {
    elemx8 dv;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y, dy;
      gelu_with_grad_f(v[e], y, dy);
      v[e] = y;
      dv[e] = (elem_t)dy;
    }
    store_chunk(g.aux + (int64_t)m * g.ld_side + n, dv, count);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (EPI == EPI_DGELU) v[e] *= (float)x[e];
    if (EPI == EPI_BIAS_RES || EPI == EPI_ACC_BF16) v[e] += (float)x[e];
    out[e] = (elem_t)v[e];
  }
  store_chunk(c, out, count);
}

// The same for 32-bit results, four columns.
__device__ __forceinline__ void fp8_epilogue4(const Fp8Args& g, floatx4 v, int m, int n, int count) {
  typedef floatx4 floatx4_any __attribute__((aligned(4)));
  float* const p = (float*)g.C + (int64_t)m * g.ldc + n;
  if (count >= 4) {
    if (g.accumulate) v += *(const floatx4_any*)p;
    *(floatx4_any*)p = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < count) p[e] = v[e] + (g.accumulate ? p[e] : 0.f);
  }
}

// A wave's TM x TN result tiles at (m0, n0), IP tile rows at a time through `stage`, the wave's own part of LDS
// (16 * IP rows of 16 * TN floats, 16-byte chunk c of row r at c ^ (r % 8): conflict-free both ways).  Straight from the MFMA's
// layout an instruction would touch 16 rows with 32 bytes each; from LDS it stores rows of up to 256 bytes.
template <int EPI, int TM, int TN, int IP>
__device__ __forceinline__ void fp8_epilogue(const Fp8Args& g, const floatx4 (&acc)[TM][TN], float* stage, int m0, int n0, int lane) {
  constexpr int WIDTH = EPI == EPI_ACC_F32 ? 4 : 8;                  // columns of a lane
  constexpr int LD = 16 * TN, LPR = LD / WIDTH, RPI = 64 / LPR;      // lanes of a row, rows of an instruction
  const int n = n0 + WIDTH * (lane % LPR), count = g.N - n;
  float bv[8];
  {
    elemx8 b = {};
    if ((EPI == EPI_BIAS || EPI == EPI_BIAS_RES || EPI == EPI_BIAS_GELU) && g.bias && count > 0) b = load_chunk(g.bias + n, count);
#pragma unroll
    for (int e = 0; e < 8; ++e) bv[e] = (float)b[e];
  }
#pragma unroll
  for (int i0 = 0; i0 < TM; i0 += IP) {
#pragma unroll
    for (int i = 0; i < IP; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        *reinterpret_cast<floatx4*>(stage + (16 * i + (lane & 15)) * LD + 4 * ((4 * j + (lane >> 4)) ^ (lane & 7))) = acc[i0 + i][j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int t = 0; t < 16 * IP; t += RPI) {
      const int row = t + lane / LPR, m = m0 + 16 * i0 + row, c = WIDTH / 4 * (lane % LPR);
      const float* s = stage + row * LD;
      if constexpr (EPI == EPI_ACC_F32) {
        if (m < g.M && count > 0) fp8_epilogue4(g, *reinterpret_cast<const floatx4*>(s + 4 * (c ^ (row & 7))), m, n, count);
        continue;
      }
      const floatx4 lo = *reinterpret_cast<const floatx4*>(s + 4 * (c ^ (row & 7)));
      const floatx4 hi = *reinterpret_cast<const floatx4*>(s + 4 * ((c + 1) ^ (row & 7)));
      float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      if (m < g.M && count > 0) fp8_epilogue8<EPI>(g, v, bv, m, n, count);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Tile of a workgroup: contiguous runs of tiles for each XCD (workgroups go round the eight), in bands of 8 tile rows.
__device__ __forceinline__ void fp8_tile_at(const Fp8Args& g, int pid, int& tm, int& tn) {
  const int band_tiles = 8 * g.tiles_n, band = pid / band_tiles, in_band = pid - band * band_tiles;
  const int rows = min(8, g.tiles_m - band * 8);
  tm = band * 8 + in_band % rows;
  tn = in_band / rows;
}

// A ring of NS tiles of 128 bytes of k in LDS, filled by the memory pipeline; a wave's part of a tile is copied by the wave,
// 8 rows of 128 bytes per instruction.  Chunk c of row r (16 bytes) lies at slot c ^ (r % 8), so that the 16 rows of a fragment
// are read without bank conflicts.  The scales of four tiles, a word per row, are copied one round of four tiles ahead.
template <int WM, int WN, int TM, int TN, int NS, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void gemm_fp8_kernel(const Fp8Args g) {
  constexpr int W = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, STAGE = (BM + BN) * FB;
  constexpr int NA = BM / 8 / W, NB = BN / 8 / W, NC = NA + NB;      // copies of a wave per tile
  constexpr int WS = (BM + BN) / 64, WSA = BM / 64;                  // waves that copy scales, of A
  static_assert(BM / 8 % W == 0 && BN / 8 % W == 0 && (NS - 1) * NC < 64 && 4 % NS == 0, "copies");
  static_assert(BM % 64 == 0 && BN % 64 == 0 && WS <= W, "scales");
  __shared__ __align__(1024) char smem[NS * STAGE + 2 * (BM + BN) * 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  int pid = blockIdx.x, tm, tn;
  if ((gridDim.x & 7) == 0) pid = (pid & 7) * (gridDim.x >> 3) + (pid >> 3);
  fp8_tile_at(g, pid, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const uint32_t Kp = (uint32_t)g.Kp, S = (uint32_t)g.S;
  const uint32_t live_m = min(BM, g.M - m0), live_n = min(BN, g.N - n0);
  const u32x4 ra = rsrc_words(g.A + (int64_t)m0 * g.Kp, live_m * Kp), rb = rsrc_words(g.B + (int64_t)n0 * g.Kp, live_n * Kp);
  const bool scales_of_a = wave < WSA;
  const u32x4 rs = scales_of_a ? rsrc_words(g.sa + (int64_t)m0 * g.S, live_m * S) : rsrc_words(g.sb + (int64_t)n0 * g.S, live_n * S);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(AXONN_LDS char*)smem;
  const uint32_t at_lane = (uint32_t)(8 * wave + (lane >> 3)) * Kp + 16u * ((lane & 7) ^ (lane >> 3));
  const uint32_t scale_lane = (uint32_t)((scales_of_a ? wave : wave - WSA) * 64 + lane) * S;
  auto copy_tile = [&](int kt, int stage) {
    const uint32_t k = kt < g.nk ? (uint32_t)kt * FB : 0, lds = lds0 + stage * STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < NA; ++i) dma_chunk16(ra, at_lane + (uint32_t)(8 * W * i) * Kp, k, lds + i * (W * 1024));
#pragma unroll
    for (int i = 0; i < NB; ++i) dma_chunk16(rb, at_lane + (uint32_t)(8 * W * i) * Kp, k, lds + BM * FB + i * (W * 1024));
  };
  auto copy_scales = [&](int kt) {                       // of tiles kt .. kt + 3
    if (wave < WS && kt < g.nk) dma_word(rs, scale_lane, kt, lds0 + NS * STAGE + (kt >> 2 & 1) * ((BM + BN) * 4) + wave * 256);
  };
  floatx4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int r = lane & 15, q = lane >> 4;
  const int f0 = r * FB + 16 * (q ^ (r & 7)), f1 = r * FB + 16 * ((q + 4) ^ (r & 7));
  auto frag = [&](const char* base) {
    union { intx8 v; u32x4 h[2]; } u;
    u.h[0] = *reinterpret_cast<const u32x4*>(base + f0);
    u.h[1] = *reinterpret_cast<const u32x4*>(base + f1);
    return u.v;
  };
  int sa[TM] = {}, sb[TN] = {};
  copy_scales(0);
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) copy_tile(i, i);
  auto load_scales = [&](int kt) {
    const int* s = reinterpret_cast<const int*>(smem + NS * STAGE + (kt >> 2 & 1) * ((BM + BN) * 4)) + r;
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = s[(wm * TM + i) * 16];
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = s[BM + (wn * TN + j) * 16];
  };
  // tile kt in `stage`; `byte` of the scale words; the words are read where first says so
  auto step = [&](auto byte, int kt, int stage, int next_stage, bool first) {
    constexpr int J = decltype(byte)::value;
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"((NS - 2) * NC) : "memory");
    lds_barrier();
    if (first) {
      copy_scales(kt + 4);
      load_scales(kt);
    }
    copy_tile(kt + NS - 1, next_stage);
    const char* tile = smem + stage * STAGE;
    auto frag_a = [&](int i) { return frag(tile + (wm * TM + i) * 16 * FB); };
    auto frag_b = [&](int j) { return frag(tile + BM * FB + (wn * TN + j) * 16 * FB); };
    intx8 fa[2];
    if constexpr (EPI == EPI_ACC_F32) {
      WideFrag fb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = widen(frag_b(j), scale_value<J>(sb[j]));
      fa[0] = frag_a(0);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i + 1 < TM) fa[(i + 1) & 1] = frag_a(i + 1);
        const WideFrag wa = widen(fa[i & 1], scale_value<J>(sa[i]));
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j].v[p], wa.v[p], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      intx8 fb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = frag_b(j);
      fa[0] = frag_a(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i + 1 < TM) fa[(i + 1) & 1] = frag_a(i + 1);
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma_fp8<J>(fb[j], fa[i & 1], acc[i][j], sb[j], sa[i]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  int kt = 0;
  for (; kt + 4 <= g.nk; kt += 4) {
    step(std::integral_constant<int, 0>{}, kt, 0, (NS - 1) % NS, true);
    step(std::integral_constant<int, 1>{}, kt + 1, 1 % NS, NS % NS, false);
    step(std::integral_constant<int, 2>{}, kt + 2, 2 % NS, (NS + 1) % NS, false);
    step(std::integral_constant<int, 3>{}, kt + 3, 3 % NS, (NS + 2) % NS, false);
  }
  for (; kt < g.nk; ++kt) {                              // the last, shorter round: the words move instead of the immediate
    step(std::integral_constant<int, 0>{}, kt, kt % NS, (kt + NS - 1) % NS, (kt & 3) == 0);
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] >>= 8;
  }
  dma_wait_all();                                        // copies of tiles past the end still write to LDS
  lds_barrier();
  constexpr int IP = TM < 2 ? TM : 2;
  static_assert(W * 16 * IP * 16 * TN * 4 <= (int)sizeof smem, "staging");
  fp8_epilogue<EPI, TM, TN, IP>(g, acc, (float*)smem + wave * (16 * IP * 16 * TN), m0 + wm * TM * 16, n0 + wn * TN * 16, lane);
}

// 128 x 128 tiles, four waves, one per SIMD, each 64 x 64 of the result: what has too few tiles for the next kernel.  LDS bounds it:
// 64 KB of fragments and 32 KB of copies per tile of k, 768 cycles of the 850 to 1050 that it takes, to 512 of MFMAs.  Eight waves of
// 64 x 32 read 96 KB: 2047 x 2048 x 8192 in 38 us, this way 32 (2110 TFLOP/s).  While
// the MFMAs of a tile of k run from registers, the next one's fragments are read and the one three ahead is copied to where
// the tile before lay, whose fragments every wave has in registers at the barrier.
template <int EPI>
__global__ __launch_bounds__(256) void gemm_fp8_mid_kernel(const Fp8Args g) {
  constexpr int BM = 128, BN = 128, STAGE = (BM + BN) * FB, SCALES = 4 * STAGE, SBUF = (BM + BN) * 4;
  __shared__ __align__(1024) char smem[SCALES + 2 * SBUF];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  int pid = blockIdx.x, tm, tn;
  if ((gridDim.x & 7) == 0) pid = (pid & 7) * (gridDim.x >> 3) + (pid >> 3);
  fp8_tile_at(g, pid, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const uint32_t Kp = (uint32_t)g.Kp, S = (uint32_t)g.S;
  const uint32_t live_m = min(BM, g.M - m0), live_n = min(BN, g.N - n0);
  const u32x4 ra = rsrc_words(g.A + (int64_t)m0 * g.Kp, live_m * Kp), rb = rsrc_words(g.B + (int64_t)n0 * g.Kp, live_n * Kp);
  const u32x4 rs = wave < 2 ? rsrc_words(g.sa + (int64_t)m0 * g.S, live_m * S) : rsrc_words(g.sb + (int64_t)n0 * g.S, live_n * S);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(AXONN_LDS char*)smem;
  const uint32_t at_lane = (uint32_t)(8 * wave + (lane >> 3)) * Kp + 16u * ((lane & 7) ^ (lane >> 3));
  const uint32_t scale_lane = (uint32_t)((wave & 1) * 64 + lane) * S;
  // copy c of 0..7 of tile kt into `slot`: 8 rows of A, then of B, per wave
  auto copy = [&](int kt, int slot, int c) {
    dma_chunk16(c < 4 ? ra : rb, at_lane + (uint32_t)(32 * (c & 3)) * Kp, kt < g.nk ? (uint32_t)kt * FB : 0,
                lds0 + slot * STAGE + wave * 1024 + c * 4096);
  };
  auto copy_scales = [&](int kt) {                       // of tiles kt .. kt + 3
    if (kt < g.nk) dma_word(rs, scale_lane, kt, lds0 + SCALES + (kt >> 2 & 1) * SBUF + wave * 256);
  };
  const int r = lane & 15, q = lane >> 4;
  const int f[2] = {r * FB + 16 * (q ^ (r & 7)), r * FB + 16 * ((q + 4) ^ (r & 7))};
  const char* const a_of = smem + wm * (64 * FB);
  const char* const b_of = smem + BM * FB + wn * (64 * FB);
  union Frag { intx8 v; u32x4 h[2]; };
  Frag fa[2][4], fb[2][4];
  int sa[4], sb[4], sa_next[4] = {}, sb_next[4] = {};
  // half x & 1 of fragment x / 2 of a tile, in the order of their use: A 0, B 0 to 3, A 1 to 3
  auto read = [&](int set, int slot, int x) {
    const int n = x >> 1, h = x & 1;
    if (n == 0 || n > 4) {
      const int i = n == 0 ? 0 : n - 4;
      fa[set][i].h[h] = *reinterpret_cast<const u32x4*>(a_of + slot * STAGE + i * 16 * FB + f[h]);
    } else {
      fb[set][n - 1].h[h] = *reinterpret_cast<const u32x4*>(b_of + slot * STAGE + (n - 1) * 16 * FB + f[h]);
    }
  };
  auto read_scale = [&](int kt, int (&a)[4], int (&b)[4], int x) {
    const int* s = reinterpret_cast<const int*>(smem + SCALES + (kt >> 2 & 1) * SBUF) + r;
    if (x < 4) a[x] = s[wm * 64 + 16 * x];
    else b[x - 4] = s[BM + wn * 64 + 16 * (x - 4)];
  };
  floatx4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  copy_scales(0);
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int c = 0; c < 8; ++c) copy(i, i, c);
  asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  lds_barrier();
#pragma unroll
  for (int x = 0; x < 16; ++x) read(0, 0, x);
#pragma unroll
  for (int x = 0; x < 8; ++x) read_scale(0, sa, sb, x);
  auto step = [&](auto byte, int kt) {
    constexpr int J = decltype(byte)::value, P = J & 1;
    asm volatile("s_waitcnt vmcnt(8)\n\ts_barrier" ::: "memory");
    if (J == 0) copy_scales(kt + 4);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const int i = x >> 2, j = x & 3;
      acc[i][j] = mfma_fp8<J>(fb[P][j].v, fa[P][i].v, acc[i][j], sb[j], sa[i]);
      if (x < 8) {
        read(P ^ 1, (J + 1) & 3, 2 * x);
        read(P ^ 1, (J + 1) & 3, 2 * x + 1);
      }
      if (x & 1) copy(kt + 3, (J + 3) & 3, x >> 1);
      if (J == 3 && x < 8) read_scale(kt + 1, sa_next, sb_next, x);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (J == 3) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sa[i] = sa_next[i];
        sb[i] = sb_next[i];
      }
    }
  };
  using std::integral_constant;
  int kt = 0;
  for (; kt + 4 <= g.nk; kt += 4) {
    step(integral_constant<int, 0>{}, kt);
    step(integral_constant<int, 1>{}, kt + 1);
    step(integral_constant<int, 2>{}, kt + 2);
    step(integral_constant<int, 3>{}, kt + 3);
  }
  if (kt < g.nk) step(integral_constant<int, 0>{}, kt);
  if (kt + 1 < g.nk) step(integral_constant<int, 1>{}, kt + 1);
  if (kt + 2 < g.nk) step(integral_constant<int, 2>{}, kt + 2);
  dma_wait_all();                                        // copies of tiles past the end still write to LDS
  lds_barrier();
  fp8_epilogue<EPI, 4, 4, 2>(g, acc, (float*)smem + wave * (16 * 2 * 64), m0 + wm * 64, n0 + wn * 64, lane);
}

// The product for problems that fill the chip with 256 x 256 tiles: four waves, one per SIMD, each 128 x 128 of the result, the
// 256 accumulators in the accumulation registers.  With 8 waves of 128 x 64 (196 KB of fragments per tile of k instead of 128 KB,
// and every wave at the barrier with nothing to do) 8192 x 20480 results over K = 5120 took 1.35 times as long (1000 us and 745, single
// launches behind pauses).  Launches one behind the other, 24 at a time, take 633 us (2710 TFLOP/s), 8192^3 382 (2880); a few behind a
// pause 654 to 791, and so under the profiler, 736.  The matrix units are busy 77 % of the cycles of 8192^3, at the 1.75 GHz that the
// chip's power leaves (zeros for operands: 3200).
//
// Half a tile of k (the rows of four of the eight fragments) is the unit of copying: a set holds half of A(kt) and half of
// B(kt + 1), 16 KB each, four sets in LDS.  A group is the 8 MFMAs of one A fragment; while it runs, the next A fragment and one B
// fragment of the next tile are read, so B's fragments are in registers a tile ahead and no group waits for LDS.  The last
// group of a half runs behind the barrier that opens the next set, which was copied one and a half tiles of k ago.
//
// A workgroup does one tile of the result after the other, and what is copied and read ahead at the end of one belongs to the
// next: its first sets arrive while the epilogue stores.  The epilogue has the LDS of one set, whose copy waits until it is done.
// The steps of a tile are rounded up to four (a word of scales), the ones past the end on zeros.
// J: which byte of a scale's register.
template <int J>
__device__ __forceinline__ void mfma_fp8_acc(floatx4& c, intx8 b, intx8 a, int sb, int sa) {
  if constexpr (J == 0)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+a"(c) : "v"(b), "v"(a), "v"(sb), "v"(sa));
  else
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0]"
                 : "+a"(c) : "v"(b), "v"(a), "v"(sb), "v"(sa));
}

template <int EPI>
__global__ __launch_bounds__(256) void gemm_fp8_big_kernel(const Fp8Args g) {
  constexpr int BM = 256, BN = 256, HALF = 128 * FB, SET = 2 * HALF, SCALES = 4 * SET, SBUF = (BM + BN) * 4;
  __shared__ __align__(1024) char smem[SCALES + 2 * SBUF];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t Kp = (uint32_t)g.Kp, S = (uint32_t)g.S;
  const int steps = (g.nk + 3) & ~3;
  // this workgroup's tiles: a run of each XCD's share
  const int n_tiles = g.tiles_m * g.tiles_n, xcds = (gridDim.x & 7) == 0 ? 8 : 1;
  const int share = (n_tiles + xcds - 1) / xcds, stride = gridDim.x / xcds;
  const int first = blockIdx.x % xcds * share, end = min(n_tiles, first + share);
  int pid = first + blockIdx.x / xcds;
  if (pid >= end) return;
  struct Tile { int m0, n0; };                           // past the last one: behind the matrix, where nothing is read
  auto tile_of = [&](int p) {
    Tile t = {g.M, g.N};
    if (p < end) {
      int tm, tn;
      fp8_tile_at(g, p, tm, tn);
      t.m0 = __builtin_amdgcn_readfirstlane(tm * BM);
      t.n0 = __builtin_amdgcn_readfirstlane(tn * BN);
    }
    return t;
  };
  // descriptor of the rows of a matrix (`ld` bytes each) from m0 on, `most` of them at most; empty unless `live`
  auto rows_of = [](const uint8_t* p, int m0, int n_rows, int most, uint32_t ld, bool live) {
    return rsrc_words(p + (int64_t)m0 * ld, live ? (uint32_t)min(most, n_rows - m0) * ld : 0);
  };
  Tile now = tile_of(pid), next = tile_of(pid + stride);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(AXONN_LDS char*)smem;
  // copies: rows 32 * wave .. + 31 of a half, whose 128 rows are rows 64 h .. + 63 of both waves' 128
  const uint32_t from = ((uint32_t)(wave >> 1) * 128 + (wave & 1) * 32 + (lane >> 3)) * Kp + 16u * ((lane & 7) ^ (lane >> 3));
  const uint32_t scale_from = (uint32_t)(64 * wave + lane) * S;
  // copy c of 0..7 of step kt: four of A(kt), then four of B(kt + 1); aim() sets where from, steps past the tile's are the next's
  u32x4 ra, rb;
  uint32_t ka, kb;
  auto aim = [&](int kt) {
    const int ta = kt < steps ? kt : kt - steps, tb = kt + 1 < steps ? kt + 1 : kt + 1 - steps;
    ra = rows_of(g.A, kt < steps ? now.m0 : next.m0, g.M, BM, Kp, ta < g.nk);
    rb = rows_of(g.B, kt + 1 < steps ? now.n0 : next.n0, g.N, BN, Kp, tb < g.nk);
    ka = (uint32_t)ta * FB;
    kb = (uint32_t)tb * FB;
  };
  auto copy = [&](int h, int slot, int c) {
    dma_chunk16(c < 4 ? ra : rb, from + (uint32_t)(64 * h + 8 * (c & 3)) * Kp, c < 4 ? ka : kb,
                lds0 + slot * SET + (c < 4 ? 0 : HALF) + wave * 4096 + (c & 3) * 1024);
  };
  int round = 0;                                         // rounds of four steps in front of this tile
  auto scale_at = [&](int kt) { return (round + (kt >> 2) & 1) * SBUF + (kt & 2); };   // of step kt and its neighbour
  auto copy_scales = [&](int kt) {                       // of steps kt .. kt + 3
    const uint32_t to = lds0 + SCALES + (round + (kt >> 2) & 1) * SBUF + wave * 256;
    const bool in = kt < steps;
    dma_word(rows_of(g.sa, in ? now.m0 : next.m0, g.M, BM, S, true), scale_from, in ? kt : 0, to);
    dma_word(rows_of(g.sb, in ? now.n0 : next.n0, g.N, BN, S, true), scale_from, in ? kt : 0, to + BM * 4);
  };
  const int r = lane & 15, q = lane >> 4;
  const int f0 = r * FB + 16 * (q ^ (r & 7)), f1 = r * FB + 16 * ((q + 4) ^ (r & 7));
  const char* const a0 = smem + wm * (64 * FB) + f0;     // fragment k of a set's A: + slot * SET + k * 16 * FB
  const char* const a1 = smem + wm * (64 * FB) + f1;
  const char* const b0 = smem + HALF + wn * (64 * FB) + f0;
  const char* const b1 = smem + HALF + wn * (64 * FB) + f1;
  const char* const sca = smem + SCALES + wm * 512 + 4 * r;      // a fragment's scales: + 64 bytes each
  const char* const scb = smem + SCALES + BM * 4 + wn * 512 + 4 * r;
  union Frag { intx8 v; u32x4 h[2]; };
  Frag fa[2], fb[2][8];
  int sa[2], sb[2][8];
  // A scale as loaded (16 bits, the rest zero): without this the compiler clears the rest again in front of the MFMA, where nobody
  // keeps the distance from a vector instruction to the MFMA that reads its result.
#define AXONN_AS_LOADED(x) asm volatile("" : "+v"(x))

  copy_scales(0);
  aim(-1);
  rb = rows_of(g.B, now.n0, g.N, BN, Kp, true);
#pragma unroll
  for (int h = 0; h < 2; ++h)                            // B(0): the second halves of sets -2 and -1
#pragma unroll
    for (int c = 4; c < 8; ++c) copy(h, 2 + h, c);
  aim(0);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < 8; ++c) copy(h, h, c);
  asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  lds_barrier();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    fb[0][j].h[0] = *reinterpret_cast<const u32x4*>(b0 + (2 + (j >> 2)) * SET + (j & 3) * 16 * FB);
    fb[0][j].h[1] = *reinterpret_cast<const u32x4*>(b1 + (2 + (j >> 2)) * SET + (j & 3) * 16 * FB);
    sb[0][j] = *reinterpret_cast<const uint16_t*>(scb + scale_at(0) + j * 64);
    AXONN_AS_LOADED(sb[0][j]);
  }
  lds_barrier();
  aim(1);
#pragma unroll
  for (int c = 0; c < 8; ++c) copy(0, 2, c);
  asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  lds_barrier();
  fa[0].h[0] = *reinterpret_cast<const u32x4*>(a0);
  fa[0].h[1] = *reinterpret_cast<const u32x4*>(a1);
  sa[0] = *reinterpret_cast<const uint16_t*>(sca + scale_at(0));
  fb[1][0].h[0] = *reinterpret_cast<const u32x4*>(b0);
  fb[1][0].h[1] = *reinterpret_cast<const u32x4*>(b1);
  sb[1][0] = *reinterpret_cast<const uint16_t*>(scb + scale_at(1));
  AXONN_AS_LOADED(sa[0]);
  AXONN_AS_LOADED(sb[1][0]);

  floatx4 acc[8][8];
  // step kt, of parity J: fragments of A in turn; what is read belongs to the next fragment, a step later behind the last one.
  // FINAL: the tile's last step, the copies of whose last group wait for the epilogue.
  auto step = [&](auto parity, auto final, int kt) {
    constexpr int J = decltype(parity)::value;
    constexpr bool FINAL = decltype(final)::value;
    const char* const sa_now = sca + scale_at(kt);
    const char* const sa_next = sca + scale_at(kt + 1);
    const char* const sb_now = scb + scale_at(kt + 1);
    const char* const sb_next = scb + scale_at(kt + 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool last = i == 7, opens = (i & 3) == 3;
      const int h = opens ? (i >> 2) ^ 1 : i >> 2;        // half of the set that is read
      const int k = (i + 1) & 3, slot = (2 * J + (last ? 2 : h)) & 3;
      const int nb = last ? J : J ^ 1;                    // the B fragment read belongs to the next step, or the one behind it
      if (opens) {
        asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
        lds_barrier();
        if (i == 3) aim(kt + 2);
        if (J == 0 && i == 3 && (kt & 3) == 0) copy_scales(kt + 4);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        mfma_fp8_acc<J>(acc[i][j], fb[J][j].v, fa[i & 1].v, sb[J][j], sa[i & 1]);
        if (j == 0) {
          fa[(i + 1) & 1].h[0] = *reinterpret_cast<const u32x4*>(a0 + slot * SET + k * 16 * FB);
          fa[(i + 1) & 1].h[1] = *reinterpret_cast<const u32x4*>(a1 + slot * SET + k * 16 * FB);
        }
        if (j == 1) {
          sa[(i + 1) & 1] = *reinterpret_cast<const uint16_t*>((last ? sa_next : sa_now) + ((i + 1) & 7) * 64);
          sb[nb][4 * h + k] = *reinterpret_cast<const uint16_t*>((last ? sb_next : sb_now) + (4 * h + k) * 64);
        }
        if (j == 2) fb[nb][4 * h + k].h[0] = *reinterpret_cast<const u32x4*>(b0 + slot * SET + k * 16 * FB);
        if (j == 3) fb[nb][4 * h + k].h[1] = *reinterpret_cast<const u32x4*>(b1 + slot * SET + k * 16 * FB);
        if (j == 7) {
          AXONN_AS_LOADED(sa[(i + 1) & 1]);
          AXONN_AS_LOADED(sb[nb][4 * h + k]);
        }
        // two of a set's eight copies in each of the four groups from the one that opens: all at once they held the MFMAs up
        if ((j == 4 || j == 6) && !(FINAL && last))
          copy(i < 3 || last ? 1 : 0, (i < 3 ? 2 * J + 3 : last ? 2 * J + 1 : 2 * J) & 3, 2 * k + (j == 6));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  using std::integral_constant;
  while (true) {
    copy(1, 3, 0);                                       // what a tile's last group leaves to the next
    copy(1, 3, 1);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) asm volatile("" : "+a"(acc[i][j]));
    asm volatile("s_nop 7");                             // behind them all: the compiler does not know that MFMAs read them
    int kt = 0;
    do {
      step(integral_constant<int, 0>{}, integral_constant<bool, false>{}, kt);
      step(integral_constant<int, 1>{}, integral_constant<bool, false>{}, kt + 1);
      kt += 2;
    } while (kt < steps - 2);
    step(integral_constant<int, 0>{}, integral_constant<bool, false>{}, kt);
    step(integral_constant<int, 1>{}, integral_constant<bool, true>{}, kt + 1);
    // the matrix unit's last results; the compiler does not know what wrote them
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
    fp8_epilogue<EPI, 8, 8, 1>(g, acc, (float*)(smem + 3 * SET) + wave * (16 * 128), now.m0 + wm * 128, now.n0 + wn * 128, lane);
    pid += stride;
    if (pid >= end) break;
    lds_barrier();                                       // every wave is done with its part of the set
    now = next;
    next = tile_of(pid + stride);
    round += steps >> 2;
  }
  dma_wait_all();                                        // copies past the end still write (zeros) to LDS
#undef AXONN_AS_LOADED
}

static void fp8_tiles(Fp8Args& g, int bm, int bn) {
  g.tiles_m = (g.M + bm - 1) / bm;
  g.tiles_n = (g.N + bn - 1) / bn;
}
template <int WM, int WN, int TM, int TN, int NS, int EPI>
static hipError_t launch_fp8_tile(Fp8Args g, hipStream_t s) {
  fp8_tiles(g, WM * TM * 16, WN * TN * 16);
  hipLaunchKernelGGL(HIP_KERNEL_NAME(gemm_fp8_kernel<WM, WN, TM, TN, NS, EPI>), dim3((unsigned)(g.tiles_m * g.tiles_n)),
                     dim3(64 * WM * WN), 0, s, g);
  return hipGetLastError();
}
template <int EPI>
static hipError_t launch_fp8_mid(Fp8Args g, hipStream_t s) {
  fp8_tiles(g, 128, 128);
  hipLaunchKernelGGL(HIP_KERNEL_NAME(gemm_fp8_mid_kernel<EPI>), dim3((unsigned)(g.tiles_m * g.tiles_n)), dim3(256), 0, s, g);
  return hipGetLastError();
}
template <int EPI>
static hipError_t launch_fp8_big(Fp8Args g, hipStream_t s) {
  fp8_tiles(g, 256, 256);
  hipLaunchKernelGGL(HIP_KERNEL_NAME(gemm_fp8_big_kernel<EPI>), dim3((unsigned)std::min(256, g.tiles_m * g.tiles_n)), dim3(256), 0, s, g);
  return hipGetLastError();
}
template <int EPI>
static hipError_t launch_fp8(const Fp8Args& g, hipStream_t s) {
  const int tile = host::choose_fp8_tile(g.M, g.N, g.nk, EPI == EPI_ACC_F32);
  if (tile == host::FP8_64x64) return launch_fp8_tile<2, 2, 2, 2, 4, EPI>(g, s);
  if constexpr (EPI == EPI_ACC_F32) {
    if (tile == host::FP8_256x256) return launch_fp8_tile<2, 4, 8, 4, 2, EPI>(g, s);
    return launch_fp8_tile<2, 2, 4, 4, 2, EPI>(g, s);
  } else {
    if (tile == host::FP8_256x256) return launch_fp8_big<EPI>(g, s);
    return launch_fp8_mid<EPI>(g, s);
  }
}

hipError_t launch_gemm_fp8(int epi, int64_t M, int64_t N, int64_t K, const void* A, const void* a_scale, const void* B, const void* b_scale,
                           void* C, int64_t ldc, const void* bias, const void* res, int64_t ld_res, void* aux, int64_t ld_aux,
                           int accumulate, hipStream_t s) {
  Fp8Args g = {};
  g.M = (int)M; g.N = (int)N; g.nk = (int)((K + FB - 1) / FB);
  g.Kp = (int64_t)g.nk * FB; g.S = (g.nk + 3) / 4 * 4;
  g.A = (const uint8_t*)A; g.B = (const uint8_t*)B; g.sa = (const uint8_t*)a_scale; g.sb = (const uint8_t*)b_scale;
  g.C = C; g.ldc = ldc; g.ld_side = epi == EPI_BIAS_RES ? ld_res : ld_aux;
  g.bias = (const elem_t*)bias; g.res = (const elem_t*)res; g.aux = (elem_t*)aux; g.accumulate = accumulate;
  switch (epi) {
    case EPI_BIAS: return launch_fp8<EPI_BIAS>(g, s);
    case EPI_BIAS_RES: return launch_fp8<EPI_BIAS_RES>(g, s);
    case EPI_BIAS_GELU: return launch_fp8<EPI_BIAS_GELU>(g, s);
    case EPI_DGELU: return launch_fp8<EPI_DGELU>(g, s);
    case EPI_ACC_F32: return launch_fp8<EPI_ACC_F32>(g, s);
    default: return launch_fp8<EPI_ACC_BF16>(g, s);
  }
}

}  // namespace axonn
