// Rows of 16-bit elements that may start at any element and have any length: chunks of 8 elements, the last one shorter.
#pragma once
#include "common.h"

namespace axonn {

#ifdef __HIPCC__
// 16 bytes at the address of any element: the memory pipeline takes unaligned addresses, one instruction as for aligned ones.
typedef elemx8 elemx8_any __attribute__((aligned(2)));

// Elements p[0..n) of a chunk, n of 8 (8 or more: all); zeros behind them, and nothing behind them is read.
__device__ __forceinline__ elemx8 load_chunk(const elem_t* p, int n) {
  if (n >= 8) return *reinterpret_cast<const elemx8_any*>(p);
  elemx8 v = {};
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) v[i] = p[i];
  return v;
}
__device__ __forceinline__ void store_chunk(elem_t* p, const elemx8& v, int n) {
  if (n >= 8) {
    *reinterpret_cast<elemx8_any*>(p) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) p[i] = v[i];
}
#endif

}  // namespace axonn
