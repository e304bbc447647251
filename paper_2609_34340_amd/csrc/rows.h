// Rows of elements in 16-byte pieces that may start at any element: loads and stores of global memory need no more than
// the element's alignment, and only a row's last piece may be part of one.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"
#include "numeric.h"

namespace vp {

typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// Vec<T>::n elements from p on, of which `left` (maybe none, or more than these) exist; past them zeros, or (of 16-bit
// ones) the LAST of them.
template <typename T, bool LAST = false> __device__ inline u32x4 load_piece(const T* p, int64_t left) {
  constexpr int n = Vec<T>::n;
  if (left >= n) return *(const u32x4_any*)p;
  u32x4 v = {0, 0, 0, 0};
  if constexpr (LAST) {
    static_assert(n == 8, "16-bit elements");
    if (left <= 0) return v;
    const int last = (int)left - 1;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const int at = i < last ? i : last;
      v[i / 2] |= (uint32_t)((const uint16_t*)p)[at] << (16 * (i % 2));
    }
    return v;
  }
#pragma unroll
  for (int i = 0; i < n - 1; ++i) {
    if (i < left) {
      if constexpr (n == 8) v[i / 2] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (i % 2));
      else v[i] = ((const uint32_t*)p)[i];
    }
  }
  return v;
}
template <typename T> __device__ inline void store_piece(T* p, u32x4 v, int64_t left) {
  constexpr int n = Vec<T>::n;
  if (left >= n) {
    *(u32x4_any*)p = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < n - 1; ++i) {
    if (i < left) {
      if constexpr (n == 8) ((uint16_t*)p)[i] = (uint16_t)(v[i / 2] >> (16 * (i % 2)));
      else ((uint32_t*)p)[i] = v[i];
    }
  }
}

// Calls f with the element type.
template <typename F> void with_type(int32_t dtype, F f) {
  if (dtype == VP_F32) f(float{});
  else if (dtype == VP_BF16) f(Bf16{});
  else f(F16{});
}

}  // namespace vp
