// Dropout whose mask follows from a counter, with the residual's sum.
//
// Four neighbouring values of a row share one 64-bit output of SplitMix64 (Steele, Lea, Flood, OOPSLA 2014): output n of a
// stream is mix(key + (n + 1) gamma), so every thread makes its own.  Each value takes 16 of the bits and stays where
// they reach round(65536 p).  16 bits: half the integer multiplies of 32, which are a quarter of the vector rate; the
// factor is that of the probability in steps of 2^-16, so the expectation stays exact.  HBM bounds it: 8192 rows of 7168
// with a residual, bf16, 65 us, 5.4 TB/s (a 1 GiB copy 4.8 to 5.2), the vector units busy a third of the time.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "numeric.h"
#include "rows.h"

namespace vp {
namespace {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

struct DropoutArgs {
  int64_t T;
  int32_t H, pieces;   // 16-byte pieces of a row
  const unsigned char *x, *residual;
  int64_t x_stride, residual_stride, out_stride;
  unsigned char* out;
  uint64_t seed;
  const int64_t* step;
  uint32_t least;
  float scale;
};

__device__ inline uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

// The state of the stream that seed and step select.
__device__ inline uint64_t stream_key(const DropoutArgs& a) {
  const uint64_t step = a.step ? (uint64_t)*a.step : 0;
  return mix((mix(a.seed + kGamma) ^ step) + kGamma);
}

constexpr int kThreads = 256, kAhead = 4;   // pieces of a thread whose loads are issued together

// LANES threads to a row.
template <typename T, int LANES, bool RES> __global__ void __launch_bounds__(kThreads) dropout_kernel(DropoutArgs a) {
  constexpr int n = Vec<T>::n;
  const uint64_t key = stream_key(a);
  const int64_t t = block_index() * (kThreads / LANES) + threadIdx.x / LANES;
  if (t >= a.T) return;
  const T *x = (const T*)(a.x + t * a.x_stride), *res = (const T*)(a.residual + t * a.residual_stride);
  T* out = (T*)(a.out + t * a.out_stride);
  const uint64_t first = key + (uint64_t)(t * ((a.H + 3) / 4) + 1) * kGamma;   // of the row's first word
  for (int j0 = threadIdx.x % LANES; j0 < a.pieces; j0 += LANES * kAhead) {
    u32x4 v[kAhead], r[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int c = (j0 + i * LANES) * n;
      v[i] = load_piece(x + c, a.H - c);
      if constexpr (RES) r[i] = load_piece(res + c, a.H - c);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int c = (j0 + i * LANES) * n;
      if (c >= a.H) break;
      float f[n], g[n];
      unpack16<T>(v[i], f);
      if constexpr (RES) unpack16<T>(r[i], g);
#pragma unroll
      for (int k = 0; k < n / 4; ++k) {
        const uint64_t bits = mix(first + (uint64_t)(uint32_t)(c / 4 + k) * kGamma);
        const uint32_t half[2] = {(uint32_t)bits, (uint32_t)(bits >> 32)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t field = e % 2 ? half[e / 2] >> 16 : half[e / 2] & 0xffffu;
          const float y = field >= a.least ? f[4 * k + e] * a.scale : 0.0f;
          f[4 * k + e] = RES ? y + g[4 * k + e] : y;
        }
      }
      store_piece(out + c, pack16<T>(f), a.H - c);
    }
  }
}

template <typename T, int LANES> void launch_as(const DropoutArgs& a, hipStream_t s) {
  constexpr int rows = kThreads / LANES;
  const dim3 grid = grid_of((a.T + rows - 1) / rows);
  if (a.residual) hipLaunchKernelGGL((dropout_kernel<T, LANES, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((dropout_kernel<T, LANES, false>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

vp_status launch_dropout(const void* x, int32_t dtype, int64_t T, int64_t H, int64_t x_stride, uint32_t least,
                         uint64_t seed, const int64_t* step, const void* residual, int64_t residual_stride, void* out,
                         int64_t out_stride, void* stream) {
  with_type(dtype, [&](auto type) {
    using E = decltype(type);
    const DropoutArgs a{T, (int32_t)H, (int32_t)((H + Vec<E>::n - 1) / Vec<E>::n), (const unsigned char*)x,
                        (const unsigned char*)residual, x_stride, residual_stride, out_stride, (unsigned char*)out, seed, step,
                        least, least < 65536 ? 65536.0f / (float)(65536 - least) : 0.0f};
    if (a.pieces <= 16) launch_as<E, 16>(a, (hipStream_t)stream);
    else if (a.pieces <= 256) launch_as<E, 64>(a, (hipStream_t)stream);
    else launch_as<E, 256>(a, (hipStream_t)stream);
  });
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "dropout launch failed");
  return VP_OK;
}

}  // namespace vp
