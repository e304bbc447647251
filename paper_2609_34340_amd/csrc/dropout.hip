// Dropout whose mask follows from a counter, with the residual's sum.
//
// Four neighbouring values of a row share one 64-bit output of SplitMix64 (Steele, Lea, Flood, OOPSLA 2014): output n of a
// stream is mix(key + (n + 1) gamma), so every thread makes its own.  Each value takes 16 of the bits and stays where
// they reach round(65536 p).  16 bits: half the integer multiplies of 32, which are a quarter of the vector rate; the
// factor is that of the probability in steps of 2^-16, so the expectation stays exact.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

struct DropoutArgs {
  int64_t T, H;
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

template <typename T> __global__ void __launch_bounds__(256) dropout_kernel(DropoutArgs a) {
  const uint64_t key = stream_key(a);
  const int64_t t = block_index(), words = (a.H + 3) / 4;
  if (t >= a.T) return;
  const T *x = (const T*)(a.x + t * a.x_stride), *res = (const T*)(a.residual + t * a.residual_stride);
  T* out = (T*)(a.out + t * a.out_stride);
  for (int64_t w = threadIdx.x; w < words; w += 256) {
    const uint64_t bits = mix(key + (uint64_t)(t * words + w + 1) * kGamma);
    for (int64_t c = w * 4; c < std::min(w * 4 + 4, a.H); ++c) {
      float v = (uint32_t)(bits >> (16 * (c % 4)) & 0xffff) >= a.least ? to_f32(x[c]) * a.scale : 0.0f;
      if (a.residual) v += to_f32(res[c]);
      out[c] = from_f32<T>(v);
    }
  }
}

}  // namespace

vp_status launch_dropout(const void* x, int32_t dtype, int64_t T, int64_t H, int64_t x_stride, uint32_t least,
                         uint64_t seed, const int64_t* step, const void* residual, int64_t residual_stride, void* out,
                         int64_t out_stride, void* stream) {
  const DropoutArgs a{T, H, (const unsigned char*)x, (const unsigned char*)residual, x_stride, residual_stride, out_stride,
                      (unsigned char*)out, seed, step, least, least < 65536 ? 65536.0f / (float)(65536 - least) : 0.0f};
  if (dtype == VP_F32) hipLaunchKernelGGL(dropout_kernel<float>, grid_of(T), dim3(256), 0, (hipStream_t)stream, a);
  else if (dtype == VP_BF16) hipLaunchKernelGGL(dropout_kernel<Bf16>, grid_of(T), dim3(256), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(dropout_kernel<F16>, grid_of(T), dim3(256), 0, (hipStream_t)stream, a);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "dropout launch failed");
  return VP_OK;
}

}  // namespace vp
