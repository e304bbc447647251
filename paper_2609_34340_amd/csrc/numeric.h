// 16-bit and 32-bit element types of the layer operators, in registers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace vp {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Bf16 { uint16_t u; };
struct F16 { uint16_t u; };

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(Bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
__device__ inline float to_f32(F16 x) { return (float)__builtin_bit_cast(_Float16, x.u); }

// Round to nearest, ties to even; NaN stays NaN.
template <typename T> __device__ inline T from_f32(float x);
template <> __device__ inline float from_f32<float>(float x) { return x; }
template <> __device__ inline Bf16 from_f32<Bf16>(float x) { return {__builtin_bit_cast(uint16_t, (__bf16)x)}; }
template <> __device__ inline F16 from_f32<F16>(float x) { return {__builtin_bit_cast(uint16_t, (_Float16)x)}; }

// 16 bytes of T as floats and back.
template <typename T> struct Vec { static constexpr int n = 8; };
template <> struct Vec<float> { static constexpr int n = 4; };

template <typename T> __device__ inline void unpack16(u32x4 v, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = to_f32(T{(uint16_t)(v[i] & 0xffffu)});
    f[2 * i + 1] = to_f32(T{(uint16_t)(v[i] >> 16)});
  }
}
template <> __device__ inline void unpack16<float>(u32x4 v, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
}
template <typename T> __device__ inline u32x4 pack16(const float* f) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(f[2 * i]).u | (uint32_t)from_f32<T>(f[2 * i + 1]).u << 16;
  return v;
}
template <> __device__ inline u32x4 pack16<float>(const float* f) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
  return v;
}

// f over groups of LPT neighbouring lanes (16 or 64), the result in every one of
// them, by data movement in the vector unit.
template <int CTRL, typename T> __device__ inline T moved(T v) {
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LPT, typename T, typename F> __device__ inline T across(T v, F f) {
#ifdef __HIP_DEVICE_COMPILE__
  v = f(v, moved<0xB1>(v));    // within pairs
  v = f(v, moved<0x4E>(v));    // fours
  v = f(v, moved<0x141>(v));   // eights: each half row mirrored
  v = f(v, moved<0x140>(v));   // rows of 16, mirrored
  if constexpr (LPT == 64) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);   // even rows, odd rows
    v = f(__builtin_bit_cast(T, (unsigned)a[0]), __builtin_bit_cast(T, (unsigned)a[1]));
    const unsigned w = __builtin_bit_cast(unsigned, v);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);   // halves
    v = f(__builtin_bit_cast(T, (unsigned)b[0]), __builtin_bit_cast(T, (unsigned)b[1]));
  }
#endif
  return v;
}

// A dimension of a grid holds fewer than 2^32 threads (a launch of more runs some of them, and returns no error): blocks of
// up to 1,024 threads past the 2^21st go on in the second dimension, whose last line may be part empty.
constexpr int64_t kGridLine = 1 << 21;
inline dim3 grid_of(int64_t blocks) {
  return blocks <= kGridLine ? dim3((unsigned)blocks) : dim3((unsigned)kGridLine, (unsigned)((blocks + kGridLine - 1) / kGridLine));
}
__device__ inline int64_t block_index() { return (int64_t)blockIdx.y * kGridLine + blockIdx.x; }

}  // namespace vp
