// Rows in 4-bit blocks (OCP microscaling format MXFP4) and back.
//
// 32 neighbouring values of a row share one power of two; each is a sign, two
// exponent bits and one mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6).  The power
// is that of the block's largest magnitude over 4, so the scaled values lie
// below 8 and those above 6 become 6; the others go to the nearest value,
// ties to the even code.  A packed row of K values holds K/2 bytes of codes
// (two a byte, the lower index in the low four bits), K/32 exponent bytes
// (bias 127; 255 marks a block that held an infinity or NaN: all its values
// are NaN) and zeros up to a multiple of 16 bytes: one row of bytes that the
// pack and unpack calls move like any other, 3.75 times smaller than 16-bit
// values.
//
// HBM bounds both directions (2 B read and 0.53 B written per 16-bit value):
// a thread holds eight values, four lanes a block, so that loads are whole
// 16-byte vectors and the maximum takes two cross-lane steps.  16,384 rows of
// 4096 bf16 values: 25.7 us there (6.6 TB/s; 45 us with the codes found by
// comparisons), 28.1 us back (6.0 TB/s); of 7168 values 48 and 66 us.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;   // values of a thread

// The codes of eight values below 8, by the conversion instruction (nearest,
// ties to the even code, ends at 6; low four bits first).
__device__ inline uint32_t codes_of(const float* f) {
#ifdef __HIP_DEVICE_COMPILE__
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], 1.0f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], 1.0f, 3);
#else
  return 0;
#endif
}

__device__ inline float value_of(uint32_t code) {
  // the three magnitude bits at the top of a float's exponent and mantissa
  const float m = __uint_as_float((code & 7u) << 22) * 0x1p126f;
  return code & 8u ? -m : m;
}

template <typename T> __device__ inline void load8(const unsigned char* p, float* f) {
  unpack16<T>(*(const u32x4*)p, f);
  if constexpr (sizeof(T) == 4) unpack16<T>(*(const u32x4*)(p + 16), f + 4);
}
template <typename T> __device__ inline void store8(unsigned char* p, const float* f) {
  *(u32x4*)p = pack16<T>(f);
  if constexpr (sizeof(T) == 4) *(u32x4*)(p + 16) = pack16<T>(f + 4);
}

struct MxArgs {
  const unsigned char* in;
  unsigned char* out;
  int64_t rows, in_stride, out_stride;   // strides in bytes
  int32_t K, per_row;                    // threads of a row: a power of two, 4 to 256
  int32_t row_bytes;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(MxArgs a) {
  const int sub = threadIdx.x & (a.per_row - 1);
  const int64_t r = block_index() * (kThreads / a.per_row) + threadIdx.x / a.per_row;
  if (r >= a.rows) return;
  const unsigned char* src = a.in + r * a.in_stride;
  unsigned char* dst = a.out + r * a.out_stride;
  // K / 8 is a multiple of four, so the four lanes of a block enter together
  for (int c = sub; c < a.K / kPer; c += a.per_row) {
    float f[kPer];
    load8<T>(src + (int64_t)c * kPer * sizeof(T), f);
    uint32_t top = 0;   // magnitudes compare as their bits; NaN above infinity
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    top = max(top, __shfl_xor(top, 1));
    top = max(top, __shfl_xor(top, 2));
    const int e = (int)(top >> 23);
    const int power = e == 255 ? 255 : max(e - 2, 0);   // the exponent byte
#pragma unroll
    for (int i = 0; i < kPer; ++i) f[i] = ldexpf(f[i], 127 - power);
    *(uint32_t*)(dst + (int64_t)c * 4) = power == 255 ? 0 : codes_of(f);
    if ((c & 3) == 0) dst[a.K / 2 + c / 4] = (unsigned char)power;
  }
  for (int i = a.K / 2 + a.K / 32 + sub; i < a.row_bytes; i += a.per_row) dst[i] = 0;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(MxArgs a) {
  const int sub = threadIdx.x & (a.per_row - 1);
  const int64_t r = block_index() * (kThreads / a.per_row) + threadIdx.x / a.per_row;
  if (r >= a.rows) return;
  const unsigned char* src = a.in + r * a.in_stride;
  unsigned char* dst = a.out + r * a.out_stride;
  for (int c = sub; c < a.K / kPer; c += a.per_row) {
    const uint32_t codes = *(const uint32_t*)(src + (int64_t)c * 4);
    const int power = src[a.K / 2 + c / 4];
    float f[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) f[i] = power == 255 ? NAN : ldexpf(value_of(codes >> (4 * i)), power - 127);
    store8<T>(dst + (int64_t)c * kPer * sizeof(T), f);
  }
}

template <typename F> void launch_rows(F kernel, MxArgs a, hipStream_t s) {
  a.per_row = 4;
  while (a.per_row < kThreads && a.per_row < a.K / kPer) a.per_row *= 2;
  const int64_t rows = kThreads / a.per_row;
  if (a.rows > 0)
    hipLaunchKernelGGL(kernel, grid_of((a.rows + rows - 1) / rows), dim3(kThreads), 0, s, a);
}

}  // namespace

int64_t mx_row_bytes(int64_t K) { return (K / 2 + K / 32 + 15) / 16 * 16; }

vp_status launch_mx_quantize(const void* x, int32_t dtype, int64_t rows, int64_t K, int64_t x_stride, void* q,
                             int64_t q_stride, void* stream) {
  MxArgs a{(const unsigned char*)x, (unsigned char*)q, rows, x_stride, q_stride, (int32_t)K, 0,
           (int32_t)mx_row_bytes(K)};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == VP_F32) launch_rows(mx_quantize_kernel<float>, a, s);
  else if (dtype == VP_BF16) launch_rows(mx_quantize_kernel<Bf16>, a, s);
  else launch_rows(mx_quantize_kernel<F16>, a, s);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "quantise launch failed");
  return VP_OK;
}

vp_status launch_mx_dequantize(const void* q, int64_t rows, int64_t K, int64_t q_stride, void* out, int32_t dtype,
                               int64_t out_stride, void* stream) {
  MxArgs a{(const unsigned char*)q, (unsigned char*)out, rows, q_stride, out_stride, (int32_t)K, 0,
           (int32_t)mx_row_bytes(K)};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == VP_F32) launch_rows(mx_dequantize_kernel<float>, a, s);
  else if (dtype == VP_BF16) launch_rows(mx_dequantize_kernel<Bf16>, a, s);
  else launch_rows(mx_dequantize_kernel<F16>, a, s);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "dequantise launch failed");
  return VP_OK;
}

}  // namespace vp
