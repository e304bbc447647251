// Dense products with bias, activation and residual, and their gradients.
//
//   forward   y = act(x W^T + b) + residual          (contraction over K)
//   grad x    d_x = (d_y W) act'(pre) + residual     (over N)
//   grad w    d_w = d_y^T x                          (over the rows, in 32 bits)
//   d_pre = d_y act'(pre), d_b = sum over rows of it
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act.h"
#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

constexpr int kTile = 64, kDepth = 16;

struct LinearArgs {
  const unsigned char *a, *b;
  int64_t a_stride, b_stride;
  int64_t M;
  int32_t N, C;
  const void* bias;
  bool bias_wide;
  int32_t act;
  const unsigned char *residual, *slope;
  int64_t residual_stride, slope_stride;
  unsigned char *out, *pre;
  bool out_wide;
  int64_t out_stride, pre_stride;
};

// A 64 x 64 tile of the output by 256 threads, sums of 32-bit products.  COLS: the operand's rows are the contraction.
template <typename T, bool COLS_A, bool COLS_B> __global__ void __launch_bounds__(256) linear_simple(LinearArgs a) {
  __shared__ float la[kDepth][kTile + 1], lb[kDepth][kTile + 1];
  const int64_t m0 = (int64_t)blockIdx.x * kTile;
  const int n0 = blockIdx.y * kTile;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  const auto at = [](const unsigned char* p, int64_t stride, bool cols, int64_t i, int64_t c) {
    return to_f32(*(const T*)(p + (cols ? c * stride + i * 2 : i * stride + c * 2)));
  };
  const int64_t depth = a.C;
  for (int64_t c0 = 0; c0 < depth; c0 += kDepth) {
    for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
      const int r = i / kDepth, c = i % kDepth;
      const bool in = c0 + c < depth;
      la[c][r] = in && m0 + r < a.M ? at(a.a, a.a_stride, COLS_A, m0 + r, c0 + c) : 0.0f;
      lb[c][r] = in && n0 + r < a.N ? at(a.b, a.b_stride, COLS_B, n0 + r, c0 + c) : 0.0f;
    }
    __syncthreads();
    for (int c = 0; c < kDepth; ++c)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] += la[c][ty + 16 * i] * lb[c][tx + 16 * j];
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty + 16 * i;
      const int n = n0 + tx + 16 * j;
      if (m >= a.M || n >= a.N) continue;
      float v = acc[i][j];
      if (a.bias) v += a.bias_wide ? ((const float*)a.bias)[n] : to_f32(((const T*)a.bias)[n]);
      if (a.pre) ((T*)(a.pre + m * a.pre_stride))[n] = from_f32<T>(v);
      const float before = a.slope ? to_f32(((const T*)(a.slope + m * a.slope_stride))[n]) : 0.0f;
      with_act(a.act, [&](auto act) { v = a.slope ? through<decltype(act)::value>(v, before) : activation<decltype(act)::value>(v); });
      const unsigned char* res = a.residual + m * a.residual_stride;
      unsigned char* out = a.out + m * a.out_stride;
      if (a.out_wide) {
        ((float*)out)[n] = v + (a.residual ? ((const float*)res)[n] : 0.0f);
      } else {
        ((T*)out)[n] = from_f32<T>(v + (a.residual ? to_f32(((const T*)res)[n]) : 0.0f));
      }
    }
}

// Through the activation, and columns' sums: workgroup (columns, part).
struct ActGradArgs {
  const unsigned char *d_y, *pre;
  int64_t d_y_stride, pre_stride, d_pre_stride;
  int64_t R, N;
  int32_t act;
  unsigned char* d_pre;
  float* part;   // [parts][N], or null
  int parts;
};

template <typename T> __global__ void __launch_bounds__(256) act_grad_kernel(ActGradArgs a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.N) return;
  float s = 0.0f;
  with_act(a.act, [&](auto act) {
    for (int64_t r = blockIdx.y; r < a.R; r += a.parts) {
      const float d = to_f32(((const T*)(a.d_y + r * a.d_y_stride))[c]);
      const float v = through<decltype(act)::value>(d, a.pre ? to_f32(((const T*)(a.pre + r * a.pre_stride))[c]) : 0.0f);
      if (a.d_pre) ((T*)(a.d_pre + r * a.d_pre_stride))[c] = from_f32<T>(v);
      s += v;
    }
  });
  if (a.part) a.part[(int64_t)blockIdx.y * a.N + c] = s;
}

int act_grad_parts(int64_t R) { return (int)std::min<int64_t>(R, 256); }

}  // namespace

size_t linear_workspace(int mode, int64_t R, int32_t N, int32_t K) { return 0; }

vp_status launch_linear(const LinearLaunch& p, void* stream) {
  const LinearArgs a{(const unsigned char*)p.a, (const unsigned char*)p.b, p.a_stride, p.b_stride,
                     p.mode == kExpertGradW ? p.N : p.R,
                     p.mode == kExpertForward ? p.N : p.K,
                     p.mode == kExpertForward ? p.K : p.mode == kExpertGradX ? p.N : (int32_t)p.R,
                     p.bias, p.bias_dtype == VP_F32, p.act, (const unsigned char*)p.residual, (const unsigned char*)p.slope,
                     p.residual_stride, p.slope_stride, (unsigned char*)p.out, (unsigned char*)p.pre,
                     p.out_dtype == VP_F32, p.out_stride, p.pre_stride};
  const dim3 grid((unsigned)((a.M + kTile - 1) / kTile), (unsigned)((a.N + kTile - 1) / kTile));
  const auto run = [&](auto t) {
    using T = decltype(t);
    if (p.mode == kExpertForward) hipLaunchKernelGGL((linear_simple<T, false, false>), grid, dim3(256), 0, (hipStream_t)stream, a);
    else if (p.mode == kExpertGradX) hipLaunchKernelGGL((linear_simple<T, false, true>), grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((linear_simple<T, true, true>), grid, dim3(256), 0, (hipStream_t)stream, a);
  };
  if (p.dtype == VP_BF16) run(Bf16{});
  else run(F16{});
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "dense product launch failed");
  return VP_OK;
}

size_t act_grad_workspace(int64_t R, int64_t N) { return (size_t)act_grad_parts(R) * N * 4; }

vp_status launch_act_grad(const void* d_y, int64_t d_y_stride, const void* pre, int64_t pre_stride, int32_t dtype,
                          int64_t R, int64_t N, int32_t act, void* d_pre, int64_t d_pre_stride, float* d_bias,
                          void* ws, void* stream) {
  const ActGradArgs a{(const unsigned char*)d_y, (const unsigned char*)pre, d_y_stride, pre_stride, d_pre_stride, R, N, act,
                      (unsigned char*)d_pre, d_bias ? (float*)ws : nullptr, act_grad_parts(R)};
  if (R > 0) {
    const dim3 grid((unsigned)((N + 255) / 256), a.parts);
    if (dtype == VP_F32) hipLaunchKernelGGL(act_grad_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else if (dtype == VP_BF16) hipLaunchKernelGGL(act_grad_kernel<Bf16>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(act_grad_kernel<F16>, grid, dim3(256), 0, (hipStream_t)stream, a);
    if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "activation gradient launch failed");
  }
  return d_bias ? launch_column_sums(a.part, a.parts, N, d_bias, stream) : VP_OK;
}

}  // namespace vp
