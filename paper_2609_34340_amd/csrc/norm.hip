// Layer norm over rows, its gradient, and sums over rows.
//
//   y = (x - m) r w + b,  m = mean(x) or 0,  r = 1 / sqrt(mean((x - m)^2) + eps)
//   u = (x - m) r, g = d_out w:  d_x = r (g - mean(g) - u mean(g u)) + residual
//   d_w = sum over rows of d_out u,  d_b = sum over rows of d_out
//
// Statistics by two passes over the row: a mean m0, then d = x - m0 with sum(d) and sum(d^2), so that m = m0 + sum(d) / H
// and the variance is (sum(d^2) - sum(d)^2 / H) / H: nothing large cancels whatever the rows' mean.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

constexpr int kThreads = 256;

struct NormArgs {
  int64_t T, H;
  const unsigned char *x, *d_out, *residual;
  const void *weight, *bias;
  bool wide;   // weight and bias are fp32
  bool center;
  int64_t x_stride, d_out_stride, residual_stride, out_stride;
  unsigned char* out;
  float* stats;
  const float* given;
  float eps;
  float* part;   // [parts][d_weight, d_bias][H]
  int parts;
};

template <typename T> __device__ inline float param(const void* p, bool wide, int64_t c) {
  return wide ? ((const float*)p)[c] : to_f32(((const T*)p)[c]);
}

// Sums of a and b over the workgroup, in every thread.
struct Pair { float a, b; };
__device__ inline Pair block_sum(Pair v, Pair* lds) {
  const auto add = [](float p, float q) { return p + q; };
  v.a = across<64>(v.a, add);
  v.b = across<64>(v.b, add);
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  Pair s{0.0f, 0.0f};
  for (int w = 0; w < kThreads / 64; ++w) {
    s.a += lds[w].a;
    s.b += lds[w].b;
  }
  __syncthreads();
  return s;
}

template <typename T> __global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs a) {
  __shared__ Pair lds[kThreads / 64];
  const int64_t t = block_index();
  if (t >= a.T) return;
  const T* x = (const T*)(a.x + t * a.x_stride);
  T* y = (T*)(a.out + t * a.out_stride);
  const float n = (float)a.H;
  float m = 0.0f;
  if (a.center) {
    Pair s{0.0f, 0.0f};
    for (int64_t c = threadIdx.x; c < a.H; c += kThreads) s.a += to_f32(x[c]);
    m = block_sum(s, lds).a / n;
  }
  Pair s{0.0f, 0.0f};
  for (int64_t c = threadIdx.x; c < a.H; c += kThreads) {
    const float d = to_f32(x[c]) - m;
    s.a += d;
    s.b += d * d;
  }
  s = block_sum(s, lds);
  const float shift = a.center ? s.a / n : 0.0f;
  const float left = s.b - s.a * shift;   // never below 0 but by rounding
  const float r = 1.0f / sqrtf((left < 0.0f ? 0.0f : left / n) + a.eps);
  if (a.stats && threadIdx.x == 0) {
    a.stats[2 * t] = m + shift;
    a.stats[2 * t + 1] = r;
  }
  for (int64_t c = threadIdx.x; c < a.H; c += kThreads) {
    float v = (to_f32(x[c]) - m - shift) * r;
    if (a.weight) v *= param<T>(a.weight, a.wide, c);
    if (a.bias) v += param<T>(a.bias, a.wide, c);
    y[c] = from_f32<T>(v);
  }
}

// Rows' shares of d_weight and d_bias: workgroup (columns, part).
template <typename T> __global__ void __launch_bounds__(kThreads) norm_params_kernel(NormArgs a) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.H) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t t = blockIdx.y; t < a.T; t += a.parts) {
    const float d = to_f32(((const T*)(a.d_out + t * a.d_out_stride))[c]);
    dw += d * ((to_f32(((const T*)(a.x + t * a.x_stride))[c]) - a.given[2 * t]) * a.given[2 * t + 1]);
    db += d;
  }
  a.part[(int64_t)blockIdx.y * a.H + c] = dw;
  a.part[((int64_t)a.parts + blockIdx.y) * a.H + c] = db;
}

template <typename T> __global__ void __launch_bounds__(kThreads) norm_grad_kernel(NormArgs a) {
  __shared__ Pair lds[kThreads / 64];
  const int64_t t = block_index();
  if (t >= a.T) return;
  const T *x = (const T*)(a.x + t * a.x_stride), *d = (const T*)(a.d_out + t * a.d_out_stride);
  const float m = a.given[2 * t], r = a.given[2 * t + 1], n = (float)a.H;
  const auto grad = [&](int64_t c) { return to_f32(d[c]) * (a.weight ? param<T>(a.weight, a.wide, c) : 1.0f); };
  Pair s{0.0f, 0.0f};
  for (int64_t c = threadIdx.x; c < a.H; c += kThreads) {
    const float g = grad(c);
    s.a += g;
    s.b += g * ((to_f32(x[c]) - m) * r);
  }
  s = block_sum(s, lds);
  const float mg = a.center ? s.a / n : 0.0f, mgu = s.b / n;
  for (int64_t c = threadIdx.x; c < a.H; c += kThreads) {
    float v = r * (grad(c) - mg - (to_f32(x[c]) - m) * r * mgu);
    if (a.residual) v += to_f32(((const T*)(a.residual + t * a.residual_stride))[c]);
    ((T*)(a.out + t * a.out_stride))[c] = from_f32<T>(v);
  }
}

__global__ void __launch_bounds__(kThreads) column_sums_kernel(const float* part, int parts, int64_t H, float* out) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= H) return;
  float s = 0.0f;
  for (int i = 0; i < parts; ++i) s += part[(int64_t)i * H + c];
  out[c] = s;
}

int norm_parts(int64_t T) { return (int)std::min<int64_t>(T, 256); }

NormArgs norm_args(const NormLaunch& p) {
  NormArgs a{};
  a.T = p.T;
  a.H = p.H;
  a.x = (const unsigned char*)p.x;
  a.d_out = (const unsigned char*)p.d_out;
  a.residual = (const unsigned char*)p.residual;
  a.weight = p.weight;
  a.bias = p.bias;
  a.wide = p.param_dtype == VP_F32;
  a.center = p.center;
  a.x_stride = p.x_stride;
  a.d_out_stride = p.d_out_stride;
  a.residual_stride = p.residual_stride;
  a.out_stride = p.out_stride;
  a.out = (unsigned char*)p.out;
  a.stats = p.stats;
  a.given = p.given;
  a.eps = p.eps;
  a.part = (float*)p.ws;
  a.parts = norm_parts(p.T);
  return a;
}

template <typename F> void typed(int32_t dtype, F f) {
  if (dtype == VP_F32) f(float{});
  else if (dtype == VP_BF16) f(Bf16{});
  else f(F16{});
}

}  // namespace

vp_status launch_column_sums(const float* part, int parts, int64_t H, float* out, void* stream) {
  hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((H + kThreads - 1) / kThreads)), dim3(kThreads), 0, (hipStream_t)stream,
                     part, parts, H, out);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "column sum launch failed");
  return VP_OK;
}

vp_status launch_layer_norm(const NormLaunch& p, void* stream) {
  const NormArgs a = norm_args(p);
  typed(p.dtype, [&](auto t) {
    hipLaunchKernelGGL(norm_kernel<decltype(t)>, grid_of(a.T), dim3(kThreads), 0, (hipStream_t)stream, a);
  });
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "norm launch failed");
  return VP_OK;
}

size_t layer_norm_grad_workspace(int64_t T, int64_t H) { return (size_t)norm_parts(T) * 2 * H * 4; }

vp_status launch_layer_norm_grad(const NormLaunch& p, void* stream) {
  const NormArgs a = norm_args(p);
  if (p.d_weight || p.d_bias) {   // before d_x, which may take d_out's place
    if (a.T > 0) {
      typed(p.dtype, [&](auto t) {
        hipLaunchKernelGGL(norm_params_kernel<decltype(t)>, dim3((unsigned)((a.H + kThreads - 1) / kThreads), a.parts),
                           dim3(kThreads), 0, (hipStream_t)stream, a);
      });
    }
    if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "norm gradient launch failed");
    vp_status st = VP_OK;
    if (p.d_weight) st = launch_column_sums(a.part, a.parts, a.H, p.d_weight, stream);
    if (st == VP_OK && p.d_bias) st = launch_column_sums(a.part + a.parts * a.H, a.parts, a.H, p.d_bias, stream);
    if (st != VP_OK) return st;
  }
  if (a.T > 0) {
    typed(p.dtype, [&](auto t) {
      hipLaunchKernelGGL(norm_grad_kernel<decltype(t)>, grid_of(a.T), dim3(kThreads), 0, (hipStream_t)stream, a);
    });
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "norm gradient launch failed");
  return VP_OK;
}

}  // namespace vp
