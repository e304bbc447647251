// The layer's output from the returned rows, and its gradient.
//
//   out_t    = residual_t + sum_j w_tj row_(t k + j)
//   d_row    = w d_out,   d_w = <d_out, row>
//
// A slot of weight zero adds nothing whatever its row holds (an assignment that
// was dropped leaves its row unwritten); its weight's gradient is the product
// too, unless that is no number: then 0.  Sums are
// in 32 bits and rounded once.  Every row is read once and the output written
// once: HBM bounds it.  One workgroup per token; a thread holds one 16-byte
// vector of the token and has up to eight rows' loads in flight.  4096 tokens
// of eight 14 KiB rows: 94 us, 5.6 TB/s (a 1 GiB copy 5.2); 96 tokens of eight
// 8 KiB rows 4.4 us, about a launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

constexpr int kMaxThreads = 512;
constexpr int kAhead = 8;   // rows whose loads are issued together

struct MergeArgs {
  int64_t T;
  const unsigned char* rows;
  int64_t row_stride;   // bytes
  const float* weights;
  int32_t k, vecs;      // 16-byte vectors of a row
  const unsigned char *residual, *d_out;
  int64_t residual_stride, d_out_stride;
  unsigned char *out, *d_rows;
  int64_t out_stride, d_rows_stride;
  float* d_weights;
};

template <typename T>
__global__ void __launch_bounds__(kMaxThreads) merge_kernel(MergeArgs a) {
  constexpr int n = Vec<T>::n;
  const int64_t t = block_index();
  if (t >= a.T) return;
  const float* w = a.weights + t * a.k;
  for (int c = threadIdx.x; c < a.vecs; c += blockDim.x) {
    float acc[n];
    if (a.residual) {
      unpack16<T>(*(const u32x4*)(a.residual + t * a.residual_stride + (int64_t)c * 16), acc);
    } else {
#pragma unroll
      for (int i = 0; i < n; ++i) acc[i] = 0.0f;
    }
    const unsigned char* src = a.rows + t * a.k * a.row_stride + (int64_t)c * 16;
    for (int j0 = 0; j0 < a.k; j0 += kAhead) {
      u32x4 r[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (j0 + j < a.k) r[j] = __builtin_nontemporal_load((const u32x4*)(src + (j0 + j) * a.row_stride));
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (j0 + j < a.k) {
          const float wj = w[j0 + j];
          if (wj != 0.0f) {
            float f[n];
            unpack16<T>(r[j], f);
#pragma unroll
            for (int i = 0; i < n; ++i) acc[i] = fmaf(wj, f[i], acc[i]);
          }
        }
    }
    *(u32x4*)(a.out + t * a.out_stride + (int64_t)c * 16) = pack16<T>(acc);
  }
}

// The token's d_out vectors stay in registers (up to kVecs per thread, then
// the row is walked again), four rows' loads are in flight; every slot's dot
// product is summed over the lanes, then over the wavefronts in their order.
// 8192 tokens of eight 4 KiB rows: 98 us, 5.8 TB/s (each row's loads
// waited for by itself, and the lanes' sums through LDS: 104; 96 tokens of eight
// 8 KiB rows 12.6 -> 7.7).
constexpr int kVecs = 2, kGradAhead = 4;
template <typename T>
__global__ void __launch_bounds__(kMaxThreads) merge_grad_kernel(MergeArgs a) {
  constexpr int n = Vec<T>::n;
  extern __shared__ float part[];   // [wavefronts][k]
  const int64_t t = block_index();
  if (t >= a.T) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
  const float* w = a.weights + t * a.k;
  for (int i = threadIdx.x; i < waves * a.k; i += blockDim.x) part[i] = 0.0f;
  __syncthreads();
  for (int base = 0; base < a.vecs; base += kVecs * blockDim.x) {   // every lane takes every pass: the sums below
    const int c0 = base + threadIdx.x;
    float d[kVecs][n];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int c = c0 + v * blockDim.x;
      u32x4 q = {0, 0, 0, 0};
      if (c < a.vecs) q = *(const u32x4*)(a.d_out + t * a.d_out_stride + (int64_t)c * 16);
      unpack16<T>(q, d[v]);
    }
    for (int j0 = 0; j0 < a.k; j0 += kGradAhead) {
      u32x4 q[kGradAhead][kVecs];
#pragma unroll
      for (int j = 0; j < kGradAhead; ++j)
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
          const int c = c0 + v * blockDim.x;
          q[j][v] = u32x4{0, 0, 0, 0};
          if (j0 + j < a.k && c < a.vecs)
            q[j][v] = __builtin_nontemporal_load((const u32x4*)(a.rows + (t * a.k + j0 + j) * a.row_stride + (int64_t)c * 16));
        }
#pragma unroll
      for (int j = 0; j < kGradAhead; ++j) {
        if (j0 + j >= a.k) break;
        const float wj = w[j0 + j];
        unsigned char* out = a.d_rows + (t * a.k + j0 + j) * a.d_rows_stride;
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
          const int c = c0 + v * blockDim.x;
          float f[n], g[n];
          unpack16<T>(q[j][v], f);
#pragma unroll
          for (int i = 0; i < n; ++i) {
            dot = fmaf(d[v][i], f[i], dot);
            g[i] = wj == 0.0f ? 0.0f : wj * d[v][i];
          }
          if (c < a.vecs) __builtin_nontemporal_store(pack16<T>(g), (u32x4*)(out + (int64_t)c * 16));
        }
        dot = across<64>(dot, [](float p, float q) { return p + q; });
        if (lane == 0) part[wave * a.k + j0 + j] += dot;
      }
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < a.k; j += blockDim.x) {
    float s = 0.0f;
    for (int v = 0; v < waves; ++v) s += part[v * a.k + j];
    a.d_weights[t * a.k + j] = w[j] == 0.0f && !isfinite(s) ? 0.0f : s;
  }
}

// Threads of a workgroup: the row's vectors over as few passes as the limit
// allows, spread evenly, up to whole wavefronts.
int threads_for(int64_t vecs, int most) {
  const int64_t passes = std::max<int64_t>(1, (vecs + most - 1) / most);
  return (int)std::max<int64_t>(64, ((vecs + passes - 1) / passes + 63) / 64 * 64);
}

}  // namespace

vp_status launch_merge(const void* rows, int32_t dtype, int64_t T, int32_t k, int64_t H, int64_t row_stride,
                       const float* weights, const void* residual, int64_t residual_stride, void* out,
                       int64_t out_stride, void* stream) {
  MergeArgs a{};
  a.T = T;
  a.rows = (const unsigned char*)rows;
  a.row_stride = row_stride;
  a.weights = weights;
  a.k = k;
  a.vecs = (int32_t)(H * dtype_size(dtype) / 16);
  a.residual = (const unsigned char*)residual;
  a.residual_stride = residual_stride;
  a.out = (unsigned char*)out;
  a.out_stride = out_stride;
  if (T > 0 && a.vecs > 0) {
    const dim3 grid = grid_of(T), block(threads_for(a.vecs, kMaxThreads));
    hipStream_t s = (hipStream_t)stream;
    if (dtype == VP_F32) hipLaunchKernelGGL(merge_kernel<float>, grid, block, 0, s, a);
    else if (dtype == VP_BF16) hipLaunchKernelGGL(merge_kernel<Bf16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(merge_kernel<F16>, grid, block, 0, s, a);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "merge launch failed");
  return VP_OK;
}

vp_status launch_merge_grad(const void* d_out, int32_t dtype, int64_t T, int32_t k, int64_t H, int64_t d_out_stride,
                            const void* rows, int64_t row_stride, const float* weights, void* d_rows,
                            int64_t d_rows_stride, float* d_weights, void* stream) {
  MergeArgs a{};
  a.T = T;
  a.rows = (const unsigned char*)rows;
  a.row_stride = row_stride;
  a.weights = weights;
  a.k = k;
  a.vecs = (int32_t)(H * dtype_size(dtype) / 16);
  a.d_out = (const unsigned char*)d_out;
  a.d_out_stride = d_out_stride;
  a.d_rows = (unsigned char*)d_rows;
  a.d_rows_stride = d_rows_stride;
  a.d_weights = d_weights;
  if (T > 0) {
    const int threads = threads_for((a.vecs + kVecs - 1) / kVecs, kMaxThreads);
    const dim3 grid = grid_of(T), block(threads);
    const size_t lds = (size_t)(threads / 64) * k * 4;
    hipStream_t s = (hipStream_t)stream;
    if (dtype == VP_F32) hipLaunchKernelGGL(merge_grad_kernel<float>, grid, block, lds, s, a);
    else if (dtype == VP_BF16) hipLaunchKernelGGL(merge_grad_kernel<Bf16>, grid, block, lds, s, a);
    else hipLaunchKernelGGL(merge_grad_kernel<F16>, grid, block, lds, s, a);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "merge gradient launch failed");
  return VP_OK;
}

}  // namespace vp
