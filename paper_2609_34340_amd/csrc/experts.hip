// Products of ragged groups of rows with their experts' weights.
//
// The expert-major rows of local expert e are rows offsets[e] .. offsets[e+1]
// of a buffer; only the device knows the offsets.  Weights are [L][N][K].
//   forward   y = x W_e^T                  (contraction over K)
//   gated     y = silu(x G^T) * (x U^T)    G, U the halves of W_e's N rows
//   grad x    dx = dy W_e                  (over N)
//   grad w    dW_e = dy^T x                (over the expert's rows, in 32 bits)
// in bf16 or fp16 with 32-bit sums, and the forward product also with both
// operands in 4-bit blocks (mx.hip) on the scaled matrix instruction, which
// multiplies the values and applies the blocks' powers of two itself.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ inline void report(int32_t* status, int code) { atomicCAS(status, 0, code); }

enum { kForward = 0, kGradX = 1, kGradW = 2 };

struct ProductArgs {
  const unsigned char *a, *b;   // the operands of the output's rows and of its columns
  int64_t a_stride, b_stride;   // bytes between rows
  int64_t b_expert;             // bytes between experts' weights (or, for grad w, of the output)
  const int64_t* offsets;
  int64_t R;                    // rows of the buffers
  int32_t L, M, N, C;           // experts; grad w's output rows; output columns (gated: of y); contraction
  int32_t half;                 // gated: rows of W_e before the second half
  unsigned char *out, *pre;
  int64_t out_stride, pre_stride;
  int32_t* status;
};

struct Group { int e; int64_t lo, hi; };   // an expert and its rows, inside the buffer

__device__ inline Group group_of(const ProductArgs& a, int e) {
  Group g{e, a.offsets[e], a.offsets[e + 1]};
  g.lo = g.lo < 0 ? 0 : g.lo > a.R ? a.R : g.lo;
  g.hi = g.hi < g.lo ? g.lo : g.hi > a.R ? a.R : g.hi;
  return g;
}

// The expert that owns tile slot `slot` of `BM` rows, or -1.
template <int BM> __device__ inline int expert_of_slot(const ProductArgs& a, int64_t slot) {
  const int lane = threadIdx.x % 64;
  int n = 0;
  for (int e0 = 0; e0 < a.L; e0 += 64) {
    const int e = e0 + lane;
    const bool in = e < a.L && a.offsets[e] / BM + e <= slot;
    const unsigned long long m = __ballot(in);
    n += __popcll(m);
    if (m != ~0ull) break;
  }
  return __builtin_amdgcn_readfirstlane(n) - 1;
}

// Offsets that decrease or pass the buffer are the caller's error; products
// stay inside the buffers all the same.
__device__ inline void check_offsets(const ProductArgs& a) {
  for (int e = threadIdx.x; e < a.L; e += blockDim.x) {
    const int64_t lo = a.offsets[e], hi = a.offsets[e + 1];
    if (lo < 0 || hi < lo || hi > a.R) report(a.status, VP_ERR_INVALID_ARGUMENT);
  }
}

__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
template <typename T> struct Frag;
template <> struct Frag<Bf16> { using type = bf16x8; using elem = __bf16; };
template <> struct Frag<F16> { using type = f16x8; using elem = _Float16; };

__device__ inline float silu(float g) { return g / (1.0f + expf(-g)); }

// A simple product: one wavefront a 16 x 16 tile, fragments straight from memory.
template <typename T, int MODE, bool GATED>
__global__ void __launch_bounds__(64) product_simple(ProductArgs a) {
  const int lane = threadIdx.x, r = lane % 16, q = lane / 16;
  if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets(a);
  Group g;
  int64_t m0;
  if (MODE == kGradW) {
    g = group_of(a, blockIdx.z);
    m0 = (int64_t)blockIdx.x * 16;
  } else {
    const int e = expert_of_slot<16>(a, blockIdx.x);
    if (e < 0) return;
    g = group_of(a, e);
    m0 = g.lo + ((int64_t)blockIdx.x - (a.offsets[e] / 16 + e)) * 16;
    if (m0 >= g.hi) return;
  }
  const int n0 = blockIdx.y * 16;
  const int rows = (int)(g.hi - g.lo);
  constexpr int kSteps = GATED ? 2 : 1;
  f32x4 acc[kSteps] = {};
  const int C = MODE == kGradW ? rows : a.C;
  for (int c0 = 0; c0 < C; c0 += 32) {
    typename Frag<T>::type fa, fb[kSteps];
    using E = typename Frag<T>::elem;
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + q * 8 + i;
      uint16_t va = 0, vb[2] = {0, 0};
      if (c < C) {
        const int n = n0 + r;
        if (MODE == kGradW) {
          if (m0 + r < a.M) va = ((const uint16_t*)(a.a + (g.lo + c) * a.a_stride))[m0 + r];
          if (n < a.N) vb[0] = ((const uint16_t*)(a.b + (g.lo + c) * a.b_stride))[n];
        } else {
          if (m0 + r < g.hi) va = ((const uint16_t*)(a.a + (m0 + r) * a.a_stride))[c];
          for (int s = 0; s < kSteps; ++s)
            if (n < a.N)
              vb[s] = MODE == kForward ? ((const uint16_t*)(a.b + g.e * a.b_expert + (int64_t)(n + s * a.half) * a.b_stride))[c]
                                       : ((const uint16_t*)(a.b + g.e * a.b_expert + (int64_t)c * a.b_stride))[n];
        }
      }
      fa[i] = __builtin_bit_cast(E, va);
      for (int s = 0; s < kSteps; ++s)
        fb[s][i] = __builtin_bit_cast(E, vb[s]);
    }
    for (int s = 0; s < kSteps; ++s) acc[s] = mma(fb[s], fa, acc[s]);
  }
  for (int i = 0; i < 4; ++i) {
    const int n = n0 + q * 4 + i;
    const int64_t m = m0 + r;
    if (n >= a.N || m >= (MODE == kGradW ? a.M : g.hi)) continue;
    if (MODE == kGradW) {
      ((float*)(a.out + g.e * a.b_expert + m * a.out_stride))[n] = acc[0][i];
    } else if (GATED) {
      ((T*)(a.out + m * a.out_stride))[n] = from_f32<T>(silu(acc[0][i]) * acc[1][i]);
      if (a.pre) {
        ((T*)(a.pre + m * a.pre_stride))[n] = from_f32<T>(acc[0][i]);
        ((T*)(a.pre + m * a.pre_stride))[n + a.half] = from_f32<T>(acc[1][i]);
      }
    } else {
      ((T*)(a.out + m * a.out_stride))[n] = from_f32<T>(acc[0][i]);
    }
  }
}

// 4-bit blocks, the simple way: the scaled instruction takes 128 values of a
// row, 32 per lane with that lane's scale.
template <typename T, bool GATED>
__global__ void __launch_bounds__(64) product_simple_mx(ProductArgs a) {
  const int lane = threadIdx.x, r = lane % 16, q = lane / 16;
  if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets(a);
  const int e = expert_of_slot<16>(a, blockIdx.x);
  if (e < 0) return;
  const Group g = group_of(a, e);
  const int64_t m0 = g.lo + ((int64_t)blockIdx.x - (a.offsets[e] / 16 + e)) * 16;
  if (m0 >= g.hi) return;
  const int n0 = blockIdx.y * 16;
  constexpr int kSteps = GATED ? 2 : 1;
  f32x4 acc[kSteps] = {};
  const int blocks = a.C / 32;
  for (int b0 = 0; b0 < blocks; b0 += 4) {
    const int b = b0 + q;
    i32x4 va = {0, 0, 0, 0}, vb[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    int sa = 0, sb[2] = {0, 0};
    if (b < blocks) {
      if (m0 + r < g.hi) {
        const unsigned char* p = a.a + (m0 + r) * a.a_stride;
        va = *(const i32x4*)(p + b * 16);
        sa = p[a.C / 2 + b];
      }
      for (int s = 0; s < kSteps; ++s)
        if (n0 + r < a.N) {
          const unsigned char* p = a.b + e * a.b_expert + (int64_t)(n0 + r + s * a.half) * a.b_stride;
          vb[s] = *(const i32x4*)(p + b * 16);
          sb[s] = p[a.C / 2 + b];
        }
    }
    const i32x8 fa = {va[0], va[1], va[2], va[3], 0, 0, 0, 0};
    for (int s = 0; s < kSteps; ++s) {
      const i32x8 fb = {vb[s][0], vb[s][1], vb[s][2], vb[s][3], 0, 0, 0, 0};
      acc[s] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa, acc[s], 4, 4, 0, sb[s], 0, sa);
    }
  }
  for (int i = 0; i < 4; ++i) {
    const int n = n0 + q * 4 + i;
    const int64_t m = m0 + r;
    if (n >= a.N || m >= g.hi) continue;
    const float z = GATED ? silu(acc[0][i]) * acc[kSteps - 1][i] : acc[0][i];
    ((T*)(a.out + m * a.out_stride))[n] = from_f32<T>(z);
  }
}

// Gradient of the gate: with s = 1 / (1 + exp(-g)),
//   dg = dh u s (1 + g (1 - s)),   du = dh g s
// for every row of the experts; 16 bytes a thread, bound by HBM.
struct GateArgs {
  const unsigned char *dh, *pre;
  unsigned char* out;
  int64_t dh_stride, pre_stride, out_stride;
  const int64_t* offsets;
  int64_t R;
  int32_t L, half;
  int32_t* status;
};

template <typename T>
__global__ void __launch_bounds__(256) gate_grad_kernel(GateArgs a) {
  const int64_t first = a.offsets[0], last = a.offsets[a.L];
  if (first < 0 || last > a.R) {
    if (threadIdx.x == 0) report(a.status, VP_ERR_INVALID_ARGUMENT);
    return;
  }
  const int64_t m = blockIdx.x;
  if (m < first || m >= last) return;
  for (int c = threadIdx.x; c < a.half / 8; c += 256) {
    float dh[8], g[8], u[8];
    unpack16<T>(*(const u32x4*)(a.dh + m * a.dh_stride + c * 16), dh);
    unpack16<T>(*(const u32x4*)(a.pre + m * a.pre_stride + c * 16), g);
    unpack16<T>(*(const u32x4*)(a.pre + m * a.pre_stride + (int64_t)a.half * 2 + c * 16), u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = 1.0f / (1.0f + expf(-g[i])), n = 1.0f / (1.0f + expf(g[i]));
      const float du = dh[i] * g[i] * s;
      g[i] = dh[i] * u[i] * s * (1.0f + g[i] * n);
      u[i] = du;
    }
    *(u32x4*)(a.out + m * a.out_stride + c * 16) = pack16<T>(g);
    *(u32x4*)(a.out + m * a.out_stride + (int64_t)a.half * 2 + c * 16) = pack16<T>(u);
  }
}

}  // namespace

vp_status launch_expert_product(const ExpertLaunch& p, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  ProductArgs a{};
  a.a = (const unsigned char*)p.a;
  a.b = (const unsigned char*)p.b;
  a.a_stride = p.a_stride;
  a.b_stride = p.b_stride;
  a.offsets = p.offsets;
  a.R = p.R;
  a.L = p.L;
  a.out = (unsigned char*)p.out;
  a.pre = (unsigned char*)p.pre;
  a.out_stride = p.out_stride;
  a.pre_stride = p.pre_stride;
  a.status = p.status;
  const int64_t slots = p.R / 16 + p.L;
  if (p.mode == kExpertForward) {
    a.C = p.K;
    a.N = p.gated ? p.N / 2 : p.N;
    a.half = p.N / 2;
    a.b_expert = p.N * p.b_stride;
    const dim3 grid((unsigned)slots, (unsigned)((a.N + 15) / 16));
    if (p.mx) {
      if (p.dtype == VP_BF16 && p.gated) hipLaunchKernelGGL((product_simple_mx<Bf16, true>), grid, dim3(64), 0, s, a);
      else if (p.dtype == VP_BF16) hipLaunchKernelGGL((product_simple_mx<Bf16, false>), grid, dim3(64), 0, s, a);
      else if (p.gated) hipLaunchKernelGGL((product_simple_mx<F16, true>), grid, dim3(64), 0, s, a);
      else hipLaunchKernelGGL((product_simple_mx<F16, false>), grid, dim3(64), 0, s, a);
    } else {
      if (p.dtype == VP_BF16 && p.gated) hipLaunchKernelGGL((product_simple<Bf16, kForward, true>), grid, dim3(64), 0, s, a);
      else if (p.dtype == VP_BF16) hipLaunchKernelGGL((product_simple<Bf16, kForward, false>), grid, dim3(64), 0, s, a);
      else if (p.gated) hipLaunchKernelGGL((product_simple<F16, kForward, true>), grid, dim3(64), 0, s, a);
      else hipLaunchKernelGGL((product_simple<F16, kForward, false>), grid, dim3(64), 0, s, a);
    }
  } else if (p.mode == kExpertGradX) {
    a.C = p.N;
    a.N = p.K;
    a.b_expert = p.N * p.b_stride;
    const dim3 grid((unsigned)slots, (unsigned)((a.N + 15) / 16));
    if (p.dtype == VP_BF16) hipLaunchKernelGGL((product_simple<Bf16, kGradX, false>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((product_simple<F16, kGradX, false>), grid, dim3(64), 0, s, a);
  } else {
    a.M = p.N;
    a.N = p.K;
    a.b_expert = (int64_t)p.N * p.out_stride;
    const dim3 grid((unsigned)((a.M + 15) / 16), (unsigned)((a.N + 15) / 16), (unsigned)p.L);
    if (p.dtype == VP_BF16) hipLaunchKernelGGL((product_simple<Bf16, kGradW, false>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((product_simple<F16, kGradW, false>), grid, dim3(64), 0, s, a);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "expert product launch failed");
  return VP_OK;
}

vp_status launch_expert_gate_grad(const void* dh, int64_t dh_stride, const void* pre, int64_t pre_stride,
                                  int32_t dtype, int64_t R, int32_t half, const int64_t* offsets, int32_t L, void* out,
                                  int64_t out_stride, int32_t* status, void* stream) {
  const GateArgs a{(const unsigned char*)dh, (const unsigned char*)pre, (unsigned char*)out, dh_stride, pre_stride,
                   out_stride, offsets, R, L, half, status};
  if (R > 0) {
    if (dtype == VP_BF16) hipLaunchKernelGGL(gate_grad_kernel<Bf16>, dim3((unsigned)R), dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(gate_grad_kernel<F16>, dim3((unsigned)R), dim3(256), 0, (hipStream_t)stream, a);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "gate gradient launch failed");
  return VP_OK;
}

}  // namespace vp
