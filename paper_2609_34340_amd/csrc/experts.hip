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
//
// A workgroup makes tiles of BM rows by BN columns of one expert.  Row tiles
// are numbered expert after expert from the offsets, by every wavefront for
// itself; the grid follows from the buffer's size.
// The tiles and their loads are product.h's.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "numeric.h"
#include "report.h"
#include "product.h"

namespace vp {
namespace {

// ----------------------------------------------------------- few rows

// Up to 64 rows of an expert by 32 of its weight rows (gated: 16 of the gate
// and the same 16 of the up half).  The weights' bytes bound it, so they go
// straight to registers, each read once with no LDS between: the four
// wavefronts take turns on 256-byte pieces of the rows (two steps), loads one
// piece ahead, and their sums are added in LDS in the wavefronts' order.  The
// rows of x come from the L2.
constexpr int kFewRows = 64, kFewCols = 32, kPiece = 256;

template <typename T, bool GATED, int MT>
__device__ inline void few_rows(const ProductArgs& a, const Group& g, int64_t m0, int n0, float* sums) {
#ifdef __HIP_DEVICE_COMPILE__
  using Out = typename Elem<T>::out;
  constexpr bool kMx = Elem<T>::mx;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, q = lane / 16;
  const int code_bytes = kMx ? a.C / 2 : a.C * 2;
  const int row_bytes = kMx ? (code_bytes + a.C / 32 + 15) / 16 * 16 : code_bytes;
  const int rows = (int)min((int64_t)(MT * 16), g.hi - m0);
  const int sx = (int)a.a_stride, sw = (int)a.b_stride;
  const auto rx = __builtin_amdgcn_make_buffer_rsrc((void*)(a.a + m0 * a.a_stride), 0, (rows - 1) * sx + row_bytes, 0x00020000);
  const auto weights = [&](int u) {
    const int n = GATED ? n0 : n0 + u * 16, valid = max(min(16, a.N - n), 0);
    const unsigned char* base = a.b + g.e * a.b_expert + (int64_t)(n + (GATED ? u * a.half : 0)) * a.b_stride;
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, valid > 0 ? (valid - 1) * sw + row_bytes : 0, 0x00020000);
  };
  const auto rw0 = weights(0), rw1 = weights(1);

  struct Piece {
    u32x4 w[2][4], x[MT][4];
    u32x4 ws[2], xs[MT];   // 4-bit blocks: sixteen powers of the row
  };
  const auto load = [&](Piece& p, int at) {   // `at`: the piece's first byte
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int byte = at + c * 64 + q * 16;
      const uint32_t off = byte < code_bytes ? (uint32_t)byte : 0x60000000u;   // past the row: zero
      p.w[0][c] = __builtin_amdgcn_raw_buffer_load_b128(rw0, off + r * sw, 0, 0);
      p.w[1][c] = __builtin_amdgcn_raw_buffer_load_b128(rw1, off + r * sw, 0, 0);
#pragma unroll
      for (int i = 0; i < MT; ++i) p.x[i][c] = __builtin_amdgcn_raw_buffer_load_b128(rx, off + (i * 16 + r) * sx, 0, 0);
    }
    if constexpr (kMx) {
      const uint32_t off = at < code_bytes ? code_bytes + at / 16 : 0x60000000u;
      p.ws[0] = __builtin_amdgcn_raw_buffer_load_b128(rw0, off + r * sw, 0, 0);
      p.ws[1] = __builtin_amdgcn_raw_buffer_load_b128(rw1, off + r * sw, 0, 0);
#pragma unroll
      for (int i = 0; i < MT; ++i) p.xs[i] = __builtin_amdgcn_raw_buffer_load_b128(rx, off + (i * 16 + r) * sx, 0, 0);
    }
  };
  f32x4 acc[2][MT] = {};
  const auto multiply = [&](const Piece& p, int at) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if constexpr (kMx) {
        const bool in = at + c * 64 + q * 16 < code_bytes;   // powers past the row: 2^-127, of zeros
        const auto power = [&](const u32x4& v) { return in ? (int)(v[c] >> (8 * q) & 0xff) : 0; };
        const auto wide = [](const u32x4& v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; };
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u)
            acc[u][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(p.w[u][c]), wide(p.x[i][c]), acc[u][i], 4, 4, 0,
                                                                         power(p.ws[u]), 0, power(p.xs[i]));
      } else {
        using F = typename Frag<T>::type;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) acc[u][i] = mma(__builtin_bit_cast(F, p.w[u][c]), __builtin_bit_cast(F, p.x[i][c]), acc[u][i]);
      }
    }
  };
  constexpr int kTurn = 4 * kPiece;
  Piece p0, p1;
  load(p0, wave * kPiece);
  for (int at = wave * kPiece; at < code_bytes; at += 2 * kTurn) {
    load(p1, at + kTurn);
    multiply(p0, at);
    load(p0, at + 2 * kTurn);
    multiply(p1, at + kTurn);
  }

  f32x4* part = (f32x4*)sums;   // [wavefront][column tile][row tile][lane]
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < MT; ++i) part[((wave * 2 + u) * MT + i) * 64 + lane] = acc[u][i];
  __syncthreads();
  for (int i = wave; i < MT; i += 4) {   // a row tile to a wavefront
    const int64_t m = m0 + i * 16 + r;
    f32x4 z[2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int w = 0; w < 4; ++w) z[u] += part[((w * 2 + u) * MT + i) * 64 + lane];
    if (m >= g.hi) continue;
    const auto put = [&](unsigned char* row, int n, f32x4 v) {
      u32x2 o;
      o.x = from_f32<Out>(v[0]).u | (uint32_t)from_f32<Out>(v[1]).u << 16;
      o.y = from_f32<Out>(v[2]).u | (uint32_t)from_f32<Out>(v[3]).u << 16;
      *(u32x2*)(row + (int64_t)n * 2) = o;
    };
    unsigned char* out = a.out + m * a.out_stride;
    const int n = n0 + q * 4;
    if constexpr (GATED) {
      if (n >= a.N) continue;
      if (a.pre) {
        put(a.pre + m * a.pre_stride, n, z[0]);
        put(a.pre + m * a.pre_stride, n + a.half, z[1]);
      }
      f32x4 h;
#pragma unroll
      for (int v = 0; v < 4; ++v) h[v] = silu(z[0][v]) * z[1][v];
      put(out, n, h);
    } else {
      if (n < a.N) put(out, n, z[0]);
      if (n + 16 < a.N) put(out, n + 16, z[1]);
    }
  }
#endif
}

template <typename T, bool GATED> __global__ void __launch_bounds__(256) product_few(ProductArgs a) {
  __shared__ float sums[4 * 2 * (kFewRows / 16) * 64 * 4];
  RowTiles<kFewRows> tiles;
  if (!tiles.init(a, threadIdx.x % 64)) {   // an error: nothing is written
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) report(a.status, VP_ERR_INVALID_ARGUMENT);
    return;
  }
  if (blockIdx.y >= tiles.total) return;
  int64_t m0;
  const Group g = tiles.find(a, blockIdx.y, &m0);
  const int n0 = blockIdx.x * (GATED ? kFewCols / 2 : kFewCols);
  const int64_t rows = g.hi - m0;
  if (rows <= 16) few_rows<T, GATED, 1>(a, g, m0, n0, sums);
  else if (rows <= 32) few_rows<T, GATED, 2>(a, g, m0, n0, sums);
  else few_rows<T, GATED, 4>(a, g, m0, n0, sums);
}

// Gradient of the gate: with s = 1 / (1 + exp(-g)),
//   dg = dh u s (1 + g (1 - s)),   du = dh g s
// for every row of the experts; 16 bytes a thread, bound by HBM: 32768 rows of
// 2048 117 us, 5.7 TB/s (163 us with the library's exponential and divide).
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
  const int64_t m = block_index(), first = a.offsets[0], last = a.offsets[a.L];
  if (m == 0) {
    for (int e = threadIdx.x; e < a.L; e += blockDim.x)
      if (!in_order(a, e)) report(a.status, VP_ERR_INVALID_ARGUMENT);
  }
  if (first < 0 || last > a.R || m < first || m >= last) return;
  for (int c = threadIdx.x; c < a.half / 8; c += 256) {
    float dh[8], g[8], u[8];
    unpack16<T>(*(const u32x4*)(a.dh + m * a.dh_stride + c * 16), dh);
    unpack16<T>(*(const u32x4*)(a.pre + m * a.pre_stride + c * 16), g);
    unpack16<T>(*(const u32x4*)(a.pre + m * a.pre_stride + (int64_t)a.half * 2 + c * 16), u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = logistic(g[i]), du = dh[i] * g[i] * s;
      g[i] = dh[i] * u[i] * s * (1.0f + g[i] * (1.0f - s));
      u[i] = du;
    }
    *(u32x4*)(a.out + m * a.out_stride + c * 16) = pack16<T>(g);
    *(u32x4*)(a.out + m * a.out_stride + (int64_t)a.half * 2 + c * 16) = pack16<T>(u);
  }
}

}  // namespace

namespace {

// One workgroup per CU runs through its share of the tiles; grad w's tiles have
// their experts' lengths, so there every tile is a workgroup of its own and
// the hardware hands them out.
template <typename T, int MODE, bool GATED, int WM, int WN, int MT, int NT>
vp_status launch_tiled(const ProductArgs& a, hipStream_t s) {
  constexpr int BM = WM * MT * 16, kTileN = WN * NT * 16 / (GATED ? 2 : 1);
  const int64_t nt = (a.N + kTileN - 1) / kTileN;
  int64_t per = MODE == kGradW ? (((a.M + BM - 1) / BM) * nt + 7) / 8 * a.L : ((a.R / BM + a.L) * nt + 7) / 8;
  if (per * 8 >= (int64_t)1 << 31) return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 tiles");
  // (a dimension of a grid holds fewer than 2^32 threads: grad w's workgroups take more than one of very many tiles)
  per = std::min<int64_t>(per, MODE == kGradW ? 1 << 19 : kCus / 8 * (BM == 128 ? 2 : 1));
  hipLaunchKernelGGL((product_tiled<T, MODE, GATED, WM, WN, MT, NT>), dim3((unsigned)(per * 8)), dim3(WM * WN * 64), 0, s, a);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "expert product launch failed");
  return VP_OK;
}

// Which kernel, from the sizes the host knows (R rows at most, spread over L
// experts; a buffer much larger than its rows in use selects tiles: 61 rows at
// four experts of 4096 x 4096, gated, 27 us in a buffer of 61, 61 in one of
// 512).  Few rows: the weights are read again for every 64 rows, at about 3.6
// TB/s (2.5 in 4-bit blocks); tiles take 0.85 us a step of the contraction
// (1.35) and 6 us around it for each round of workgroups, and read all weights
// at 4.5 TB/s or less.  Measured, few rows against tiles, us: 64 rows at 4
// experts of 4096 x 4096 35 / 60, 256 at 4 50 / 60, 256 at 1 48 / 60, 512 at 1
// 91 / 62, 512 at 8 of 2048 x 2048 29 / 33, 768 at 8 52 / 35; in 4-bit blocks
// 256 at 1 of 4096 x 4096 19 / 27, 512 at 1 34 / 27.
template <typename T> bool few_rows_win(const ProductArgs& a, int64_t weight_rows) {
  constexpr bool kMx = Elem<T>::mx;
  const int64_t tiles = a.R / kFewRows + a.L;
  if (tiles >= 65536) return false;   // the grid's second dimension
  const double expert = (double)weight_rows * (double)a.b_stride;   // bytes
  const double few = ((double)a.R / kFewRows + 0.5 * a.L) * expert / (kMx ? 2500.0 : 3600.0);   // ns
  const double rounds = std::max(1.0, ((double)a.R / 256 + 0.5 * a.L) * ((double)weight_rows / 256) / kCus);
  const double steps = (double)a.C / (kMx ? 256 : 64);
  return few < std::max((6000.0 + (kMx ? 1350.0 : 850.0) * steps) * rounds, a.L * expert / 4500.0);
}

// 128 x 128 tiles where they are at most two and a half for each CU, else 256 x
// 256.  Measured, 128 against 256, us: 2048 rows, one expert, 2048 x 2048 39 / 52,
// 4096 rows at 8 of them 48 / 54, 2048 rows at 4 of 4096 x 4096 87 / 94, 8192 rows
// at 8 of 2048 x 2048 93 / 67, 4096 rows, one of 4096 x 4096 185 / 119.  Grad w
// where 256 x 256 leave half of the CUs without a tile: 2048 rows, one expert,
// 2048 x 2048 42 / 59, 1024 rows at 8 of them (512 tiles) 40 / 36.
template <typename T, int MODE, bool GATED> vp_expert_kind kind_of(const ProductArgs& a) {
  const int64_t columns = GATED ? 2 * (int64_t)a.N : a.N;
  if constexpr (MODE == kForward) {
    if (few_rows_win<T>(a, columns)) return VP_EXPERT_FEW_ROWS;
  }
  const bool small = MODE == kGradW ? (int64_t)a.L * ((a.M + 255) / 256) * ((a.N + 255) / 256) <= kCus / 2
                                    : (a.R / 128 + a.L / 2 + 1) * ((columns + 127) / 128) <= kCus * 5 / 2;
  return small ? VP_EXPERT_TILES_128 : VP_EXPERT_TILES_256;
}

template <typename T, int MODE, bool GATED> vp_status launch_product_as(const ProductArgs& a, hipStream_t s) {
  const vp_expert_kind kind = kind_of<T, MODE, GATED>(a);
  if constexpr (MODE == kForward) {
    if (kind == VP_EXPERT_FEW_ROWS) {
      const unsigned cols = GATED ? kFewCols / 2 : kFewCols;
      hipLaunchKernelGGL((product_few<T, GATED>), dim3((a.N + cols - 1) / cols, (unsigned)(a.R / kFewRows + a.L)), dim3(256), 0, s, a);
      if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "expert product launch failed");
      return VP_OK;
    }
  }
  return kind == VP_EXPERT_TILES_128 ? launch_tiled<T, MODE, GATED, 2, 2, 4, 4>(a, s)
                                     : launch_tiled<T, MODE, GATED, 2, 4, 8, 4>(a, s);
}

// Calls f with the product's element type, direction and gate as types.
template <typename F> auto as_types(const ExpertLaunch& p, F f) {
  const bool bf = p.dtype == VP_BF16;
  const auto typed = [&](auto mode, auto gated) {
    return bf ? f(Bf16{}, mode, gated) : f(F16{}, mode, gated);
  };
  if (p.mode == kExpertGradX) return typed(std::integral_constant<int, kGradX>{}, std::false_type{});
  if (p.mode == kExpertGradW) return typed(std::integral_constant<int, kGradW>{}, std::false_type{});
  constexpr std::integral_constant<int, kForward> forward{};
  if (!p.mx) return p.gated ? typed(forward, std::true_type{}) : typed(forward, std::false_type{});
  if (p.gated) return bf ? f(Mx<Bf16>{}, forward, std::true_type{}) : f(Mx<F16>{}, forward, std::true_type{});
  return bf ? f(Mx<Bf16>{}, forward, std::false_type{}) : f(Mx<F16>{}, forward, std::false_type{});
}

ProductArgs product_args(const ExpertLaunch& p) {
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
  if (p.mode == kExpertForward) {
    a.C = p.K;
    a.N = p.gated ? p.N / 2 : p.N;
    a.half = p.N / 2;
    a.b_expert = p.N * p.b_stride;
  } else if (p.mode == kExpertGradX) {
    a.C = p.N;
    a.N = p.K;
    a.b_expert = p.N * p.b_stride;
  } else {
    a.M = p.N;
    a.N = p.K;
    a.b_expert = (int64_t)p.N * p.out_stride;
  }
  return a;
}

}  // namespace

vp_status launch_expert_product(const ExpertLaunch& p, void* stream) {
  const ProductArgs a = product_args(p);
  return as_types(p, [&](auto type, auto mode, auto gated) {
    return launch_product_as<decltype(type), decltype(mode)::value, decltype(gated)::value>(a, (hipStream_t)stream);
  });
}

vp_expert_kind expert_kind(const ExpertLaunch& p) {
  const ProductArgs a = product_args(p);
  return as_types(p, [&](auto type, auto mode, auto gated) {
    return kind_of<decltype(type), decltype(mode)::value, decltype(gated)::value>(a);
  });
}

vp_status launch_expert_gate_grad(const void* dh, int64_t dh_stride, const void* pre, int64_t pre_stride,
                                  int32_t dtype, int64_t R, int32_t half, const int64_t* offsets, int32_t L, void* out,
                                  int64_t out_stride, int32_t* status, void* stream) {
  const GateArgs a{(const unsigned char*)dh, (const unsigned char*)pre, (unsigned char*)out, dh_stride, pre_stride,
                   out_stride, offsets, R, L, half, status};
  if (R > 0) {
    if (dtype == VP_BF16) hipLaunchKernelGGL(gate_grad_kernel<Bf16>, grid_of(R), dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(gate_grad_kernel<F16>, grid_of(R), dim3(256), 0, (hipStream_t)stream, a);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "gate gradient launch failed");
  return VP_OK;
}

vp_status take_unclaimed_experts(int32_t* out, void* stream) {
  hipLaunchKernelGGL(take_unclaimed_kernel, dim3(1), dim3(1), 0, (hipStream_t)stream, out);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "status launch failed");
  return VP_OK;
}

}  // namespace vp
