// Dense products with bias, activation and residual, and their gradients.
//
//   forward   y = act(x W^T + b) + residual          (contraction over K)
//   grad x    d_x = (d_y W) act'(pre) + residual     (over N)
//   grad w    d_w = d_y^T x                          (over the rows, in 32 bits)
//   d_pre = d_y act'(pre), d_b = sum over rows of it
//
// Many rows go through product.h's tiles, of 128 x 128 or 256 x 256 results,
// few through linear_few (up to 32, and up to 128 by fewer columns).  Where the results are too few for 256 CUs the
// contraction is taken in parts, whose sums linear_join adds in their order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "act.h"
#include "divide.h"
#include "internal.h"
#include "numeric.h"
#include "product.h"
#include "rows.h"

namespace vp {
namespace {

// Four neighbouring results of row m from column n on: the epilogue and the store.
template <typename T> __device__ inline void finish4(const DenseArgs& a, int64_t m, int n, f32x4 v) {
  const auto half4 = [](const unsigned char* p) {
    const u32x2 h = *(const u32x2*)p;
    return f32x4{to_f32(T{(uint16_t)(h.x & 0xffffu)}), to_f32(T{(uint16_t)(h.x >> 16)}), to_f32(T{(uint16_t)(h.y & 0xffffu)}),
                 to_f32(T{(uint16_t)(h.y >> 16)})};
  };
  const auto put_half = [&](unsigned char* p) {
    u32x2 o;
    o.x = from_f32<T>(v[0]).u | (uint32_t)from_f32<T>(v[1]).u << 16;
    o.y = from_f32<T>(v[2]).u | (uint32_t)from_f32<T>(v[3]).u << 16;
    *(u32x2*)p = o;
  };
  if (a.bias) v += bias4<T>(a, n);
  if (a.pre) put_half(a.pre + m * a.pre_stride + (int64_t)n * 2);
  if (a.slope) {
    const f32x4 z = half4(a.slope + m * a.slope_stride + (int64_t)n * 2);
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = through<decltype(act)::value>(v[i], z[i]);
    });
  } else {
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = activation<decltype(act)::value>(v[i]);
    });
  }
  if (a.wide) {
    if (a.residual) v += *(const f32x4*)(a.residual + m * a.residual_stride + (int64_t)n * 4);
    *(f32x4*)(a.out + m * a.out_stride + (int64_t)n * 4) = v;
  } else {
    if (a.residual) v += half4(a.residual + m * a.residual_stride + (int64_t)n * 2);
    put_half(a.out + m * a.out_stride + (int64_t)n * 2);
  }
}

// ----------------------------------------------------------- few rows

// Up to 64 rows by 64 columns of one part of the contraction, forward.  The
// weights go straight to registers, each read once.  The rows of x would be
// read again for every 16 columns (64 rows by 4096 x 4096: 64 MB from the L2, 7
// us), so they go through LDS, a chunk of 256 values at a time: two wavefronts
// for 32 columns each, and two more for the other half of the chunk, whose sums
// are added in LDS at the end.  Loads run two chunks ahead.  16-byte piece c of
// row r lies at place c ^ (r & 15), so that a fragment's 16 rows meet no bank
// twice.  Few rows are bound by the weights' bytes (one row by 16384 x 4096 at
// 4.4 TB/s), 64 by a chunk's way through LDS and its barrier, 1.7 us against
// 1.06 with up to 16: 61 rows by 4096 x 4096, weights from memory, in four
// parts: 13 us (2.6 TB/s), and 4 for the join; 96 by 256 x 7168 in 14: 7.5 and
// 4.5.  Tried and dropped: four chunks ahead for up to 32 rows (12.5 -> 13.0
// us at one row: the weights' rate bounds it, not their latency), up to 16 rows
// by 16 columns without parts (10.4 -> 8.6 us at one row by 4096 x 4096, 11.0 ->
// 11.4 at 16 rows, 17 -> 20 at 16 by 8192 x 4096).
constexpr int kFewRows = 64, kFewCols = 64, kFewChunk = 256;

template <typename T, int MT>
__device__ inline void few_rows(const DenseArgs& a, int64_t m0, int n0, int part, unsigned char* lds) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int kRow = kFewChunk * 2, kBuffer = MT * 16 * kRow, kAhead = 2;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, q = lane / 16, group = wave % 2, half = wave / 2;
  const int rows = (int)min((int64_t)(MT * 16), a.R - m0);
  const int c0 = part * a.chunk, bytes = min(a.chunk, a.C - c0) * 2;   // of the part
  const int sx = (int)a.a_stride, sw = (int)a.b_stride;
  const auto rx = __builtin_amdgcn_make_buffer_rsrc((void*)(a.a + m0 * a.a_stride + (int64_t)c0 * 2), 0,
                                                    (rows - 1) * sx + bytes, 0x00020000);
  const auto weights = [&](int u) {
    const int n = n0 + group * 32 + u * 16, valid = max(min(16, a.N - n), 0);
    return __builtin_amdgcn_make_buffer_rsrc((void*)(a.b + (int64_t)n * a.b_stride + (int64_t)c0 * 2), 0,
                                             valid > 0 ? (valid - 1) * sw + bytes : 0, 0x00020000);
  };
  const auto rw0 = weights(0), rw1 = weights(1);
  struct Chunk { u32x4 w[2][4], x[2 * MT]; } ahead[kAhead];
  const int row0 = threadIdx.x / 32, piece = threadIdx.x % 32;   // of x, as this thread brings it
  const auto load_x = [&](Chunk& k, int at) {   // `at`: the chunk's first byte; past the part: zero
    const uint32_t off = at + piece * 16 < bytes ? (uint32_t)(at + piece * 16) : 0x60000000u;
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) k.x[i] = __builtin_amdgcn_raw_buffer_load_b128(rx, off + (row0 + 8 * i) * sx, 0, 0);
  };
  const auto load_w = [&](Chunk& k, int at) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int byte = at + half * (kRow / 2) + c * 64 + q * 16;
      const uint32_t off = byte < bytes ? (uint32_t)byte : 0x60000000u;
      k.w[0][c] = __builtin_amdgcn_raw_buffer_load_b128(rw0, off + r * sw, 0, 0);
      k.w[1][c] = __builtin_amdgcn_raw_buffer_load_b128(rw1, off + r * sw, 0, 0);
    }
  };
  f32x4 acc[2][MT] = {};
  const auto chunk = [&](Chunk& k, unsigned char* buffer, int at) {
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
      const int row = row0 + 8 * i;
      *(u32x4*)(buffer + row * kRow + (piece ^ (row & 15)) * 16) = k.x[i];
    }
    load_x(k, at + kAhead * kRow);
    __syncthreads();   // one for each chunk: a wavefront here has read the chunk before the last, whose buffer this was
    using F = typename Frag<T>::type;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      u32x4 x[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) x[i] = *(const u32x4*)(buffer + (i * 16 + r) * kRow + (((half * 4 + c) * 4 + q) ^ r) * 16);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[u][i] = mma(__builtin_bit_cast(F, k.w[u][c]), __builtin_bit_cast(F, x[i]), acc[u][i]);
    }
    load_w(k, at + kAhead * kRow);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    load_x(ahead[i], i * kRow);
    load_w(ahead[i], i * kRow);
  }
  for (int at = 0; at < bytes; at += kAhead * kRow) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) chunk(ahead[i], lds + (i & 1) * kBuffer, at + i * kRow);   // past the part: zeros
  }
  __syncthreads();
  f32x4* each = (f32x4*)lds;   // [wavefront][column tile][row tile][lane]
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < MT; ++i) each[((wave * 2 + u) * MT + i) * 64 + lane] = acc[u][i];
  __syncthreads();
  // the two halves' sums: a column tile to a wavefront
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int n = n0 + group * 32 + half * 16 + q * 4;
    const int64_t m = m0 + i * 16 + r;
    const f32x4 z = each[((group * 2 + half) * MT + i) * 64 + lane] + each[(((group + 2) * 2 + half) * MT + i) * 64 + lane];
    if (m >= a.R || n >= a.N) continue;
    if (a.raw) *(f32x4*)(a.out + part * a.part_bytes + m * a.out_stride + (int64_t)n * 4) = z;
    else finish4<T>(a, m, n, z);
  }
#endif
}

template <typename T, int MT> __global__ void __launch_bounds__(256, 2) linear_few(DenseArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * MT * 16 * kFewChunk * 2];
  few_rows<T, MT>(a, (int64_t)blockIdx.z * kFewRows, blockIdx.x * kFewCols, blockIdx.y, lds);
}

// The parts' sums [parts][M][N] in their order, and the epilogue: four neighbouring results a thread.
template <typename T> __global__ void __launch_bounds__(256) linear_join(DenseArgs a, const float* sums, int parts, int64_t M) {
  const int64_t i = block_index() * 256 + threadIdx.x;
  const int quads = a.N / 4;
  if (i >= M * quads) return;
  const int64_t m = fdiv53(i, quads);
  f32x4 v = {};
#pragma unroll 8
  for (int p = 0; p < parts; ++p) v += *(const f32x4*)(sums + (p * M * quads + i) * 4);
  finish4<T>(a, m, (int)(i - m * quads) * 4, v);
}

// Through the activation, and the columns' sums.  A wavefront has 64 pieces of
// 16 bytes of a row; the workgroup's four take turns on the rows of one part,
// kActAhead rows' loads at a time, and join their columns' sums in LDS.  HBM
// bounds it: gelu's of 8191 rows of 4096, bf16, 42 us, 4.8 TB/s, and 4.7 for the
// parts' sums.
struct ActGradArgs {
  const unsigned char *d_y, *pre;
  int64_t d_y_stride, pre_stride, d_pre_stride;
  int64_t R;
  int32_t N;
  unsigned char* d_pre;
  float* part;   // [parts][N], or null
  int parts;
};
constexpr int kActAhead = 4;

template <typename T, int ACT> __global__ void __launch_bounds__(256) act_grad_kernel(ActGradArgs a) {
  constexpr int n = Vec<T>::n;
  __shared__ float lds[4][64 * n];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int c = ((int)blockIdx.x * 64 + lane) * n, left = a.N - c;
  const int64_t stride = (int64_t)a.parts * 4;
  float s[n] = {};
  for (int64_t r0 = (int64_t)blockIdx.y * 4 + wave; r0 < a.R; r0 += stride * kActAhead) {
    u32x4 d[kActAhead], z[kActAhead];
#pragma unroll
    for (int i = 0; i < kActAhead; ++i) {
      const int64_t r = r0 + i * stride;
      const int in = r < a.R ? left : 0;
      d[i] = load_piece((const T*)(a.d_y + r * a.d_y_stride) + c, in);
      if constexpr (ACT != VP_ACT_NONE) z[i] = load_piece((const T*)(a.pre + r * a.pre_stride) + c, in);
    }
#pragma unroll
    for (int i = 0; i < kActAhead; ++i) {
      const int64_t r = r0 + i * stride;
      if (r >= a.R) break;
      float f[n], v[n];
      unpack16<T>(d[i], f);
      if constexpr (ACT != VP_ACT_NONE) {
        unpack16<T>(z[i], v);
#pragma unroll
        for (int e = 0; e < n; ++e) f[e] = through<ACT>(f[e], v[e]);
      }
      if (a.d_pre) store_piece((T*)(a.d_pre + r * a.d_pre_stride) + c, pack16<T>(f), left);
#pragma unroll
      for (int e = 0; e < n; ++e) s[e] += f[e];
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int e = 0; e < n; ++e) lds[wave][e * 64 + lane] = s[e];
  __syncthreads();
  for (int k = threadIdx.x; k < 64 * n; k += 256) {
    const int at = ((int)blockIdx.x * 64 + k / n) * n + k % n, l = k % n * 64 + k / n;
    if (at < a.N) a.part[(int64_t)blockIdx.y * a.N + at] = lds[0][l] + lds[1][l] + lds[2][l] + lds[3][l];
  }
}

constexpr int kActBlocks = 2048;   // workgroups, about

// Parts of the rows: the columns' workgroups follow from the type, of which the workspace knows nothing, so there are
// as many as 16-bit rows need.
int act_grad_parts(int64_t R, int64_t N) {
  const int64_t columns = (N + 511) / 512;
  return (int)std::min<int64_t>((R + 3) / 4, std::max<int64_t>(kActBlocks / columns, 1));
}

// How a product is computed, from its sizes alone: M rows and N columns of results, a contraction of C.
struct LinearPlan {
  vp_linear_kind kind;
  int parts;
  int64_t chunk;   // of the contraction: a part's values
};

// The least of an estimate in us.  Few rows: a chunk of 256 values takes 1.06 with up to 16 rows, 1.25 with 32, 1.7
// with 64 (1.6 times that where two workgroups share a CU), or its weights' time at 5.2 TB/s for all of them (once for
// every 64 rows); 3 around them, and for parts 6 for the second launch (on the device 4, but a call of two launches takes the host 3
// longer) and the sums' way out and back at 3 TB/s.  Measured in 1, 2, 4, 8 parts, weights from memory: 1 row by 4096
// x 4096 20, 15, 12.5, 12.0; 61 rows 31, 22, 16.8, 18.0; 128 rows 31, 22.0, 22.8 (tiles in 8 parts 21.2); 1 by 16384 x
// 4096 30, 34; 96 rows by 256 x 7168 in 4, 7, 14, 28 parts 18, 14, 11.9, 11.9; 1 by 512 x 512 4.8, 6.3, by 512 x 1536
// 8.7, 8.3, by 2048 x 2048 11.4, 10.0, 8.3, 7.6.
//
// Tiles read the weights once for 128 rows, so from 33 rows on the two are compared, in parts of 16 steps or more (of
// fewer the estimate of tiles says too little), neither faster than its weights come: at 4.2 TB/s through few rows, 4.4
// through tiles alone, 5.2 through the others.  Measured, weights from memory, us (few rows / tiles): 33 rows by 28672 x
// 4096 65 / 64; 64 rows 70 / 66, by 57344 x 4096 127 / 109, by 131072 x 4096 257 / 196; 65 rows by 4096 x 4096 22 / 21,
// by 14336 x 4096 52 / 36, by 28672 x 4096 105 / 60, by 131072 x 4096 466 / 192; of 414 sizes that go through tiles
// for this, or by other parts, the worst is 64 by 32768 x 8192, 132 / 139.  With up to 32 rows tiles take 0.8 to 1.7 times as long.
//
// Tiles: a step of 64 values takes 0.72 for a 128 x 128 tile alone on its CU, 1.1 for two, 1.65 for a 256 x 256 tile;
// a round of tiles ends with 3 or 9 for its results; parts as above.  Measured, us (128 / 256 tiles, parts in
// brackets): 16381 rows by 4096 x 4096 546 / 417; 2048 rows 71 / 96; 512 rows 46 [1], 36.0 [2], 36.7 [4] / 93 [1], 48
// [4]; 256 rows 32 [2], 25.5 [4], 29 [8]; 16384 by 256 x 4096 58-62 [1], 67 [2] / 99 [1], 67 [4], its weights'
// gradient 60 [4], 66 [8], 74 [16] / 342 [1], 63 [16], its rows' gradient 59 / 70; rows' gradient of 96 rows by 4096 x
// 4096 45 [1], 21.6 [4], 19.6 [8], 22.5 [16].
LinearPlan plan_of(int mode, int64_t R, int32_t N_, int32_t K) {
  const int64_t M = mode == kExpertGradW ? N_ : R, N = mode == kExpertForward ? N_ : K;
  const int64_t C = mode == kExpertForward ? K : mode == kExpertGradX ? N_ : R;
  const auto ceil_of = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const auto in_parts = [&](vp_linear_kind kind, int64_t parts) {
    LinearPlan p{kind, 1, std::max<int64_t>(C, 1)};
    if (parts > 1) {
      const int64_t unit = kind == VP_LINEAR_FEW_ROWS ? kFewChunk : 64;
      p.chunk = ceil_of(ceil_of(C, parts), unit) * unit;
      p.parts = (int)ceil_of(C, p.chunk);
    }
    return p;
  };
  const auto join = [&](const LinearPlan& p) {
    return p.parts > 1 ? 6.0 + (double)p.parts * (double)M * (double)N * 8.0 / 3e6 : 0.0;
  };
  LinearPlan best{VP_LINEAR_FEW_ROWS, 1, std::max<int64_t>(C, 1)};
  double least = 0.0;
  const auto take = [&](const LinearPlan& p, double time) {
    if (least == 0.0 || time < least) {
      least = time;
      best = p;
    }
  };
  const bool few = mode == kExpertForward && M <= 2 * kFewRows;
  const double weights = few ? 2.0 * (double)N * (double)K : 0.0;   // bytes that bound a product of few rows
  if (few) {
    const int64_t tiles = ceil_of(M, kFewRows) * ceil_of(N, kFewCols), most = C / kFewChunk;
    const double chunk = M <= 16 ? 1.06 : M <= 32 ? 1.25 : 1.7;
    const int64_t one_each = kCus / std::max<int64_t>(tiles, 1);
    for (const int64_t parts : std::initializer_list<int64_t>{1, 2, 4, 8, 16, 32, one_each, most}) {
      if (parts > std::max<int64_t>(most, 1) || parts > 64) continue;
      const LinearPlan p = in_parts(VP_LINEAR_FEW_ROWS, parts);
      const double bytes = (double)(tiles * p.parts) * (kFewCols * kFewChunk * 2);
      const double crowd = std::max(1.0, 0.8 * (double)(tiles * p.parts) / kCus);
      take(p, 3.0 + (double)ceil_of(p.chunk, kFewChunk) * std::max(chunk * crowd, bytes / 5.2e6) + join(p));
    }
    if (M <= 32) return best;
    least = std::max(least, 3.0 + weights * (double)ceil_of(M, kFewRows) / 4.2e6);   // tiles follow
  }
  for (const bool large : {true, false}) {
    const int64_t side = large ? 256 : 128, tiles = ceil_of(M, side) * ceil_of(N, side);
    for (int64_t parts = 1; parts == 1 || (parts <= 64 && C >= 128 * parts); parts *= 2) {
      LinearPlan p = in_parts(VP_LINEAR_TILES_256, parts);
      const double steps = (double)ceil_of(p.chunk, 64), groups = (double)(tiles * p.parts);
      if (!large) p.kind = groups <= kCus ? VP_LINEAR_TILES_ALONE : VP_LINEAR_TILES_128;
      const double rounds = std::max(1.0, std::ceil(groups / (large ? kCus : 2 * kCus)));
      const double step = large ? 1.65 : p.kind == VP_LINEAR_TILES_ALONE ? 0.72 : 1.1;
      const double stream = 3.0 + weights / (p.kind == VP_LINEAR_TILES_ALONE ? 4.4e6 : 5.2e6);
      if (few && steps < 16) break;
      take(p, std::max(rounds * (step * steps + (large ? 9.0 : 3.0)), stream) + join(p));
    }
  }
  return best;
}

template <typename T, int MODE, int WM, int WN, int MT, int NT, int STAGES = 2>
vp_status launch_dense_tiled(const DenseArgs& a, hipStream_t s) {
  constexpr int BM = WM * MT * 16, BN = WN * NT * 16;
  const int64_t mt = ((MODE == kGradW ? a.M : a.R) + BM - 1) / BM, nt = (a.N + BN - 1) / BN;
  const int64_t tiles = mt * nt * a.parts;
  if (tiles >= (int64_t)1 << 31) return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 tiles");
  const int64_t per = std::min<int64_t>((tiles + 7) / 8, kCus / 8 * (BM == 128 && STAGES == 2 ? 2 : 1));
  const auto kernel = product_tiled<T, MODE, false, WM, WN, MT, NT, DenseArgs, STAGES>;
  const int lds = STAGES == 2 ? 0 : STAGES * (BM + BN) * kStep;
  if (lds && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return set_error(VP_ERR_HIP, "dense product launch failed");
  hipLaunchKernelGGL(kernel, dim3((unsigned)(per * 8)), dim3(WM * WN * 64), lds, s, a);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "dense product launch failed");
  return VP_OK;
}

template <typename T, int MODE> vp_status launch_as(DenseArgs a, const LinearPlan& p, float* ws, hipStream_t s) {
  const DenseArgs whole = a;
  const int64_t M = MODE == kGradW ? a.M : a.R;
  a.parts = p.parts;
  a.chunk = (int32_t)p.chunk;
  if (p.parts > 1) {   // raw sums to the workspace
    a.raw = a.wide = true;
    a.out = (unsigned char*)ws;
    a.out_stride = (int64_t)a.N * 4;
    a.part_bytes = M * a.out_stride;
    a.pre = nullptr;
  }
  vp_status st = VP_OK;
  if (p.kind == VP_LINEAR_FEW_ROWS) {
    if constexpr (MODE == kForward) {
      const dim3 grid((unsigned)((a.N + kFewCols - 1) / kFewCols), (unsigned)p.parts, (unsigned)((M + kFewRows - 1) / kFewRows));
      if (M <= 16) hipLaunchKernelGGL((linear_few<T, 1>), grid, dim3(256), 0, s, a);
      else if (M <= 32) hipLaunchKernelGGL((linear_few<T, 2>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((linear_few<T, 4>), grid, dim3(256), 0, s, a);
      if (hipGetLastError() != hipSuccess) st = set_error(VP_ERR_HIP, "dense product launch failed");
    }
  } else {
    st = p.kind == VP_LINEAR_TILES_256     ? launch_dense_tiled<T, MODE, 2, 4, 8, 4>(a, s)
         : p.kind == VP_LINEAR_TILES_ALONE ? launch_dense_tiled<T, MODE, 2, 4, 4, 2, 4>(a, s)
                                           : launch_dense_tiled<T, MODE, 2, 2, 4, 4>(a, s);
  }
  if (st != VP_OK || p.parts == 1) return st;
  hipLaunchKernelGGL(linear_join<T>, grid_of((M * (a.N / 4) + 255) / 256), dim3(256), 0, s, whole, (const float*)ws, p.parts, M);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "dense product launch failed");
  return VP_OK;
}

}  // namespace

vp_linear_kind linear_kind(int mode, int64_t R, int32_t N, int32_t K, int32_t* parts) {
  const LinearPlan p = plan_of(mode, R, N, K);
  if (parts) *parts = p.parts;
  return p.kind;
}

size_t linear_workspace(int mode, int64_t R, int32_t N, int32_t K) {
  const LinearPlan p = plan_of(mode, R, N, K);
  const int64_t results = mode == kExpertForward ? R * N : mode == kExpertGradX ? R * K : (int64_t)N * K;
  return p.parts > 1 ? (size_t)(p.parts * results * 4) : 0;
}

vp_status launch_linear(const LinearLaunch& p, void* stream) {
  DenseArgs a{};
  a.a = (const unsigned char*)p.a;
  a.b = (const unsigned char*)p.b;
  a.a_stride = p.a_stride;
  a.b_stride = p.b_stride;
  a.R = p.R;
  a.M = p.N;
  a.N = p.mode == kExpertForward ? p.N : p.K;
  a.C = p.mode == kExpertForward ? p.K : p.N;   // (grad w's is R)
  a.bias = p.bias;
  a.bias_wide = p.bias_dtype == VP_F32;
  a.act = p.act;
  a.residual = (const unsigned char*)p.residual;
  a.residual_stride = p.residual_stride;
  a.slope = (const unsigned char*)p.slope;
  a.slope_stride = p.slope_stride;
  a.out = (unsigned char*)p.out;
  a.out_stride = p.out_stride;
  a.wide = p.out_dtype == VP_F32;
  a.pre = (unsigned char*)p.pre;
  a.pre_stride = p.pre_stride;
  const LinearPlan plan = plan_of(p.mode, p.R, p.N, p.K);
  const hipStream_t s = (hipStream_t)stream;
  const auto run = [&](auto t) {
    using T = decltype(t);
    if (p.mode == kExpertForward) return launch_as<T, kForward>(a, plan, (float*)p.ws, s);
    if (p.mode == kExpertGradX) return launch_as<T, kGradX>(a, plan, (float*)p.ws, s);
    return launch_as<T, kGradW>(a, plan, (float*)p.ws, s);
  };
  return p.dtype == VP_BF16 ? run(Bf16{}) : run(F16{});
}

size_t act_grad_workspace(int64_t R, int64_t N) { return (size_t)act_grad_parts(R, N) * N * 4; }

vp_status launch_act_grad(const void* d_y, int64_t d_y_stride, const void* pre, int64_t pre_stride, int32_t dtype,
                          int64_t R, int64_t N, int32_t act, void* d_pre, int64_t d_pre_stride, float* d_bias,
                          void* ws, void* stream) {
  const ActGradArgs a{(const unsigned char*)d_y, (const unsigned char*)pre, d_y_stride, pre_stride, d_pre_stride, R, (int32_t)N,
                      (unsigned char*)d_pre, d_bias ? (float*)ws : nullptr, act_grad_parts(R, N)};
  if (R > 0) {
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      const dim3 grid((unsigned)((N + 64 * Vec<T>::n - 1) / (64 * Vec<T>::n)), a.parts);
      with_act(act, [&](auto f) {
        hipLaunchKernelGGL((act_grad_kernel<T, decltype(f)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
      });
    });
    if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "activation gradient launch failed");
  }
  return d_bias ? launch_column_sums(a.part, a.parts, N, N, d_bias, nullptr, stream) : VP_OK;
}

}  // namespace vp
