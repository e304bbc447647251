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
// A workgroup makes one tile of BM rows by BN columns of one expert.  Tiles
// are numbered without a count of any expert's: expert e owns the slots from
// floor(offsets[e] / BM) + e on, at least as many as its rows need, and a
// slot past its rows is empty.  So the grid follows from the buffer's size,
// and a tile finds its expert by counting the experts whose first slot is at
// or below its own.
//
// Each step of the contraction brings 128 bytes of every row of both operands
// to LDS (64 16-bit values, or 256 4-bit ones) by direct loads, double
// buffered.  Both operands are read through buffer descriptors that end with
// the expert's last row: what lies outside reads as zero, so no neighbour's
// row (which may hold anything) enters a sum.  The places in LDS are permuted
// so that the matrix fragments' reads meet no bank twice:
//   rows by contraction   16-byte chunk c of row r at place c ^ (r & 7); a
//                         fragment lane reads its row's chunk whole
//   contraction by rows   (grad x's weights, both operands of grad w) 32-byte
//                         piece p of contraction row c at place p ^ f(c), read
//                         through the transposing LDS load
// The product is computed as its transpose, so that a lane's four results are
// neighbours in the output row.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
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

// ---------------------------------------------------------------- tiled products

constexpr int kStep = 128;   // bytes of a row that one step of the contraction takes

// Starts a direct load of 16 bytes per lane from `off` of `bytes` bytes at
// `base` to 1 KB of LDS at `lds` (both the same for the whole wavefront).  It
// returns nothing in registers, and the loops below wait for it themselves:
// through the builtin the compiler puts a wait for all loads before every
// transposing LDS read.
__device__ inline void direct_load(const unsigned char* base, int bytes, uint32_t off, unsigned char* lds) {
#ifdef __HIP_DEVICE_COMPILE__
  const uint64_t b = (uint64_t)base;
  const i32x4 rsrc = {(int)(uint32_t)b, (int)((b >> 32) & 0xffff), bytes, 0x00020000};
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(at), "v"(off), "s"(rsrc) : "memory", "m0");
#endif
}

// Address of the permuted place of 32-byte piece p of contraction row c.
__device__ inline int piece_place(int p, int c) { return p ^ ((c & 3) | ((c >> 3) & 1) << 2); }

// One operand of a tile: ROWS rows (columns of the output, or its rows) in LDS.
// COLS: the buffer's rows are the contraction, ROWS neighbouring elements of
// each; otherwise a buffer row is an operand row, 128 bytes of it per step.
template <int ROWS, bool COLS, int WAVES> struct Operand {
  static constexpr int kLoads = ROWS * kStep / 1024 / WAVES;   // direct loads of 64 x 16 bytes by each wavefront
  static constexpr int kSlots = ROWS / 8;                      // COLS: 16-byte slots of a contraction row
  const unsigned char* base;   // of the current step
  int stride;                  // bytes, at most 4 MiB
  int left;                    // rows by contraction: bytes to the end of the last valid row; COLS: rows left
  int width;                   // rows by contraction: bytes of a row left; COLS: bytes of a row from the tile's first column
  int bytes;                   // what the step may read from its base on
  uint32_t past;               // rows by contraction: added where the lane's chunk lies past the row's end
  uint32_t off[kLoads];

  // For rows by contraction `row_of(i)` gives the buffer row of operand row i, relative to `base`.
  template <typename F> __device__ void init(int wave, int lane, F row_of) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      if (COLS) {
        const int c = (wave * kLoads + j) * (64 / kSlots) + lane / kSlots, slot = lane % kSlots;
        off[j] = (uint32_t)(c * stride) + piece_place(slot / 2, c) * 32 + (slot & 1) * 16;
      } else {
        const int i = (wave * kLoads + j) * 8 + lane / 8;
        off[j] = (uint32_t)(row_of(i) * stride) + ((lane & 7) ^ (i & 7)) * 16;
      }
    }
    bounds(lane);
  }
  __device__ void bounds(int lane) {
    bytes = max(COLS ? (min(left, 64) - 1) * stride + width : left, 0);
    // chunks past a row's end read outside the buffer, as zero
    past = !COLS && ((lane & 7) ^ (lane >> 3)) * 16 >= width ? 0x60000000u : 0u;
  }
  // Starts the j-th of the step's loads.
  __device__ void issue(unsigned char* lds, int wave, int j) const {
    direct_load(base, bytes, off[j] + past, lds + (wave * kLoads + j) * 1024);
  }
  __device__ void next(int lane) {
    if (COLS) {
      base += 64 * stride;
      left -= 64;
    } else {
      base += kStep;
      left -= kStep;
      width -= kStep;
    }
    bounds(lane);
  }
};

template <typename T> struct Mx { using out = T; };   // both operands in 4-bit blocks, results of type T
template <typename T> struct Elem { using out = T; static constexpr bool mx = false; };
template <typename T> struct Elem<Mx<T>> { using out = T; static constexpr bool mx = true; };

// WM x WN wavefronts, each with MT x NT fragments of 16 x 16 results.
template <typename T, int MODE, bool GATED, int WM, int WN, int MT, int NT>
__global__ void __launch_bounds__(WM * WN * 64) product_tiled(ProductArgs a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host's pass knows none of the builtins below
  using Out = typename Elem<T>::out;
  constexpr bool kMx = Elem<T>::mx, kColsA = MODE == kGradW, kColsB = MODE != kForward;
  constexpr int BM = WM * MT * 16, BN = WN * NT * 16, kWaves = WM * WN;
  constexpr int kTileN = GATED ? BN / 2 : BN;   // output columns
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2][(BM + BN) * kStep];
  // 4-bit blocks: the powers of two of four steps, 32 bytes a row, double buffered
  __shared__ __attribute__((aligned(1024))) unsigned char powers[kMx ? 2 : 1][kMx ? (BM + BN) * 32 : 16];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, q = lane / 16;
  if (blockIdx.x == 0) check_offsets(a);

  // which tile: XCD x (block % 8) takes a contiguous eighth of the tiles (of
  // every expert's, for grad w), in blocks of eight row tiles by all columns
  const int nt = (a.N + kTileN - 1) / kTileN;
  const int xcd = blockIdx.x & 7;
  const int64_t idx = blockIdx.x >> 3;
  constexpr int kBand = 8;
  Group g;
  int64_t m0, slot;
  int ni;
  if (MODE == kGradW) {
    const int mt = (a.M + BM - 1) / BM;
    const int64_t per = ((int64_t)mt * nt + 7) / 8;
    const int64_t e = idx / per, t = xcd * per + idx % per;
    if (e >= a.L || t >= (int64_t)mt * nt) return;
    const int band = (int)(t / (kBand * nt)), in = (int)(t % (kBand * nt));
    const int high = min(kBand, mt - band * kBand);
    slot = band * kBand + in % high;
    ni = in / high;
    g = group_of(a, (int)e);
    m0 = slot * BM;
  } else {
    int64_t rows = a.offsets[a.L];
    rows = rows < 0 ? 0 : rows > a.R ? a.R : rows;
    const int64_t slots = rows / BM + a.L, total = slots * nt, per = (total + 7) / 8, t = xcd * per + idx;
    if (idx >= per || t >= total) return;
    const int64_t band = t / (kBand * nt);
    const int in = (int)(t % (kBand * nt));
    const int high = (int)min((int64_t)kBand, slots - band * kBand);
    slot = band * kBand + in % high;
    ni = in / high;
    const int e = expert_of_slot<BM>(a, slot);
    if (e < 0) return;
    g = group_of(a, e);
    m0 = g.lo + (slot - (a.offsets[e] / BM + e)) * BM;
    if (m0 < g.lo || m0 >= g.hi) return;
  }
  const int n0 = ni * kTileN;

  // operands and the steps of the contraction
  const int64_t rows = g.hi - g.lo;
  const int64_t C = MODE == kGradW ? rows : a.C;               // elements
  const int row_bytes = kMx ? a.C / 2 : a.C * 2;
  const int64_t steps = MODE == kGradW || MODE == kGradX ? (C + 63) / 64 : (row_bytes + kStep - 1) / kStep;
  Operand<BM, kColsA, kWaves> oa;
  Operand<BN, kColsB, kWaves> ob;
  oa.stride = (int)a.a_stride;
  ob.stride = (int)a.b_stride;
  if (kColsA) {
    oa.base = a.a + g.lo * a.a_stride + m0 * 2;
    oa.left = (int)rows;
    oa.width = (int)((a.M - m0) * 2);
  } else {
    oa.base = a.a + m0 * a.a_stride;
    const int64_t valid = min((int64_t)BM, g.hi - m0);
    oa.left = (int)((valid - 1) * a.a_stride) + row_bytes;
    oa.width = row_bytes;
  }
  oa.init(wave, lane, [](int i) { return i; });
  if (MODE == kGradW) {
    ob.base = a.b + g.lo * a.b_stride + n0 * 2;
    ob.left = (int)rows;
    ob.width = (a.N - n0) * 2;
  } else if (MODE == kGradX) {
    ob.base = a.b + g.e * a.b_expert + n0 * 2;
    ob.left = a.C;
    ob.width = (a.N - n0) * 2;
  } else {
    // gated: of every 64 operand rows the first 32 are gate rows, the others the same up rows
    ob.base = a.b + g.e * a.b_expert + (int64_t)n0 * a.b_stride;
    const int64_t end = ((int64_t)(GATED ? a.half + a.N : a.N) - n0 - 1) * a.b_stride + row_bytes;
    ob.left = (int)min(end, (int64_t)(GATED ? a.half + kTileN : BN) * a.b_stride);
    ob.width = row_bytes;
  }
  const int half = a.half;
  ob.init(wave, lane, [=](int i) { return GATED ? i / 64 * 32 + i % 32 + (i & 32 ? half : 0) : i; });

  // places of this lane's fragments in LDS
  const int wm = wave / WN, wn = wave % WN;
  const auto chunk = [=](int kk) { return kMx ? 2 * q + kk : 4 * kk + q; };
  uint32_t pa[kColsA ? MT : 1], pb[kColsB ? NT : 1];
  if (kColsA) {
#pragma unroll
    for (int i = 0; i < MT; ++i) pa[i] = (q * 8 + r / 4) * (BM * 2) + piece_place(wm * MT + i, q * 8 + r / 4) * 32 + (r & 3) * 8;
  } else {
    pa[0] = (wm * MT * 16 + r) * kStep;
  }
  if (kColsB) {
#pragma unroll
    for (int i = 0; i < NT; ++i) pb[i] = (q * 8 + r / 4) * (BN * 2) + piece_place(wn * NT + i, q * 8 + r / 4) * 32 + (r & 3) * 8;
  } else {
    pb[0] = (wn * NT * 16 + r) * kStep;
  }
  const auto frag = [&](const unsigned char* p, auto cols, auto width, uint32_t place, int i, int kk) -> i32x4 {
    if constexpr (decltype(cols)::value) {
      constexpr int kRow = decltype(width)::value * 2;
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const unsigned char* at = p + place + kk * 32 * kRow;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * kRow));
      const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
      return i32x4{(int)l.x, (int)l.y, (int)h.x, (int)h.y};
    } else {
      return *(const i32x4*)(p + place + i * 16 * kStep + (chunk(kk) ^ (r & 7)) * 16);
    }
  };

  // 4-bit blocks: a load covers 32 rows' powers of four steps, first their
  // first 16 bytes (two steps), then the others; a lane's two blocks of a step
  // are neighbouring bytes
  constexpr int kPowerLoads = kMx ? (BM + BN) / 32 / kWaves : 1;
  static_assert(!kMx || (BM + BN) / 32 % kWaves == 0, "whole loads");
  uint32_t power_off[kPowerLoads] = {};
  if constexpr (kMx) {
#pragma unroll
    for (int j = 0; j < kPowerLoads; ++j) {
      const int i = (wave * kPowerLoads + j) * 32 + lane % 32;
      const int64_t row = i < BM ? i : GATED ? (i - BM) / 64 * 32 + (i - BM) % 32 + ((i - BM) & 32 ? half : 0) : i - BM;
      power_off[j] = (uint32_t)(row * (i < BM ? a.a_stride : a.b_stride)) + row_bytes + lane / 32 * 16;
    }
  }
  const unsigned char *power_a = oa.base, *power_b = ob.base;
  const int power_end_a = oa.left - row_bytes, power_end_b = ob.left - row_bytes;   // the last row's first byte
  const auto load_powers = [&](int64_t s) {   // of steps s .. s + 3
    if constexpr (kMx) {
      const int whole = (row_bytes + a.C / 32 + 15) / 16 * 16;   // bytes of a packed row
#pragma unroll
      for (int j = 0; j < kPowerLoads; ++j) {
        const int i0 = (wave * kPowerLoads + j) * 32;
        const bool is_a = i0 < BM;
        direct_load(is_a ? power_a : power_b, (is_a ? power_end_a : power_end_b) + whole, power_off[j] + (uint32_t)(s * 8),
                    powers[(s / 4) & 1] + i0 * 32);
      }
    }
  };
  // The two powers of fragment row `row` + r in step s; blocks past the row's
  // last count as 2^-127 (their codes are zero).
  const auto read_power = [&](int64_t s, int row) -> int {
    if constexpr (kMx) {
      const int left = a.C / 32 - (int)s * 8 - 2 * q;
      const int mask = left >= 2 ? 0xffff : left == 1 ? 0xff : 0;
      const unsigned char* at = powers[(s / 4) & 1] + ((s & 2) << 8) + (s & 1) * 8 + 2 * q + r * 16;
      return *(const uint16_t*)(at + row / 32 * 1024 + row % 32 * 16) & mask;
    }
    return 0;
  };
  const auto read_a = [&](int64_t s, int kk, int i) {
    return frag(lds[s & 1], std::bool_constant<kColsA>{}, std::integral_constant<int, BM>{}, pa[kColsA ? i : 0], i, kk);
  };
  const auto read_b = [&](int64_t s, int kk, int i) {
    return frag(lds[s & 1] + BM * kStep, std::bool_constant<kColsB>{}, std::integral_constant<int, BN>{}, pb[kColsB ? i : 0], i, kk);
  };
  static_assert(NT <= MT && decltype(oa)::kLoads + decltype(ob)::kLoads == MT, "one load and at most one fragment of each operand per row of products");
  constexpr int kLoadsA = decltype(oa)::kLoads, kLoads = MT;
  const auto issue = [&](int64_t s, int j) {
    if (j < kLoadsA) oa.issue(lds[s & 1], wave, j);
    else ob.issue(lds[s & 1] + BM * kStep, wave, j - kLoadsA);
  };
  const auto load = [&](int64_t s) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) issue(s, j);
    oa.next(lane);
    ob.next(lane);
  };

  f32x4 acc[MT][NT] = {};
  // One row of fragments: i of the rows' by all of the columns'.
  const auto multiply = [&](auto half_step, int i, const i32x4& fa, const i32x4 (&fb)[NT], int sa, const int (&sb)[NT]) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if constexpr (kMx) {
        constexpr int kk = decltype(half_step)::value;
        const i32x8 wa = {fa[0], fa[1], fa[2], fa[3], 0, 0, 0, 0};
        const i32x8 wb = {fb[j][0], fb[j][1], fb[j][2], fb[j][3], 0, 0, 0, 0};
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, acc[i][j], 4, 4, kk, sb[j], kk, sa);
      } else {
        using F = typename Frag<T>::type;
        acc[i][j] = mma(__builtin_bit_cast(F, fb[j]), __builtin_bit_cast(F, fa), acc[i][j]);
      }
    }
  };

  // A step is two halves of 32 16-bit (128 4-bit) values.  While one half is
  // multiplied the next one's fragments are read; in the middle of a step its
  // LDS half has been read by all and takes the loads of the step after next.
  // Steps past the last load zeros that nothing multiplies.
  i32x4 fa0[MT], fb0[NT], fa1[MT], fb1[NT];
  int sa[MT] = {}, sb[NT] = {};
  if (steps > 0) {
    load_powers(0);
    load(0);
    load(1);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < MT; ++i) fa0[i] = read_a(0, 0, i);
#pragma unroll
    for (int i = 0; i < NT; ++i) fb0[i] = read_b(0, 0, i);
#pragma unroll
    for (int i = 0; i < MT; ++i) sa[kMx ? i : 0] = read_power(0, (wm * MT + i) * 16);
#pragma unroll
    for (int i = 0; i < NT; ++i) sb[kMx ? i : 0] = read_power(0, BM + (wn * NT + i) * 16);
  }
  for (int64_t s = 0; s < steps; ++s) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      fa1[i] = read_a(s, 1, i);
      if (i < NT) fb1[i] = read_b(s, 1, i);
      __builtin_amdgcn_sched_barrier(0);
      multiply(std::integral_constant<int, 0>{}, i, fa0[i], fb0, sa[kMx ? i : 0], sb);
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (kMx && ((s + 2) & 3) == 0) load_powers(s + 2);
    // one load between rows of products: issued together they would hold up
    // every wavefront's matrix instructions behind the CU's one load path
    int sb1[NT] = {};
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      issue(s + 2, i);
      fa0[i] = read_a(s + 1, 0, i);
      if (i < NT) {
        fb0[i] = read_b(s + 1, 0, i);
        if (kMx) sb1[i] = read_power(s + 1, BM + (wn * NT + i) * 16);
      }
      __builtin_amdgcn_sched_barrier(0);
      multiply(std::integral_constant<int, 1>{}, i, fa1[i], fb1, sa[kMx ? i : 0], sb);
      __builtin_amdgcn_sched_barrier(0);
      if (kMx) sa[i] = read_power(s + 1, (wm * MT + i) * 16);
    }
    oa.next(lane);
    ob.next(lane);
    if constexpr (kMx) {
#pragma unroll
      for (int i = 0; i < NT; ++i) sb[i] = sb1[i];
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the last loads end before the LDS is another workgroup's

  const auto put = [&](unsigned char* at, f32x4 v) {
    u32x2 o;
    o.x = from_f32<Out>(v[0]).u | (uint32_t)from_f32<Out>(v[1]).u << 16;
    o.y = from_f32<Out>(v[2]).u | (uint32_t)from_f32<Out>(v[3]).u << 16;
    *(u32x2*)at = o;
  };
  const int64_t end = MODE == kGradW ? a.M : g.hi;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + (wm * MT + i) * 16 + r;
    if (m >= end) continue;
    unsigned char* out = a.out + (MODE == kGradW ? g.e * a.b_expert : 0) + m * a.out_stride;
    if constexpr (GATED) {
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) {
        const int n = n0 + wn * NT * 8 + j * 16 + q * 4;
        if (n >= a.N) continue;
        const f32x4 gate = acc[i][j / 2 * 4 + j % 2], up = acc[i][j / 2 * 4 + j % 2 + 2];
        f32x4 h;
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = silu(gate[v]) * up[v];
        put(out + n * 2, h);
        if (a.pre) {
          put(a.pre + m * a.pre_stride + n * 2, gate);
          put(a.pre + m * a.pre_stride + (int64_t)(n + a.half) * 2, up);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int n = n0 + (wn * NT + j) * 16 + q * 4;
        if (n >= a.N) continue;
        if constexpr (MODE == kGradW) *(f32x4*)(out + (int64_t)n * 4) = acc[i][j];
        else put(out + (int64_t)n * 2, acc[i][j]);
      }
    }
  }
#endif
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

namespace {

// Grids cover the buffer's tiles for any offsets, rounded up to the eight XCDs.
template <typename T, int MODE, bool GATED, int WM, int WN, int MT, int NT>
vp_status launch_tiled(const ProductArgs& a, hipStream_t s) {
  constexpr int BM = WM * MT * 16, kTileN = WN * NT * 16 / (GATED ? 2 : 1);
  const int64_t nt = (a.N + kTileN - 1) / kTileN;
  const int64_t per = MODE == kGradW ? (((a.M + BM - 1) / BM) * nt + 7) / 8 * a.L : ((a.R / BM + a.L) * nt + 7) / 8;
  if (per * 8 >= (int64_t)1 << 31) return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 tiles");
  hipLaunchKernelGGL((product_tiled<T, MODE, GATED, WM, WN, MT, NT>), dim3((unsigned)(per * 8)), dim3(WM * WN * 64), 0, s, a);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "expert product launch failed");
  return VP_OK;
}

template <typename T, int MODE, bool GATED> vp_status launch_product_as(const ProductArgs& a, hipStream_t s) {
  return launch_tiled<T, MODE, GATED, 2, 4, 8, 4>(a, s);
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
  const bool bf = p.dtype == VP_BF16;
  if (p.mode == kExpertForward) {
    a.C = p.K;
    a.N = p.gated ? p.N / 2 : p.N;
    a.half = p.N / 2;
    a.b_expert = p.N * p.b_stride;
    if (p.mx) {
      if (bf && p.gated) return launch_product_as<Mx<Bf16>, kForward, true>(a, s);
      if (bf) return launch_product_as<Mx<Bf16>, kForward, false>(a, s);
      if (p.gated) return launch_product_as<Mx<F16>, kForward, true>(a, s);
      return launch_product_as<Mx<F16>, kForward, false>(a, s);
    } else {
      if (bf && p.gated) return launch_product_as<Bf16, kForward, true>(a, s);
      if (bf) return launch_product_as<Bf16, kForward, false>(a, s);
      if (p.gated) return launch_product_as<F16, kForward, true>(a, s);
      return launch_product_as<F16, kForward, false>(a, s);
    }
  } else if (p.mode == kExpertGradX) {
    a.C = p.N;
    a.N = p.K;
    a.b_expert = p.N * p.b_stride;
    if (bf) return launch_product_as<Bf16, kGradX, false>(a, s);
    return launch_product_as<F16, kGradX, false>(a, s);
  } else {
    a.M = p.N;
    a.N = p.K;
    a.b_expert = (int64_t)p.N * p.out_stride;
    if (bf) return launch_product_as<Bf16, kGradW, false>(a, s);
    return launch_product_as<F16, kGradW, false>(a, s);
  }
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
