// The tiled product on the matrix units, which the experts' products and the
// dense ones share.
//
// Each step of the contraction brings 128 bytes of every row of both operands
// to LDS (64 16-bit values, or 256 4-bit ones) by direct loads, two or four
// steps ahead.  Both operands are read through buffer descriptors that end with
// the operand's last row: what lies outside reads as zero, so no neighbour's
// row (which may hold anything) enters a sum.  The places in LDS are permuted
// so that the matrix fragments' reads meet no bank twice (in 4-bit blocks, whose
// lanes take neighbouring chunks, some do):
//   rows by contraction   16-byte chunk c of row r at place c ^ (r & 7); a
//                         fragment lane reads its row's chunk whole
//   contraction by rows   (grad x's weights, both operands of grad w) 32-byte
//                         piece p of contraction row c at place p ^ f(c), read
//                         through the transposing LDS load
// The product is computed as its transpose, so that a lane's four results are
// neighbours in the output row.  (The experts' products report offsets out of
// order: their source includes report.h before this.)
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "act.h"
#include "internal.h"
#include "numeric.h"

namespace vp {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

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

// A dense product: one group of rows, the contraction in `parts` of `chunk`
// values.  Of several parts each writes its sums, raw and in 32 bits,
// part_bytes after the last one's; else the epilogue follows (see finish).
struct DenseArgs : ProductArgs {
  int32_t parts, chunk;
  int64_t part_bytes;
  const void* bias;
  const unsigned char *residual, *slope;   // slope: what act's derivative is taken at (grad x)
  int64_t residual_stride, slope_stride;
  int32_t act;
  bool bias_wide, wide, raw;               // 32-bit bias; 32-bit results (and residual); no epilogue
};

// Four neighbouring values of a dense product's bias, from column n on.
template <typename T> __device__ inline f32x4 bias4(const DenseArgs& a, int n) {
  if (a.bias_wide) return *(const f32x4*)((const float*)a.bias + n);
  const u32x2 v = *(const u32x2*)((const T*)a.bias + n);
  return {to_f32(T{(uint16_t)(v.x & 0xffffu)}), to_f32(T{(uint16_t)(v.x >> 16)}), to_f32(T{(uint16_t)(v.y & 0xffffu)}),
          to_f32(T{(uint16_t)(v.y >> 16)})};
}

// The offsets do not change while a kernel runs: they are read by scalar loads,
// which a wavefront need not wait for behind its loads to LDS.
__device__ inline int64_t offset_at(const ProductArgs& a, int e) {
  return ((const __attribute__((address_space(4))) int64_t*)a.offsets)[e];
}

struct Group { int e; int64_t lo, hi; };   // an expert and its rows

__device__ inline Group group_of(const ProductArgs& a, int e) { return {e, offset_at(a, e), offset_at(a, e + 1)}; }

// Offsets that decrease or leave the buffer are the caller's error.
template <typename Args> __device__ inline bool in_order(const Args& a, int e) {
  const int64_t lo = a.offsets[e], hi = a.offsets[e + 1];
  return lo >= 0 && lo <= hi && hi <= a.R;
}

// Row tiles of BM rows, expert after expert.  Lane l of every wavefront holds
// the first tile of its run of experts (one each up to 64 experts).
template <int BM> struct RowTiles {
  int run;         // experts of a lane
  int64_t first;   // this lane's first tile
  int64_t total;

  __device__ static int64_t of(const Group& g) { return (g.hi - g.lo + BM - 1) / BM; }
  // False, and no tiles, for offsets out of order: every wavefront finds the same.
  __device__ bool init(const ProductArgs& a, int lane) {
    run = (a.L + 63) / 64;
    int64_t sum = 0;
    bool good = true;
    for (int e = lane * run; e < min((lane + 1) * run, a.L); ++e) {
      if (in_order(a, e)) sum += of(Group{e, a.offsets[e], a.offsets[e + 1]});
      else good = false;
    }
    if (!__all(good)) {
      first = total = 0;
      return false;
    }
    int64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t v = __shfl_up(incl, d);
      incl += lane >= d ? v : 0;
    }
    first = incl - sum;
    total = __shfl(incl, 63);
    total = (int64_t)((uint64_t)__builtin_amdgcn_readfirstlane((int)(total >> 32)) << 32 |
                      (uint32_t)__builtin_amdgcn_readfirstlane((int)total));
    return true;
  }
  // The expert of tile `t` (below the total) and the first row of the tile.
  __device__ Group find(const ProductArgs& a, int64_t t, int64_t* m0) const {
    const int l = __popcll(__ballot(first <= t)) - 1;
    t -= (int64_t)((uint64_t)__builtin_amdgcn_readlane((int)(first >> 32), l) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)first, l));
    Group g = group_of(a, l * run);
    while (t >= of(g) && g.e + 1 < min((l + 1) * run, a.L)) {
      t -= of(g);
      g = group_of(a, g.e + 1);
    }
    *m0 = g.lo + t * BM;
    return g;
  }
};

// The expert with the n-th most rows (ties: the lower index first), of at most
// 64; of more, the n-th.
__device__ inline int nth_largest(const ProductArgs& a, int n, int lane) {
  if (a.L > 64) return n;
  Group g{lane, 0, 0};
  if (lane < a.L) {
    g.lo = a.offsets[lane];
    g.hi = a.offsets[lane + 1];
  }
  const int rows = (int)(g.hi - g.lo);
  int before = 0;
  for (int e = 0; e < a.L; ++e) {
    const int other = __builtin_amdgcn_readlane(rows, e);
    before += other > rows || (other == rows && e < lane);
  }
  return __builtin_ctzll(__ballot(lane < a.L && before == n));
}

__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
template <typename T> struct Frag;
template <> struct Frag<Bf16> { using type = bf16x8; };
template <> struct Frag<F16> { using type = f16x8; };

__device__ inline float silu(float g) { return activation<VP_ACT_SILU>(g); }

// ---------------------------------------------------------------- tiled products

constexpr int kStep = 128;   // bytes of a row that one step of the contraction takes
constexpr int kCus = 256;

// Starts a direct load of 16 bytes per lane from `off` of `bytes` bytes at
// `base` to 1 KB of LDS at `lds` (both the same for the whole wavefront).  It
// returns nothing in registers, and the loops below wait for it themselves:
// through the builtin the compiler puts a wait for all loads before every
// transposing LDS read.
__device__ inline void direct_load(const unsigned char* base, int bytes, uint32_t off, unsigned char* lds) {
#ifdef __HIP_DEVICE_COMPILE__
  const uint64_t b = (uint64_t)base;
  const auto same = [](uint32_t v) { return __builtin_amdgcn_readfirstlane((int)v); };   // in scalar registers
  const uint64_t words01 = (uint64_t)(uint32_t)same((uint32_t)(b >> 32) & 0xffff) << 32 | (uint32_t)same((uint32_t)b);
  const uint64_t words23 = 0x00020000ull << 32 | (uint32_t)same(bytes);
  const int at = same((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
  // A memory instruction may read a scalar register only five wait states after a vector instruction wrote it (the
  // read of a lane, or a spilled register's return, which the compiler may put right before this block); a scalar
  // instruction waits by itself, so the descriptor is moved by those.  They are also the wait state that m0 needs.
  // (No-operations in their place took up to 2% more of the smaller products.)
  asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 s[96:97], %2\n\ts_mov_b64 s[98:99], %3\n\t"
               "buffer_load_dwordx4 %1, s[96:99], 0 offen lds"
               :: "s"(at), "v"(off), "s"(words01), "s"(words23)
               : "memory", "s96", "s97", "s98", "s99");   // nothing else in these kernels uses m0
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

  // Once: this lane's offsets.  For rows by contraction `row_of(i)` gives the
  // buffer row of operand row i, relative to `base`.
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
  }
  __device__ void start(const unsigned char* at, int left_, int width_, int lane) {
    base = at;
    left = left_;
    width = width_;
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

// Steps of a contraction over an expert's rows, of which a buffer may hold 2^31 - 1.
constexpr __host__ __device__ int row_steps(int rows) { return rows / 64 + (rows % 64 != 0); }
static_assert(row_steps(0) == 0 && row_steps(64) == 1 && row_steps(65) == 2 && row_steps(0x7fffffff) == 1 << 25, "whole steps");

template <typename T> struct Mx { using out = T; };   // both operands in 4-bit blocks, results of type T
template <typename T> struct Elem { using out = T; static constexpr bool mx = false; };
template <typename T> struct Elem<Mx<T>> { using out = T; static constexpr bool mx = true; };

// A tile's results: where they go, its rows and columns inside the output, and
// the steps of its contraction.
struct TileOut {
  unsigned char *out, *pre;
  int rows, cols, steps;
};
struct DenseOut : TileOut {
  int64_t m0;   // its first row and column
  int n0;
};
// And where its operands begin and how much of them there is (see Operand).
template <typename Out> struct TileIn : Out {
  const unsigned char *a, *b;
  int a_left, a_width, b_left, b_width;
};

// The steps of a kernel that holds more than two come with the launch: knowing their size the compiler would give the one
// workgroup that a CU then holds both register files, and move sums between them.
extern __shared__ __attribute__((aligned(1024))) unsigned char more_steps[];

// Wavefronts that a SIMD has registers for at least: of the dense products' 128 x 128 tiles two workgroups share a CU (and
// with the registers of one, sums move between the two register files).
template <typename Args> constexpr int waves_of() { return std::is_same_v<Args, DenseArgs> ? 2 : 1; }

// Measured: 32768 rows by 4096 x 4096, bf16 0.83-0.88 ms (1.25-1.33 PFLOP/s; the
// library's product of that size 0.71 ms, 1.55), gated 0.82 and with the values
// before the gate 0.89, its row gradient 0.82-0.88, its weight gradient
// 0.82-0.89, 4-bit blocks 0.28-0.30 (3.7-3.9 PFLOP/s).  The matrix units are
// busy 62 % of the time at 1.8 to 1.9 GHz, to which the card's power holds the
// clock (registers alone, random operands: 1.75-1.85 PFLOP/s).  Without the
// loads 0.73 ms, without the LDS reads 0.85; waiting for neither changes
// nothing, nor does bringing the lines to the L2 ahead.  A tile costs 4 to 6 us
// beside its steps (results of all CUs go out together).
//
// WM x WN wavefronts, each with MT x NT fragments of 16 x 16 results.  A
// workgroup takes every gridDim / 8-th tile of its XCD's and runs through
// their steps as one stream: the loads are two steps ahead (STAGES), so that the next
// tile's first steps arrive while this one's results are written.
template <typename T, int MODE, bool GATED, int WM, int WN, int MT, int NT, typename Args = ProductArgs, int STAGES = 2>
__global__ void __launch_bounds__(WM * WN * 64, waves_of<Args>()) product_tiled(Args a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host's pass knows none of the builtins below
  using Out = typename Elem<T>::out;
  constexpr bool kMx = Elem<T>::mx, kColsA = MODE == kGradW, kColsB = MODE != kForward;
  constexpr bool kDense = std::is_same_v<Args, DenseArgs>;
  using TileTo = std::conditional_t<kDense, DenseOut, TileOut>;
  using TileAt = TileIn<TileTo>;
  constexpr int BM = WM * MT * 16, BN = WN * NT * 16, kWaves = WM * WN;
  constexpr int kTileN = GATED ? BN / 2 : BN;   // output columns
  constexpr int kSize = MODE == kGradW ? 4 : 2;
  constexpr bool kFixed = STAGES == 2;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kFixed ? STAGES : 1][kFixed ? (BM + BN) * kStep : 16];
  // 4-bit blocks: the powers of two of four steps, 32 bytes a row, double buffered
  __shared__ __attribute__((aligned(1024))) unsigned char powers[kMx ? 2 : 1][kMx ? (BM + BN) * 32 : 16];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, q = lane / 16;
  const int wm = wave / WN, wn = wave % WN;
  const int half = a.half;
  const int row_bytes = kMx ? a.C / 2 : a.C * 2;

  // Tiles: XCD x (block % 8) takes a contiguous eighth of them (of every
  // expert's, for grad w), in bands of four row tiles by all columns: what 32
  // workgroups hold at a time (4 by 8 tiles) shares most of its bytes in the
  // XCD's L2 (bands of 4, 8, 16, 32: 1.21, 1.18, 1.15, 1.11 PFLOP/s, 32768
  // rows, 4096 x 4096, gated).
  constexpr int kBand = 4;
  const int nt = (a.N + kTileN - 1) / kTileN, mt = MODE == kGradW ? (a.M + BM - 1) / BM : 0;
  RowTiles<BM> row_tiles;
  if constexpr (!kDense) {
    if (!row_tiles.init(a, lane)) {   // an error: nothing is written
      if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, VP_ERR_INVALID_ARGUMENT);
      return;
    }
  }
  int64_t slots = mt;   // row tiles (dense: of every part)
  int64_t high_slots = 0;   // dense: of one part
  if constexpr (kDense) {
    high_slots = MODE == kGradW ? mt : (a.R + BM - 1) / BM;
    slots = high_slots * a.parts;
  } else if constexpr (MODE != kGradW) {
    slots = row_tiles.total;
  }
  const uint32_t all = (uint32_t)(slots * nt), per = (all + 7) / 8;   // tiles, below 2^31; this XCD's
  const uint32_t first = blockIdx.x >> 3, stride = gridDim.x >> 3, last = MODE == kGradW && !kDense ? per * a.L : per;
  const auto dense_tile = [&](TileAt& t, int part, int64_t m0, int n0) {
    if constexpr (kDense) {
      const int64_t c0 = (int64_t)part * a.chunk;
      const int depth = (int)min((int64_t)a.chunk, (MODE == kGradW ? a.R : a.C) - c0);
      t.rows = (int)min((int64_t)BM, (MODE == kGradW ? a.M : a.R) - m0);
      t.cols = min(kTileN, a.N - n0);
      if (MODE == kGradW) {
        t.a = a.a + c0 * a.a_stride + m0 * 2;
        t.b = a.b + c0 * a.b_stride + n0 * 2;
        t.a_left = t.b_left = depth;
        t.a_width = (int)(a.M - m0) * 2;
        t.b_width = (a.N - n0) * 2;
        t.steps = row_steps(depth);
      } else {
        t.a = a.a + m0 * a.a_stride + c0 * 2;
        t.a_left = (t.rows - 1) * (int)a.a_stride + depth * 2;
        t.a_width = depth * 2;
        t.steps = (depth * 2 + kStep - 1) / kStep;
        if (MODE == kGradX) {
          t.b = a.b + c0 * a.b_stride + n0 * 2;
          t.b_left = depth;
          t.b_width = (a.N - n0) * 2;
        } else {
          t.b = a.b + n0 * a.b_stride + c0 * 2;
          t.b_left = (t.cols - 1) * (int)a.b_stride + depth * 2;
          t.b_width = depth * 2;
        }
      }
      t.steps = max(t.steps, STAGES);   // steps past the last add zeros
      t.m0 = m0;
      t.n0 = n0;
      t.out = a.out + part * a.part_bytes + m0 * a.out_stride + (int64_t)n0 * (a.wide ? 4 : 2);
      t.pre = a.pre ? a.pre + m0 * a.pre_stride + (int64_t)n0 * 2 : nullptr;
    }
  };
  const auto tile_at = [&](uint32_t idx, TileAt& t) -> bool {
    const uint32_t in_xcd = MODE == kGradW && !kDense ? idx % per : idx, at = (blockIdx.x & 7) * per + in_xcd;
    if (at >= all) return false;
    const uint32_t band = at / (uint32_t)(kBand * nt), in = at - band * (kBand * nt);
    const uint32_t high = min((uint32_t)kBand, (uint32_t)slots - band * kBand);
    const int64_t slot = band * kBand + in % high;
    const int n0 = (int)(in / high) * kTileN;
    if constexpr (kDense) {
      const int part = (int)((uint32_t)slot / (uint32_t)high_slots);
      dense_tile(t, part, (slot - part * high_slots) * BM, n0);
      return true;
    }
    Group g;
    int64_t m0;
    if (MODE == kGradW) {
      // the longest contractions first: the tiles are handed out as workgroups end
      g = group_of(a, nth_largest(a, (int)(idx / per), lane));
      m0 = slot * BM;
      t.rows = (int)min((int64_t)BM, a.M - m0);
    } else {
      g = row_tiles.find(a, slot, &m0);
      t.rows = (int)min((int64_t)BM, g.hi - m0);
    }
    const int rows = (int)(g.hi - g.lo);
    if (MODE == kGradW) {
      t.a = a.a + g.lo * a.a_stride + m0 * 2;
      t.b = a.b + g.lo * a.b_stride + n0 * 2;
      t.a_left = t.b_left = rows;
      t.a_width = (int)(a.M - m0) * 2;
      t.b_width = (a.N - n0) * 2;
      t.steps = row_steps(rows);   // an expert without rows: zeros
    } else {
      t.a = a.a + m0 * a.a_stride;
      t.a_left = (t.rows - 1) * (int)a.a_stride + row_bytes;
      t.a_width = row_bytes;
      t.steps = (row_bytes + kStep - 1) / kStep;
      if (MODE == kGradX) {
        t.b = a.b + g.e * a.b_expert + n0 * 2;
        t.b_left = a.C;
        t.b_width = (a.N - n0) * 2;
      } else {
        // gated: of every 64 operand rows the first 32 are gate rows, the others the same up rows
        t.b = a.b + g.e * a.b_expert + n0 * a.b_stride;
        const int64_t end = ((int64_t)(GATED ? half + a.N : a.N) - n0 - 1) * a.b_stride + row_bytes;
        t.b_left = (int)min(end, (int64_t)(GATED ? half + kTileN : BN) * a.b_stride);
        t.b_width = row_bytes;
      }
    }
    t.steps = max(t.steps, 2);   // steps past the last add zeros
    t.cols = min(kTileN, a.N - n0);
    t.out = a.out + (MODE == kGradW ? g.e * a.b_expert : 0) + m0 * a.out_stride + (int64_t)n0 * kSize;
    t.pre = GATED && a.pre ? a.pre + m0 * a.pre_stride + (int64_t)n0 * 2 : nullptr;
    return true;
  };
  const auto find = [&](uint32_t& idx, TileAt& t) {   // the first tile at or after idx
    for (; idx < last; idx += stride)
      if (tile_at(idx, t)) return true;
    return false;
  };

  // what is loaded, STAGES steps ahead of what is multiplied
  Operand<BM, kColsA, kWaves> oa;
  Operand<BN, kColsB, kWaves> ob;
  TileAt ahead;
  uint32_t load_idx = first;
  int load_step = 0, load_group = 0;
  if (!find(load_idx, ahead)) return;
  TileTo cur = ahead, next = ahead, after = ahead;   // of the multiplied tile and those begun since
  int begun = 0;   // how many of these: a tile has STAGES steps at least, so at most two
  const auto begin = [&] {
    oa.start(ahead.a, ahead.a_left, ahead.a_width, lane);
    ob.start(ahead.b, ahead.b_left, ahead.b_width, lane);
  };
  oa.stride = (int)a.a_stride;
  ob.stride = (int)a.b_stride;
  oa.init(wave, lane, [](int i) { return i; });
  ob.init(wave, lane, [=](int i) { return GATED ? i / 64 * 32 + i % 32 + (i & 32 ? half : 0) : i; });
  begin();
  const auto advance = [&] {
    if (++load_step < ahead.steps) {
      oa.next(lane);
      ob.next(lane);
      return;
    }
    load_idx += stride;
    load_step = 0;
    if (find(load_idx, ahead)) {
      begin();
      (begun == 0 ? next : after) = ahead;
      ++begun;
    } else {   // nothing is left: the loads bring zeros that nothing multiplies
      ahead.steps = 0x7fffffff;
      oa.start(ahead.a, 0, 0, lane);
      ob.start(ahead.b, 0, 0, lane);
    }
  };

  const auto stage = [&](int pos) -> unsigned char* {
    if constexpr (kFixed) return lds[pos & 1];
    else return more_steps + (pos & (STAGES - 1)) * ((BM + BN) * kStep);
  };
  // places of this lane's fragments in LDS
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
  const auto read_a = [&](int pos, int kk, int i) {
    return frag(stage(pos), std::bool_constant<kColsA>{}, std::integral_constant<int, BM>{}, pa[kColsA ? i : 0], i, kk);
  };
  const auto read_b = [&](int pos, int kk, int i) {
    return frag(stage(pos) + BM * kStep, std::bool_constant<kColsB>{}, std::integral_constant<int, BN>{}, pb[kColsB ? i : 0], i, kk);
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
      const int i = (wave * kPowerLoads + j) * 32 + lane % 32, n = i - BM;
      const int row = i < BM ? i : GATED ? n / 64 * 32 + n % 32 + (n & 32 ? half : 0) : n;
      power_off[j] = (uint32_t)(row * (i < BM ? oa.stride : ob.stride)) + row_bytes + lane / 32 * 16;
    }
  }
  const auto load_powers = [&] {   // of the next four steps to load
    if constexpr (kMx) {
      if (load_step % 4 != 0) return;
      const int tail = (row_bytes + a.C / 32 + 15) / 16 * 16 - row_bytes;   // a packed row's bytes after the codes
#pragma unroll
      for (int j = 0; j < kPowerLoads; ++j) {
        const int i0 = (wave * kPowerLoads + j) * 32;
        const bool is_a = i0 < BM;
        direct_load(is_a ? ahead.a : ahead.b, (is_a ? ahead.a_left : ahead.b_left) + tail,
                    power_off[j] + (uint32_t)(load_step * 8), powers[load_group & 1] + i0 * 32);
      }
      ++load_group;
    }
  };
  // The two powers of fragment row `row` + r in a step; blocks past the row's
  // last count as 2^-127 (their codes are zero).
  const auto read_power = [&](int group, int step, int row) -> int {
    if constexpr (kMx) {
      const int left = a.C / 32 - step * 8 - 2 * q;
      const int mask = left >= 2 ? 0xffff : left == 1 ? 0xff : 0;
      const unsigned char* at = powers[group & 1] + ((step & 2) << 8) + (step & 1) * 8 + 2 * q + r * 16;
      return *(const uint16_t*)(at + row / 32 * 1024 + row % 32 * 16) & mask;
    }
    return 0;
  };

  constexpr int kLoadsA = decltype(oa)::kLoads, kLoadsB = decltype(ob)::kLoads;
  // where the loads go among the rows of products: the columns' before the
  // middle of the step if there are rows enough, else all after it
  constexpr bool kEarly = MT == NT + 4;
  constexpr bool kTwo = kLoadsA == 2;   // loads of each operand: two, or four
  static_assert((kEarly || MT == 4) && kLoadsA == kLoadsB && (kLoadsA == 4 || (kTwo && !kEarly)), "the loads' places among the rows of products");
  const auto issue_a = [&](int pos, int j) { oa.issue(stage(pos), wave, j); };
  const auto issue_b = [&](int pos, int j) { ob.issue(stage(pos) + BM * kStep, wave, j); };
  const auto load = [&](int pos) {
    load_powers();
#pragma unroll
    for (int j = 0; j < kLoadsB; ++j) issue_b(pos, j);
#pragma unroll
    for (int j = 0; j < kLoadsA; ++j) issue_a(pos, j);
    advance();
  };

  f32x4 acc[MT][NT] = {};
  // One row of fragments: i of the rows' by all of the columns'.
  const auto multiply = [&](auto half_step, int i, const i32x4& fa, const i32x4 (&fb)[NT], int sa, const int (&sb)[NT]) {
    __builtin_amdgcn_sched_barrier(0);
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
    // the compiler would move these pure instructions past the loads' branches, to where the sums are next used
#pragma unroll
    for (int j = 0; j < (kMx ? NT : 0); ++j) asm volatile("" : "+v"(acc[i][j]));
    __builtin_amdgcn_sched_barrier(0);
  };

  // Results go through a descriptor of the tile's rows inside the output; what
  // lies outside is dropped there, so every wavefront issues the same number
  // of stores.  Neighbouring 16-lane rows exchange halves of two fragments,
  // after which a lane holds eight neighbouring 16-bit results.
  constexpr int kStores = MODE == kGradW ? MT * NT : GATED ? MT * NT / 4 : MT * NT / 2;
  const auto put = [&](unsigned char* base, int64_t row_stride, int rows, int cols, auto value) {
    const int bytes = rows > 0 ? (rows - 1) * (int)row_stride + cols * kSize : 0;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(base, 0, bytes, 0x00020000);
    constexpr int kCols = GATED ? NT / 2 : NT;   // output fragments of a wavefront's row
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint32_t row = (uint32_t)(((wm * MT + i) * 16 + r) * (int)row_stride);
      if constexpr (MODE == kGradW) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          const int n = (wn * kCols + j) * 16 + q * 4;
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, value(i, j)), rsrc,
                                                     n < cols ? row + n * 4 : 0x60000000u, 0, 0);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kCols; j += 2) {
          u32x2 p[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const f32x4 v = value(i, j + u);
            p[u].x = from_f32<Out>(v[0]).u | (uint32_t)from_f32<Out>(v[1]).u << 16;
            p[u].y = from_f32<Out>(v[2]).u | (uint32_t)from_f32<Out>(v[3]).u << 16;
          }
          const auto x = __builtin_amdgcn_permlane16_swap(p[0].x, p[1].x, false, false);
          const auto y = __builtin_amdgcn_permlane16_swap(p[0].y, p[1].y, false, false);
          const u32x4 o = {x[0], y[0], x[1], y[1]};
          const int n = (wn * kCols + j + (q & 1)) * 16 + (q >> 1) * 8;
          __builtin_amdgcn_raw_buffer_store_b128(o, rsrc, n < cols ? row + n * 2 : 0x60000000u, 0, 0);
        }
      }
    }
  };
  // The epilogue of a dense product, two neighbouring fragments at a time (all
  // of them through one step after the other would spill; the bias is what the
  // sums begin with).  A lane's four results of fragment (i, j) are row (wm MT +
  // i) 16 + r, columns (wn NT + j) 16 + 4 q on.  16-bit operands of the epilogue
  // come as the stores go, 16 bytes a lane for two fragments, and are brought to
  // the fragments' places by the same exchange; their loads run kFar pairs ahead.
  // 16381 rows by 4096 x 4096: 417-435 us without, 495-510 with bias, gelu, kept
  // values and residual (of which the residual and the kept values, 268 MB, 50 and
  // gelu 10-20); row by row of fragments, with the spilled registers, 560.
  const auto finish = [&](const TileTo& t) {
    if constexpr (kDense) {
      const auto resource = [&](const unsigned char* base, int64_t stride, int size) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, base ? (t.rows - 1) * (int)stride + t.cols * size : 0, 0x00020000);
      };
      const auto out = resource(t.out, a.out_stride, a.wide ? 4 : 2);
      // (the compiler must not know these places: it would compute all rows' offsets before the first tile, and spill)
      int row0 = wm * MT * 16 + r, quad = q;
      asm volatile("" : "+v"(row0), "+v"(quad));
      const auto wide_at = [&](int i, int j, int64_t stride) -> uint32_t {   // of 32-bit values
        const int n = (wn * NT + j) * 16 + quad * 4;
        return n < t.cols ? (uint32_t)(row0 * (int)stride + n * 4 + i * 16 * (int)stride) : 0x60000000u;
      };
      const auto put_wide = [&](int i, int j, const f32x4& v) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), out, wide_at(i, j, a.out_stride), 0, 0);
      };
      if (MODE == kGradW || a.raw) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) put_wide(i, j, acc[i][j]);
        return;
      }
      const auto half_at = [&](int p, int64_t stride) -> uint32_t {   // of pair p's 16-bit values
        const int i = p / (NT / 2), j = p % (NT / 2) * 2, n = (wn * NT + j + (quad & 1)) * 16 + (quad >> 1) * 8;
        return n < t.cols ? (uint32_t)(row0 * (int)stride + n * 2 + i * 16 * (int)stride) : 0x60000000u;
      };
      const auto put_half = [&](const auto& to, int64_t stride, int p, const f32x4 (&v)[2]) {
        u32x2 h[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          h[u].x = from_f32<Out>(v[u][0]).u | (uint32_t)from_f32<Out>(v[u][1]).u << 16;
          h[u].y = from_f32<Out>(v[u][2]).u | (uint32_t)from_f32<Out>(v[u][3]).u << 16;
        }
        const auto x = __builtin_amdgcn_permlane16_swap(h[0].x, h[1].x, false, false);
        const auto y = __builtin_amdgcn_permlane16_swap(h[0].y, h[1].y, false, false);
        const u32x4 o = {x[0], y[0], x[1], y[1]};
        __builtin_amdgcn_raw_buffer_store_b128(o, to, half_at(p, stride), 0, 0);
      };
      const auto get_half = [&](const u32x4& o, f32x4 (&v)[2]) {
        const auto x = __builtin_amdgcn_permlane16_swap(o[0], o[2], false, false);
        const auto y = __builtin_amdgcn_permlane16_swap(o[1], o[3], false, false);
#pragma unroll
        for (int u = 0; u < 2; ++u)
          v[u] = f32x4{to_f32(Out{(uint16_t)(x[u] & 0xffffu)}), to_f32(Out{(uint16_t)(x[u] >> 16)}),
                       to_f32(Out{(uint16_t)(y[u] & 0xffffu)}), to_f32(Out{(uint16_t)(y[u] >> 16)})};
      };
      const auto before = resource(t.pre, a.pre_stride, 2);
      const auto slope = resource(a.slope ? a.slope + t.m0 * a.slope_stride + (int64_t)t.n0 * 2 : nullptr, a.slope_stride, 2);
      const int size = a.wide ? 4 : 2;
      const auto residual = resource(a.residual ? a.residual + t.m0 * a.residual_stride + (int64_t)t.n0 * size : nullptr, a.residual_stride, size);
      const bool half_residual = a.residual && !a.wide;
      constexpr int kPairs = MT * NT / 2, kFar = 2;
      u32x4 far_slope[kFar], far_residual[kFar];
#pragma unroll
      for (int p = 0; p < kFar; ++p) {
        if (MODE == kGradX && a.slope) far_slope[p] = __builtin_amdgcn_raw_buffer_load_b128(slope, half_at(p, a.slope_stride), 0, 0);
        if (half_residual) far_residual[p] = __builtin_amdgcn_raw_buffer_load_b128(residual, half_at(p, a.residual_stride), 0, 0);
      }
#pragma unroll
      for (int p = 0; p < kPairs; ++p) {
        const int i = p / (NT / 2), j = p % (NT / 2) * 2;
        __builtin_amdgcn_sched_barrier(0);
        f32x4 v[2] = {acc[i][j], acc[i][j + 1]}, z[2];
        if constexpr (MODE == kForward) {
          if (t.pre) put_half(before, a.pre_stride, p, v);
          with_act(a.act, [&](auto act) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int c = 0; c < 4; ++c) v[u][c] = activation<decltype(act)::value>(v[u][c]);
          });
        } else if (a.slope) {
          get_half(far_slope[p % kFar], z);
          if (p + kFar < kPairs) far_slope[p % kFar] = __builtin_amdgcn_raw_buffer_load_b128(slope, half_at(p + kFar, a.slope_stride), 0, 0);
          with_act(a.act, [&](auto act) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int c = 0; c < 4; ++c) v[u][c] = through<decltype(act)::value>(v[u][c], z[u][c]);
          });
        }
        if (a.wide) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (a.residual)
              v[u] += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(residual, wide_at(i, j + u, a.residual_stride), 0, 0));
            put_wide(i, j + u, v[u]);
          }
        } else {
          if (half_residual) {
            get_half(far_residual[p % kFar], z);
            if (p + kFar < kPairs) far_residual[p % kFar] = __builtin_amdgcn_raw_buffer_load_b128(residual, half_at(p + kFar, a.residual_stride), 0, 0);
            v[0] += z[0];
            v[1] += z[1];
          }
          put_half(out, a.out_stride, p, v);
        }
      }
    }
  };
  // What a tile's sums begin with: zeros, or the bias of their columns.
  const auto first_sums = [&](const TileTo& t) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      f32x4 v = {0, 0, 0, 0};
      if constexpr (kDense && MODE == kForward) {
        const int n = t.n0 + (wn * NT + j) * 16 + q * 4;
        if (a.bias && !a.raw && n < a.N) v = bias4<Out>(a, n);
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[i][j] = v;
    }
  };
  const auto write = [&](const TileTo& t) {
    if constexpr (GATED) {
      // a wavefront's columns: of every four fragments two of the gate, then the same two of the up half
      const auto gate = [&](int i, int j) { return acc[i][j / 2 * 4 + j % 2]; };
      const auto up = [&](int i, int j) { return acc[i][j / 2 * 4 + j % 2 + 2]; };
      if (t.pre) {
        put(t.pre, a.pre_stride, t.rows, t.cols, gate);
        put(t.pre + (int64_t)half * 2, a.pre_stride, t.rows, t.cols, up);
      }
      put(t.out, a.out_stride, t.rows, t.cols, [&](int i, int j) {
        const f32x4 g = gate(i, j), u = up(i, j);
        f32x4 h;
#pragma unroll
        for (int v = 0; v < 4; ++v) h[v] = silu(g[v]) * u[v];
        return h;
      });
    } else if constexpr (kDense) {
      finish(t);
    } else {
      put(t.out, a.out_stride, t.rows, t.cols, [&](int i, int j) { return acc[i][j]; });
    }
  };

  // A step is two halves of 32 16-bit (128 4-bit) values, each MT rows of
  // products.  A row's fragment is replaced by its next half's as soon as the
  // row is done, so one set of them is enough; the columns' are read half a
  // step ahead.  Once every wavefront has read a step's columns (in its first
  // half) or rows (after the second half's first row) their place takes the
  // loads of the step after next.  These are spread between the rows of
  // products: issued together they hold up every wavefront's matrix
  // instructions behind the CU's one load path.
  constexpr std::integral_constant<int, 0> kFirst{};
  constexpr std::integral_constant<int, 1> kSecond{};
  i32x4 fa[MT], fb0[NT], fb1[NT];
  int sa[MT] = {}, sb[NT] = {};
  int step = 0, group = 0;
  static_assert(STAGES == 2 || (!kEarly && !kMx && STAGES == 4), "places of the steps ahead");
  load(0);
  load(1);
  if constexpr (STAGES == 4) {
    load(2);
    load(3);
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STAGES == 2 ? 0 : (STAGES - 1) * (kLoadsA + kLoadsB)) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < MT; ++i) fa[i] = read_a(0, 0, i);
#pragma unroll
  for (int i = 0; i < NT; ++i) fb0[i] = read_b(0, 0, i);
#pragma unroll
  for (int i = 0; i < MT; ++i) sa[i] = read_power(0, 0, (wm * MT + i) * 16);
#pragma unroll
  for (int i = 0; i < NT; ++i) sb[i] = read_power(0, 0, BM + (wn * NT + i) * 16);
  if constexpr (kDense && MODE == kForward) first_sums(cur);
  bool stored = false;
  // loads that were started after the next step's: of the steps after it, and those of this step's first half
  constexpr int kYounger = (STAGES - 2) * (kLoadsA + kLoadsB) + (kEarly ? kLoadsB : 0);
  for (int pos = 0;; ++pos) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (i < NT) fb1[i] = read_b(pos, 1, i);
      if (kEarly && i == NT + 1) {
        issue_b(pos + STAGES, 0);
        issue_b(pos + STAGES, 1);
      } else if (kEarly && i > NT + 1) {
        issue_b(pos + STAGES, i - NT);
      }
      multiply(kFirst, i, fa[i], fb0, sa[i], sb);
      if (kEarly && i == NT) {   // every wavefront has read the step's columns
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      fa[i] = read_a(pos, 1, i);
    }
    multiply(kSecond, 0, fa[0], fb1, sa[0], sb);
    // the next step has arrived (the stores of the tile before may be on
    // their way), and no wavefront reads this step's half any more
    if (stored) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kStores + kYounger) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kYounger) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const bool end = step + 1 == cur.steps;
    const int next_step = end ? 0 : step + 1;
    if (next_step % 4 == 0) ++group;
    load_powers();
    int sb1[NT] = {};
    fa[0] = read_a(pos + 1, 0, 0);
    sa[0] = read_power(group, next_step, wm * MT * 16);
    if (!kEarly) {
      issue_b(pos + STAGES, 0);
      issue_b(pos + STAGES, 1);
    }
#pragma unroll
    for (int i = 1; i < MT; ++i) {
      if (kEarly) {
        if (i % 2) issue_a(pos + STAGES, i / 2);
      } else if constexpr (kTwo) {
        if (i <= 2) issue_a(pos + STAGES, i - 1);
      } else {
        if (i == 1) {
          issue_b(pos + STAGES, 2);
          issue_b(pos + STAGES, 3);
        } else {
          issue_a(pos + STAGES, 2 * i - 4);
          issue_a(pos + STAGES, 2 * i - 3);
        }
      }
      const auto column = [&](int j) {
        fb0[j] = read_b(pos + 1, 0, j);
        sb1[j] = read_power(group, next_step, BM + (wn * NT + j) * 16);
      };
      if (i <= NT) column(i - 1);
      if (!kEarly && NT == MT && i == MT - 1) column(NT - 1);
      multiply(kSecond, i, fa[i], fb1, sa[i], sb);
      fa[i] = read_a(pos + 1, 0, i);
      sa[i] = read_power(group, next_step, (wm * MT + i) * 16);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) sb[i] = sb1[i];
    advance();
    stored = false;
    ++step;
    if (end) {
      write(cur);
      stored = kDense || !cur.pre;   // (a dense tile's other stores and loads come before its last, which are as many or more)
      if (begun == 0) break;
      cur = next;
      next = after;
      --begun;
      step = 0;
      if constexpr (kDense && MODE == kForward) {
        first_sums(cur);
      } else {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the last loads end before the LDS is another workgroup's
#endif
}

}  // namespace
}  // namespace vp
