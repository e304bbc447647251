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
//
// Each step of the contraction brings 128 bytes of every row of both operands
// to LDS (64 16-bit values, or 256 4-bit ones) by direct loads, double
// buffered.  Both operands are read through buffer descriptors that end with
// the expert's last row: what lies outside reads as zero, so no neighbour's
// row (which may hold anything) enters a sum.  The places in LDS are permuted
// so that the matrix fragments' reads meet no bank twice (in 4-bit blocks, whose
// lanes take neighbouring chunks, some do):
//   rows by contraction   16-byte chunk c of row r at place c ^ (r & 7); a
//                         fragment lane reads its row's chunk whole
//   contraction by rows   (grad x's weights, both operands of grad w) 32-byte
//                         piece p of contraction row c at place p ^ f(c), read
//                         through the transposing LDS load
// The product is computed as its transpose, so that a lane's four results are
// neighbours in the output row.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "numeric.h"
#include "report.h"

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

// To a few units of the last place of 32 bits for |g| in the tens (the product
// with log2 e is rounded), far inside the 16 bits that the result is rounded
// to; the library's exponential and divide cost a gated tile 64 times 30
// instructions a lane.
__device__ inline float fast_sigmoid(float g) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504089f));
#else
  return g;
#endif
}
__device__ inline float silu(float g) { return g * fast_sigmoid(g); }

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
// And where its operands begin and how much of them there is (see Operand).
struct TileAt : TileOut {
  const unsigned char *a, *b;
  int a_left, a_width, b_left, b_width;
};

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
// their steps as one stream: the loads are two steps ahead, so that the next
// tile's first steps arrive while this one's results are written.
template <typename T, int MODE, bool GATED, int WM, int WN, int MT, int NT>
__global__ void __launch_bounds__(WM * WN * 64) product_tiled(ProductArgs a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host's pass knows none of the builtins below
  using Out = typename Elem<T>::out;
  constexpr bool kMx = Elem<T>::mx, kColsA = MODE == kGradW, kColsB = MODE != kForward;
  constexpr int BM = WM * MT * 16, BN = WN * NT * 16, kWaves = WM * WN;
  constexpr int kTileN = GATED ? BN / 2 : BN;   // output columns
  constexpr int kSize = MODE == kGradW ? 4 : 2;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2][(BM + BN) * kStep];
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
  if (!row_tiles.init(a, lane)) {   // an error: nothing is written
    if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, VP_ERR_INVALID_ARGUMENT);
    return;
  }
  const int64_t slots = MODE == kGradW ? mt : row_tiles.total;   // row tiles
  const uint32_t all = (uint32_t)(slots * nt), per = (all + 7) / 8;   // tiles, below 2^31; this XCD's
  const uint32_t first = blockIdx.x >> 3, stride = gridDim.x >> 3, last = MODE == kGradW ? per * a.L : per;
  const auto tile_at = [&](uint32_t idx, TileAt& t) -> bool {
    const uint32_t in_xcd = MODE == kGradW ? idx % per : idx, at = (blockIdx.x & 7) * per + in_xcd;
    if (at >= all) return false;
    const uint32_t band = at / (uint32_t)(kBand * nt), in = at - band * (kBand * nt);
    const uint32_t high = min((uint32_t)kBand, (uint32_t)slots - band * kBand);
    const int64_t slot = band * kBand + in % high;
    const int n0 = (int)(in / high) * kTileN;
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

  // what is loaded, two steps ahead of what is multiplied
  Operand<BM, kColsA, kWaves> oa;
  Operand<BN, kColsB, kWaves> ob;
  TileAt ahead;
  uint32_t load_idx = first;
  int load_step = 0, load_group = 0;
  if (!find(load_idx, ahead)) return;
  TileOut cur = ahead, next = ahead, after = ahead;   // of the multiplied tile and those begun since
  int begun = 0;   // how many of these: a tile has two steps at least, so at most two
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
    return frag(lds[pos & 1], std::bool_constant<kColsA>{}, std::integral_constant<int, BM>{}, pa[kColsA ? i : 0], i, kk);
  };
  const auto read_b = [&](int pos, int kk, int i) {
    return frag(lds[pos & 1] + BM * kStep, std::bool_constant<kColsB>{}, std::integral_constant<int, BN>{}, pb[kColsB ? i : 0], i, kk);
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
  static_assert((kEarly || MT == 4) && kLoadsA == 4 && kLoadsB == 4, "the loads' places among the rows of products");
  const auto issue_a = [&](int pos, int j) { oa.issue(lds[pos & 1], wave, j); };
  const auto issue_b = [&](int pos, int j) { ob.issue(lds[pos & 1] + BM * kStep, wave, j); };
  const auto load = [&](int pos) {
    load_powers();
#pragma unroll
    for (int j = 0; j < 4; ++j) issue_b(pos, j);
#pragma unroll
    for (int j = 0; j < 4; ++j) issue_a(pos, j);
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
  const auto write = [&](const TileOut& t) {
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
  load(0);
  load(1);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
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
  bool stored = false;
  for (int pos = 0;; ++pos) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (i < NT) fb1[i] = read_b(pos, 1, i);
      if (kEarly && i == NT + 1) {
        issue_b(pos + 2, 0);
        issue_b(pos + 2, 1);
      } else if (kEarly && i > NT + 1) {
        issue_b(pos + 2, i - NT);
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
    if (stored) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kStores + (kEarly ? kLoadsB : 0)) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kEarly ? kLoadsB : 0) : "memory");
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
      issue_b(pos + 2, 0);
      issue_b(pos + 2, 1);
    }
#pragma unroll
    for (int i = 1; i < MT; ++i) {
      if (kEarly) {
        if (i % 2) issue_a(pos + 2, i / 2);
      } else {
        if (i == 1) {
          issue_b(pos + 2, 2);
          issue_b(pos + 2, 3);
        } else {
          issue_a(pos + 2, 2 * i - 4);
          issue_a(pos + 2, 2 * i - 3);
        }
      }
      const auto column = [&](int j) {
        fb0[j] = read_b(pos + 1, 0, j);
        sb1[j] = read_power(group, next_step, BM + (wn * NT + j) * 16);
      };
      if (i <= NT) column(i - 1);
      if (!kEarly && i == MT - 1) column(NT - 1);
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
      stored = !cur.pre;
      if (begun == 0) break;
      cur = next;
      next = after;
      --begun;
      step = 0;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the last loads end before the LDS is another workgroup's
#endif
}

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
      const float s = fast_sigmoid(g[i]), du = dh[i] * g[i] * s;
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
