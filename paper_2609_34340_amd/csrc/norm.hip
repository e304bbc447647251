// Layer norm over rows, its gradient, and sums over rows.
//
//   y = (x - m) r w + b,  m = mean(x) or 0,  r = 1 / sqrt(mean((x - m)^2) + eps)
//   u = (x - m) r, g = d_out w:  d_x = r (g - mean(g) - u mean(g u)) + residual
//   d_w = sum over rows of d_out u,  d_b = sum over rows of d_out
//
// A row stays in the registers of its lanes (16 of them, a wavefront, or a workgroup), so it is read once; longer rows
// are read again.  Statistics: every wavefront takes the mean of its values, then their deviations d from it, whose sum
// corrects the mean and the sum of squares; a workgroup joins its wavefronts' by the formula for two groups' variances
// (Chan, Golub, LeVeque 1979).  Means are kept as a base and a small shift, so nothing cancels in the results however far
// from zero the rows lie.  The statistics hold their sum, rounded: the gradient's u are off by up to half a unit of m's
// last place times r, all of a row by the same (2e-4 where m is 5000 times the deviation).
//
// HBM bounds both directions, and first the instructions had to become few enough: workgroups run through rows with their
// parameters in registers and the next row's loads on the way, pieces of rows that are whole carry no checks, and the
// wavefronts' statistics are joined across lanes (in a loop over the wavefronts by every lane they were more instructions
// than the row's values: 16384 rows of 7168, bf16, 414 a wavefront and row, 98.7 us; now 240 and 90 us, 5.2 TB/s, where a
// 1 GiB copy reaches 4.8 to 5.2).  96 rows of 4096 take 3.5 us, about a launch.  The gradient of 8192 rows of 4096 with a
// residual: 57 us, 4.7 TB/s, and 5 for the sums of its 256 workgroups; its registers (an output's sums for every column)
// leave a CU one workgroup, and two rows' loads ahead make up for it (one: 62 us; 128 registers and two workgroups spill:
// 122).  Rows that begin at any element cost little in 32 bits (4095 rows of 2047: 27 us, of 2048 22; forward 17.0, 15.6),
// in 16 half as much again forward (8192 rows of 4095: 42, of 4096 29) and nearly twice the time in the gradient (with its
// sums 93, 53).  Rows that are read again: 2048 of 32768 in 32 bits 170 us, their gradient 340; of 65536 in 16 bits 182, 422.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "numeric.h"
#include "rows.h"

namespace vp {
namespace {

struct NormArgs {
  int64_t T;
  int32_t H;
  const unsigned char *x, *d_out, *residual;
  const void *weight, *bias;
  bool center;
  int64_t x_stride, d_out_stride, residual_stride, out_stride;
  unsigned char* out;
  float* stats;
  const float* given;
  float eps;
  float* part;   // gradient: [workgroup][d_weight, d_bias][H], or null
};

__device__ inline float plus(float p, float q) { return p + q; }
// A value that a wavefront's lanes share, so that what follows from it (a row's address) takes scalar registers.
__device__ inline int same(int v) { return __builtin_amdgcn_readfirstlane(v); }

// To one unit of the last place; the hardware's takes the smallest numbers for 0, so these are scaled.
__device__ inline float inverse_root(float v) {
#ifdef __HIP_DEVICE_COMPILE__
  return v < 0x1p-100f ? __builtin_amdgcn_rsqf(v * 0x1p100f) * 0x1p50f : __builtin_amdgcn_rsqf(v);
#else
  return v;
#endif
}

// n neighbouring parameters, from column c of H on, as they lie in memory.
template <typename P, int n> struct Params {
  static constexpr int kVecs = n / Vec<P>::n;
  u32x4 v[kVecs];
  __device__ void load(const void* p, int c, int H) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) v[i] = load_piece((const P*)p + c + i * Vec<P>::n, H - c - i * Vec<P>::n);
  }
  __device__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) unpack16<P>(v[i], f + i * Vec<P>::n);
  }
};

// LANES lanes to a row (16 or 64; 0: the workgroup), each with up to NV pieces of it.
template <int LANES> struct RowOf {
  int lane, lanes, group, groups;   // within the row; rows of the workgroup
  __device__ RowOf() {
    lanes = LANES ? LANES : blockDim.x;
    lane = LANES ? threadIdx.x % LANES : threadIdx.x;
    group = LANES == 16 ? threadIdx.x / 16 : LANES ? same(threadIdx.x / 64) : 0;
    groups = LANES ? blockDim.x / LANES : 1;
  }
};

// How many of the row's values the lanes first .. first + 63 hold, of NV pieces of n each.
template <int NV, int n> __device__ inline int held(int first, int lanes, int H) {
  int sum = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) sum += min(max(H - (first + i * lanes) * n, 0), 64 * n);
  return sum;
}

constexpr int kMaxWaves = 16;

constexpr int kWaves = 6;   // wavefronts of a SIMD that the registers are kept to

template <typename T, typename P, int LANES, int NV>
__global__ void __launch_bounds__(LANES ? 256 : 1024, NV == 2 ? kWaves : 4) norm_kernel(NormArgs a) {
  constexpr int n = Vec<T>::n, kSum = LANES == 16 ? 16 : 64;
  __shared__ float from[2][3][kMaxWaves];   // base, shift and squares of each wavefront, for two rows in turn
  const RowOf<LANES> row;
  const int wave = same(threadIdx.x / 64), waves = blockDim.x / 64;
  constexpr bool kKeep = NV == 2;   // parameters stay in registers; with four pieces of a lane these would spill
  Params<P, n> w[kKeep ? NV : 1], b[kKeep ? NV : 1];
#pragma unroll
  for (int i = 0; i < (kKeep ? NV : 0); ++i) {
    const int c = (row.lane + i * row.lanes) * n;
    if (a.weight) w[i].load(a.weight, c, a.H);
    if (a.bias) b[i].load(a.bias, c, a.H);
  }
  const float count = (float)a.H;
  // of this wavefront's share of the row
  const int mine = LANES ? a.H : held<NV, n>(wave * 64, row.lanes, a.H);
  const bool full = mine == kSum * NV * n;   // no lane past the row's end
  const float each = 1.0f / (float)max(mine, 1), part_of_row = 1.0f / count;
  // of wavefront lane % 16, for the joint statistics
  const float theirs = LANES == 0 && (threadIdx.x & 15) < waves ? (float)held<NV, n>((threadIdx.x & 15) * 64, row.lanes, a.H) : 0.0f;
  const int64_t stride = (int64_t)gridDim.x * gridDim.y * row.groups;
  int64_t t = block_index() * row.groups + row.group;
  u32x4 next[NV] = {};
  const auto fetch = [&](int64_t at) {
    if (at >= a.T) return;   // what is there stays, and goes nowhere
    const T* x = (const T*)(a.x + at * a.x_stride);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (row.lane + i * row.lanes) * n;
      next[i] = full ? *(const u32x4_any*)(x + c) : load_piece(x + c, a.H - c);
    }
  };
  fetch(t);
  // every group of lanes goes on to the workgroup's last row, for the barriers and the exchanges between lanes
  for (int64_t t0 = t - row.group, turn = 0; t0 < a.T; t0 += stride, t += stride, ++turn) {
    float base = 0.0f, s = 0.0f, squares = 0.0f, d[NV][n];
#pragma unroll
    for (int i = 0; i < NV; ++i) unpack16<T>(next[i], d[i]);   // zeros past the row's end
    fetch(t + stride);
    if (a.center) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < n; ++e) base += d[i][e];
      base = across<kSum>(base, plus) * each;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < n; ++e) d[i][e] -= base;
      if (!full) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < n; ++e)
            if (e >= a.H - (row.lane + i * row.lanes) * n) d[i][e] = 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < n; ++e) {
        s += d[i][e];
        squares = __builtin_fmaf(d[i][e], d[i][e], squares);
      }
    squares = across<kSum>(squares, plus);
    float shift = 0.0f;
    if (a.center) {
      s = across<kSum>(s, plus);
      shift = s * each;
      squares -= s * shift;
    }
    const float mine_base = base;
    if constexpr (LANES == 0) {
      float (*all)[kMaxWaves] = from[turn & 1];
      if (threadIdx.x % 64 == 0) {
        all[0][wave] = base;
        all[1][wave] = shift;
        all[2][wave] = squares;
      }
      __syncthreads();
      // lane l of every 16 has wavefront l's
      const int l = threadIdx.x & 15;
      const bool in = l < waves;
      const float first = all[0][0], theirs_mean = in ? all[0][l] - first + all[1][l] : 0.0f;
      float total = in ? all[2][l] : 0.0f, delta = 0.0f;   // delta: of the row's mean from `first`
      if (a.center) {
        delta = across<16>(theirs * theirs_mean, plus) * part_of_row;
        const float d = theirs_mean - delta;
        total = __builtin_fmaf(theirs * d, d, total);
      }
      total = across<16>(total, plus);
      base = first;
      shift = delta;
      squares = total;
    }
    // (below 0 only by rounding; the hardware's root is as near as a rounded one and a division)
    const float r = inverse_root((squares < 0.0f ? 0.0f : squares * part_of_row) + a.eps);
    if (t >= a.T) continue;
    if (a.stats && row.lane == 0) {
      a.stats[2 * t] = base + shift;
      a.stats[2 * t + 1] = r;
    }
    const float off = (mine_base - base - shift) * r;   // d is from this wavefront's mean
    T* y = (T*)(a.out + t * a.out_stride);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (row.lane + i * row.lanes) * n;
      if (!full && c >= a.H) break;
      float f[n], p[n];
      constexpr auto at = [](int k) { return kKeep ? k : 0; };
#pragma unroll
      for (int e = 0; e < n; ++e) f[e] = __builtin_fmaf(d[i][e], r, off);
      if (a.weight) {
        if (!kKeep) w[0].load(a.weight, c, a.H);
        w[at(i)].get(p);
#pragma unroll
        for (int e = 0; e < n; ++e) f[e] *= p[e];
      }
      if (a.bias) {
        if (!kKeep) b[0].load(a.bias, c, a.H);
        b[at(i)].get(p);
#pragma unroll
        for (int e = 0; e < n; ++e) f[e] += p[e];
      }
      if (full) *(u32x4_any*)(y + c) = pack16<T>(f);
      else store_piece(y + c, pack16<T>(f), a.H - c);
    }
  }
}

// Two sums at a time.
struct Pair { float a, b; };
__device__ inline Pair wave_sum(Pair v) { return {across<64>(v.a, plus), across<64>(v.b, plus)}; }

// The gradient.  A workgroup's row groups of `waves` wavefronts (or 16 lanes) each run through rows and keep the sums of
// their columns' d_weight and d_bias in registers; at the end the groups' sums are joined in LDS, and the workgroups' by
// column_sums_kernel: the same order at every call.
constexpr int kGradThreads = 512;   // 1024 would leave 128 registers to a lane, and spill

template <typename T, typename P, int LANES, int NV>
__global__ void __launch_bounds__(kGradThreads) norm_grad_kernel(NormArgs a, int waves) {
  constexpr int n = Vec<T>::n, kSum = LANES == 16 ? 16 : 64;
  __shared__ Pair from[2][kGradThreads / 64];
  __shared__ float sums[kGradThreads * n];
  const int wave = same(threadIdx.x / 64);
  const int lanes = LANES ? LANES : waves * 64, groups = blockDim.x / lanes;
  const int group = LANES == 16 ? threadIdx.x / 16 : LANES ? wave : wave / waves, lane = threadIdx.x - group * lanes;
  constexpr bool kKeep = NV == 2;   // the weight stays in registers, and the residual is loaded ahead
  constexpr auto at = [](int k) { return kKeep ? k : 0; };
  Params<P, n> w[kKeep ? NV : 1];
  float dw[NV][n] = {}, db[NV][n] = {};
#pragma unroll
  for (int i = 0; i < (kKeep ? NV : 0); ++i)
    if (a.weight) w[i].load(a.weight, (lane + i * lanes) * n, a.H);
  const float count = (float)a.H;
  const int64_t stride = (int64_t)gridDim.x * groups;
  int64_t t = (int64_t)blockIdx.x * groups + group;
  // Past the row's end g is 0, but u of a zero would be -m r, which may pass 32 bits.  Lanes that hold nothing take x from
  // the row's beginning, and a partial piece goes on with its last value (16 bits), or its u are 0 (32 bits: 33.8 us for
  // 4095 rows of 2047, with the loads 34.8; every place checked in a branch costs whole rows 1 to 2%).
  constexpr bool kLast = n == 8;
  // Two rows ahead where registers allow: one row's arithmetic is shorter than a load.
  constexpr int kAhead = kKeep ? 2 : 1;
  struct Row { u32x4 x[NV], d[NV], res[kKeep ? NV : 1]; float m, r; } next[kAhead];
  const auto fetch = [&](Row& to, int64_t at_row) {
    const T *x = (const T*)(a.x + at_row * a.x_stride), *d = (const T*)(a.d_out + at_row * a.d_out_stride);
    const bool in = at_row < a.T;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * lanes) * n, cx = c < a.H ? c : 0;
      to.x[i] = load_piece<T, kLast>(x + cx, in ? a.H - cx : 0);
      to.d[i] = load_piece(d + c, in ? a.H - c : 0);   // zeros past the row's end
      if (kKeep && a.residual) to.res[at(i)] = load_piece((const T*)(a.residual + at_row * a.residual_stride) + c, in ? a.H - c : 0);
    }
    to.m = in ? a.given[2 * at_row] : 0.0f;
    to.r = in ? a.given[2 * at_row + 1] : 0.0f;
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(next[i], t + i * stride);
  int turn = 0;
  const auto one_row = [&](Row& row) {
    const float m = row.m, r = row.r;
    float u[NV][n], g[NV][n], p[n];
    u32x4 res[kKeep ? NV : 1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      unpack16<T>(row.x[i], u[i]);
      unpack16<T>(row.d[i], g[i]);
      if (kKeep) res[at(i)] = row.res[at(i)];
    }
    fetch(row, t + kAhead * stride);
    Pair s{0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < n; ++e) {
        u[i][e] = (u[i][e] - m) * r;
        if (!kLast && e > 0) u[i][e] = e < a.H - (lane + i * lanes) * n ? u[i][e] : 0.0f;
        dw[i][e] = __builtin_fmaf(g[i][e], u[i][e], dw[i][e]);
        db[i][e] += g[i][e];
      }
      if (a.weight) {
        if (!kKeep) w[0].load(a.weight, (lane + i * lanes) * n, a.H);
        w[at(i)].get(p);
#pragma unroll
        for (int e = 0; e < n; ++e) g[i][e] *= p[e];
      }
#pragma unroll
      for (int e = 0; e < n; ++e) {
        s.a += g[i][e];
        s.b = __builtin_fmaf(g[i][e], u[i][e], s.b);
      }
    }
    s = {across<kSum>(s.a, plus), across<kSum>(s.b, plus)};
    if constexpr (LANES == 0) {
      Pair* all = from[turn & 1];
      ++turn;
      if (threadIdx.x % 64 == 0) all[wave] = s;
      __syncthreads();
      s = {0.0f, 0.0f};
      for (int i = group * waves; i < (group + 1) * waves; ++i) {
        s.a += all[i].a;
        s.b += all[i].b;
      }
    }
    if (t >= a.T) return;
    const float mg = a.center ? -r * (s.a / count) : 0.0f, mgu = -r * (s.b / count);
    T* out = (T*)(a.out + t * a.out_stride);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * lanes) * n;
      if (c >= a.H) break;
      float f[n];
#pragma unroll
      for (int e = 0; e < n; ++e) f[e] = __builtin_fmaf(r, g[i][e], __builtin_fmaf(mgu, u[i][e], mg));
      if (a.residual) {
        if (!kKeep) res[0] = load_piece((const T*)(a.residual + t * a.residual_stride) + c, a.H - c);
        unpack16<T>(res[at(i)], p);
#pragma unroll
        for (int e = 0; e < n; ++e) f[e] += p[e];
      }
      store_piece(out + c, pack16<T>(f), a.H - c);
    }
  };
  // every group goes on to the workgroup's last row, for the barriers and the exchanges between lanes
  for (int64_t t0 = t - group; t0 < a.T;) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t0 < a.T) one_row(next[i]);
      t0 += stride;
      t += stride;
    }
  }
  if (!a.part) return;
  const auto join = [&](float (&mine)[NV][n], float* to) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < n; ++e) sums[e * blockDim.x + threadIdx.x] = mine[i][e];   // [element][group][lane]
      __syncthreads();
      for (int k = threadIdx.x; k < lanes * n; k += blockDim.x) {
        const int e = k / lanes, l = k % lanes, c = (l + i * lanes) * n + e;
        float s = 0.0f;
        for (int q = 0; q < groups; ++q) s += sums[e * blockDim.x + q * lanes + l];
        if (c < a.H) to[c] = s;
      }
    }
  };
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.H;
  join(dw, part);
  join(db, part + a.H);
}

// ------------------------------------------------------------- long rows

// Rows that no workgroup's registers hold: read again for every step, from the L2 as a rule.
constexpr int kLong = 1024;

__device__ inline Pair block_sum(Pair v, Pair* lds) {
  v = wave_sum(v);
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  Pair s{0.0f, 0.0f};
  for (int w = 0; w < kLong / 64; ++w) {
    s.a += lds[w].a;
    s.b += lds[w].b;
  }
  __syncthreads();
  return s;
}

template <typename T, typename P> __global__ void __launch_bounds__(kLong) norm_long_kernel(NormArgs a) {
  constexpr int n = Vec<T>::n;
  __shared__ Pair lds[kLong / 64];
  const int64_t t = block_index();
  if (t >= a.T) return;
  const T* x = (const T*)(a.x + t * a.x_stride);
  T* y = (T*)(a.out + t * a.out_stride);
  const float count = (float)a.H;
  const auto each = [&](auto f) {   // f(column, values, how many of them)
    for (int c = threadIdx.x * n; c < a.H; c += kLong * n) {
      float v[n];
      unpack16<T>(load_piece(x + c, a.H - c), v);
      f(c, v, a.H - c);
    }
  };
  float m = 0.0f;
  if (a.center) {
    Pair s{0.0f, 0.0f};
    each([&](int, const float* v, int) {
#pragma unroll
      for (int e = 0; e < n; ++e) s.a += v[e];
    });
    m = block_sum(s, lds).a / count;
  }
  Pair s{0.0f, 0.0f};
  each([&](int, const float* v, int left) {
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const float d = e < left ? v[e] - m : 0.0f;
      s.a += d;
      s.b = __builtin_fmaf(d, d, s.b);
    }
  });
  s = block_sum(s, lds);
  const float shift = a.center ? s.a / count : 0.0f, squares = s.b - s.a * shift;
  const float r = inverse_root((squares < 0.0f ? 0.0f : squares / count) + a.eps);
  if (a.stats && threadIdx.x == 0) {
    a.stats[2 * t] = m + shift;
    a.stats[2 * t + 1] = r;
  }
  each([&](int c, float* v, int left) {
    Params<P, n> p;
    float f[n];
#pragma unroll
    for (int e = 0; e < n; ++e) v[e] = (v[e] - m - shift) * r;
    if (a.weight) {
      p.load(a.weight, c, a.H);
      p.get(f);
#pragma unroll
      for (int e = 0; e < n; ++e) v[e] *= f[e];
    }
    if (a.bias) {
      p.load(a.bias, c, a.H);
      p.get(f);
#pragma unroll
      for (int e = 0; e < n; ++e) v[e] += f[e];
    }
    store_piece(y + c, pack16<T>(v), left);
  });
}

// d_x of a long row.
template <typename T, typename P> __global__ void __launch_bounds__(kLong) norm_grad_long_kernel(NormArgs a) {
  constexpr int n = Vec<T>::n;
  __shared__ Pair lds[kLong / 64];
  const int64_t t = block_index();
  if (t >= a.T) return;
  const T *x = (const T*)(a.x + t * a.x_stride), *d = (const T*)(a.d_out + t * a.d_out_stride);
  const float m = a.given[2 * t], r = a.given[2 * t + 1], count = (float)a.H;
  const auto each = [&](auto f) {   // f(column, u, g, how many of them)
    for (int c = threadIdx.x * n; c < a.H; c += kLong * n) {
      float u[n], g[n], p[n];
      unpack16<T>(load_piece(x + c, a.H - c), u);
      unpack16<T>(load_piece(d + c, a.H - c), g);
#pragma unroll
      for (int e = 0; e < n; ++e) u[e] = (u[e] - m) * r;
      if (a.weight) {
        Params<P, n> w;
        w.load(a.weight, c, a.H);
        w.get(p);
#pragma unroll
        for (int e = 0; e < n; ++e) g[e] *= p[e];
      }
      f(c, u, g, a.H - c);
    }
  };
  Pair s{0.0f, 0.0f};
  each([&](int, const float* u, const float* g, int left) {
#pragma unroll
    for (int e = 0; e < n; ++e) {
      s.a += g[e];
      s.b = __builtin_fmaf(g[e], e < left ? u[e] : 0.0f, s.b);
    }
  });
  s = block_sum(s, lds);
  const float mg = a.center ? s.a / count : 0.0f, mgu = s.b / count;
  each([&](int c, float* u, const float* g, int left) {
    float res[n];
#pragma unroll
    for (int e = 0; e < n; ++e) u[e] = r * (g[e] - mg - u[e] * mgu);
    if (a.residual) {
      unpack16<T>(load_piece((const T*)(a.residual + t * a.residual_stride) + c, left), res);
#pragma unroll
      for (int e = 0; e < n; ++e) u[e] += res[e];
    }
    store_piece((T*)(a.out + t * a.out_stride) + c, pack16<T>(u), left);
  });
}

// d_weight and d_bias of long rows: a thread takes a piece of the columns and every parts-th row.
template <typename T> __global__ void __launch_bounds__(256) norm_params_long_kernel(NormArgs a, int parts) {
  constexpr int n = Vec<T>::n;
  const int c = (blockIdx.x * 256 + threadIdx.x) * n;
  if (c >= a.H) return;
  float dw[n] = {}, db[n] = {};
  for (int64_t t = blockIdx.y; t < a.T; t += parts) {
    const float m = a.given[2 * t], r = a.given[2 * t + 1];
    float x[n], d[n];
    unpack16<T>(load_piece((const T*)(a.x + t * a.x_stride) + c, a.H - c), x);
    unpack16<T>(load_piece((const T*)(a.d_out + t * a.d_out_stride) + c, a.H - c), d);
#pragma unroll
    for (int e = 0; e < n; ++e) {
      dw[e] = __builtin_fmaf(d[e], (x[e] - m) * r, dw[e]);
      db[e] += d[e];
    }
  }
  float* part = a.part + (int64_t)blockIdx.y * 2 * a.H;
#pragma unroll
  for (int e = 0; e < n; ++e) {
    if (c + e < a.H) {
      part[c + e] = dw[e];
      part[a.H + c + e] = db[e];
    }
  }
}

// ---------------------------------------------------------------- sums over rows

// part [parts][width]: columns below `split` go to first, the others to second (either may be null).  A workgroup has 32
// columns; a thread sums four of them over every 32nd part, and the threads' sums are added in order.
constexpr int kSumCols = 32, kSumSlices = 32;

__global__ void __launch_bounds__(256) column_sums_kernel(const float* part, int parts, int64_t width, int64_t split,
                                                          float* first, float* second) {
  __shared__ f32x4 lds[kSumSlices][kSumCols / 4];
  const int quad = threadIdx.x % (kSumCols / 4), slice = threadIdx.x / (kSumCols / 4);
  const int64_t c = (int64_t)blockIdx.x * kSumCols + quad * 4;
  f32x4 s = {0, 0, 0, 0};
  if (c < width) {
#pragma unroll 8
    for (int i = slice; i < parts; i += kSumSlices) {
      const u32x4 v = load_piece(part + (int64_t)i * width + c, width - c);
      s += __builtin_bit_cast(f32x4, v);
    }
  }
  lds[slice][quad] = s;
  __syncthreads();
  if (threadIdx.x >= kSumCols) return;
  const int64_t at = (int64_t)blockIdx.x * kSumCols + threadIdx.x;
  if (at >= width) return;
  float sum = 0.0f;
  for (int i = 0; i < kSumSlices; ++i) sum += lds[i][threadIdx.x / 4][threadIdx.x % 4];
  float* to = at < split ? first : second;
  if (to) to[at < split ? at : at - split] = sum;
}

// ------------------------------------------------------------------- host

// Lanes of a row and pieces of a lane, from the row's pieces.
struct NormPlan { int lanes, per; int waves; };   // lanes 0: `waves` wavefronts; per 0: a long row
NormPlan plan_of(int64_t pieces, bool grad) {
  const int most = (grad ? kGradThreads : 1024) / 64;   // wavefronts
  const int64_t two = (pieces + 127) / 128, four = (pieces + 255) / 256;
  if (pieces <= 32) return {16, 2, 0};
  if (pieces <= 128) return {64, 2, 0};
  if (two <= most) return {0, 2, (int)two};
  if (four <= most) return {0, 4, (int)four};
  return {0, 0, 0};
}

constexpr int kCus = 256;
constexpr int kParts = kCus;   // workgroups of the gradient, at most: registers allow one or two on a CU

NormArgs norm_args(const NormLaunch& p) {
  NormArgs a{};
  a.T = p.T;
  a.H = (int32_t)p.H;
  a.x = (const unsigned char*)p.x;
  a.d_out = (const unsigned char*)p.d_out;
  a.residual = (const unsigned char*)p.residual;
  a.weight = p.weight;
  a.bias = p.bias;
  a.center = p.center;
  a.x_stride = p.x_stride;
  a.d_out_stride = p.d_out_stride;
  a.residual_stride = p.residual_stride;
  a.out_stride = p.out_stride;
  a.out = (unsigned char*)p.out;
  a.stats = p.stats;
  a.given = p.given;
  a.eps = p.eps;
  a.part = p.d_weight || p.d_bias ? (float*)p.ws : nullptr;
  return a;
}

// Calls f with the rows' type and the parameters'.
template <typename F> void with_types(const NormLaunch& p, F f) {
  with_type(p.dtype, [&](auto t) {
    if (p.param_dtype == VP_F32) f(t, float{});
    else f(t, t);
  });
}

// Calls f with the lanes and pieces as types.
template <typename F> void with_plan(const NormPlan& p, F f) {
  if (p.lanes == 16) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
  else if (p.lanes == 64) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  else if (p.per == 2) f(std::integral_constant<int, 0>{}, std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 0>{}, std::integral_constant<int, 4>{});
}

}  // namespace

vp_status launch_column_sums(const float* part, int parts, int64_t width, int64_t split, float* first, float* second,
                             void* stream) {
  hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((width + kSumCols - 1) / kSumCols)), dim3(256), 0, (hipStream_t)stream,
                     part, parts, width, split, first, second);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "column sum launch failed");
  return VP_OK;
}

vp_status launch_layer_norm(const NormLaunch& p, void* stream) {
  const NormArgs a = norm_args(p);
  const hipStream_t s = (hipStream_t)stream;
  with_types(p, [&](auto t, auto q) {
    using T = decltype(t);
    using P = decltype(q);
    const NormPlan plan = plan_of((p.H + Vec<T>::n - 1) / Vec<T>::n, false);
    if (plan.per == 0) {
      hipLaunchKernelGGL((norm_long_kernel<T, P>), grid_of(a.T), dim3(kLong), 0, s, a);
      return;
    }
    with_plan(plan, [&](auto lanes, auto per) {
      constexpr int L = decltype(lanes)::value, V = decltype(per)::value;
      const int threads = L ? 256 : plan.waves * 64, rows = L ? 256 / std::max(L, 1) : 1;
      // workgroups that keep their parameters over many rows: as many as are resident at once
      const int64_t blocks = std::min<int64_t>((a.T + rows - 1) / rows, kCus * std::max(4 * (V == 2 ? kWaves : 4) * 64 / threads, 1));
      hipLaunchKernelGGL((norm_kernel<T, P, L, V>), grid_of(blocks), dim3(threads), 0, s, a);
    });
  });
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "norm launch failed");
  return VP_OK;
}

size_t layer_norm_grad_workspace(int64_t T, int64_t H) { return (size_t)std::min<int64_t>(T, kParts) * 2 * H * 4; }

vp_status launch_layer_norm_grad(const NormLaunch& p, void* stream) {
  const NormArgs a = norm_args(p);
  const hipStream_t s = (hipStream_t)stream;
  int parts = (int)std::min<int64_t>(a.T, kParts);
  if (a.T > 0) {
    with_types(p, [&](auto t, auto q) {
      using T = decltype(t);
      using P = decltype(q);
      const int64_t pieces = (p.H + Vec<T>::n - 1) / Vec<T>::n;
      const NormPlan plan = plan_of(pieces, true);
      if (plan.per == 0) {
        if (a.part) {   // before d_x, which may take d_out's place
          hipLaunchKernelGGL((norm_params_long_kernel<T>), dim3((unsigned)((pieces + 255) / 256), parts), dim3(256), 0, s, a, parts);
        }
        hipLaunchKernelGGL((norm_grad_long_kernel<T, P>), grid_of(a.T), dim3(kLong), 0, s, a);
        return;
      }
      with_plan(plan, [&](auto lanes, auto per) {
        constexpr int L = decltype(lanes)::value, V = decltype(per)::value;
        const int rows = L ? kGradThreads / std::max(L, 1) : std::max(1, kGradThreads / 64 / plan.waves);
        const int threads = L ? kGradThreads : rows * plan.waves * 64;
        parts = (int)std::min<int64_t>((a.T + rows - 1) / rows, kParts);
        hipLaunchKernelGGL((norm_grad_kernel<T, P, L, V>), dim3(parts), dim3(threads), 0, s, a, plan.waves);
      });
    });
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "norm gradient launch failed");
  return a.part || (a.T == 0 && (p.d_weight || p.d_bias))
             ? launch_column_sums((const float*)p.ws, parts, 2 * p.H, p.H, p.d_weight, p.d_bias, stream)
             : VP_OK;
}

}  // namespace vp
