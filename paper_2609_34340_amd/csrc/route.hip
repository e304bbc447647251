// Routing to experts and its gradient.
//
// A token's scores are the softmax over its E logits or each logit's sigmoid.
// The experts are chosen by score + bias (the bias balances the load and takes
// no part in the weights); without a bias by the logits themselves, which have
// the same order.  With groups, the groups with the largest sums of their
// best one or two keys are kept and the rest left out.  The k best keys win,
// ties to the lowest index; their weights are scale * score, divided by their
// sum when renormalised.
//
// What bounds it: T * E * 2 or 4 bytes are read once (16,384 tokens of 256
// 16-bit logits: 8.4 MB, 1.6 us), so the work is the choice itself: k rounds
// of a maximum over E.  LPT lanes share a token, V keys each in registers: a
// round is V/2 three-way maxima, log2(LPT) cross-lane steps for the value, the
// same for the lowest index that has it, and V steps that strike it out.  The
// cross-lane steps stay in the vector unit (inside rows of 16 lanes by data
// movement in the operand, across them by row swaps): through LDS permutes
// 16,384 tokens of 256 take 13.7 us, this way 13.2, and 96 tokens 14 and 8 (sigmoid,
// bias, eight groups).
//
// Sixteen lanes per token (four tokens side by side in a wavefront) where there
// are tokens to fill the CUs: fewer lanes take fewer cross-lane steps and share
// each instruction among more tokens.  A whole wavefront for few tokens, whose
// call is one token's latency, and above 256 experts.
//
// Keys are unsigned integers in the order of the floats, so that a struck-out
// key (0), one that may not be chosen (1) and every number are comparable.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "numeric.h"
#include "report.h"

namespace vp {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kTaken = 0, kMasked = 1;   // below the key of every number

__device__ inline uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // -0 counts as +0
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ inline float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

struct RouteArgs {
  const void* logits;
  int64_t T, stride;   // elements between rows
  int32_t E, k, sigmoid, n_groups, top_groups, group_top, renorm;
  float scale;
  const float* bias;
  int32_t* ids;
  float* weights;
};

// Expert of register v on lane `sub`: lanes side by side, so that a register's load covers whole lines.
template <int LPT> __device__ inline int expert_of(int v, int sub) { return v * LPT + sub; }

template <typename T, int LPT, int V>
__global__ void __launch_bounds__(kThreads) route_kernel(RouteArgs a) {
  const int kTok = blockDim.x / LPT;
  extern __shared__ uint32_t lds[];
  const int E = a.E, k = a.k, tok = threadIdx.x / LPT, sub = threadIdx.x % LPT;
  const int64_t t = block_index() * kTok + tok;
  const bool live = t < a.T;
  const T* row = (const T*)a.logits + (live ? t : a.T - 1) * a.stride;   // a spare token repeats the last one

  float x[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = expert_of<LPT>(v, sub);
    x[v] = e < E ? to_f32(row[e]) : -INFINITY;
  }
  // softmax: maximum and sum over the row, in 32 bits
  float top = -INFINITY, inv = 1.0f;
  if (!a.sigmoid) {
#pragma unroll
    for (int v = 0; v < V; ++v) top = fmaxf(top, x[v]);
    top = across<LPT>(top, [](float p, float q) { return fmaxf(p, q); });
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) sum += x[v] == -INFINITY ? 0.0f : expf(x[v] - top);   // NaN stays in the sum
    sum = across<LPT>(sum, [](float p, float q) { return p + q; });
    inv = 1.0f / sum;
  }
  const auto score = [&](float z) {
    if (z == -INFINITY) return 0.0f;
    return a.sigmoid ? sigmoid(z) : expf(z - top) * inv;
  };
  uint32_t key[V];
  const bool by_logit = !a.bias && a.n_groups == 1;
  // A NaN is in every score of its row (an infinity too), and so in the weights.  The choice is made by the scores of
  // the numbers: NaN left out, infinity their limit.  (From the row again: in registers, another pass over them would
  // cost the 4,096-expert kernel a wavefront per SIMD.)
  float key_inv = inv;
  if (!a.sigmoid && !by_logit && !(inv == inv)) {   // the same in all lanes of the token
    float sum = 0.0f;
    for (int e = sub; e < E; e += LPT) {
      const float z = to_f32(row[e]);
      sum += z == -INFINITY || !(z == z) ? 0.0f : z == top ? 1.0f : expf(z - top);
    }
    key_inv = 1.0f / across<LPT>(sum, [](float p, float q) { return p + q; });
  }
  const auto key_score = [&](float z) { return a.sigmoid ? sigmoid(z) : (z == top ? 1.0f : expf(z - top)) * key_inv; };
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = expert_of<LPT>(v, sub);
    float s = x[v];
    if (!by_logit) {
      s = key_score(s);
      if (a.bias && e < E) s += a.bias[e];
    }
    key[v] = e >= E ? kTaken : (x[v] == -INFINITY || !(s == s)) ? kMasked : ordered(s);
  }

  uint32_t* ids = lds + tok * (k + 1);   // this token's choices
  if (a.n_groups > 1) {
    // group scores by one lane per group over the token's keys in LDS
    // (rows of E + 1 words), then each group's rank among the groups
    uint32_t* keys = lds + kTok * (k + 1) + tok * (E + 1 + 2 * a.n_groups);
    float* gs = (float*)(keys + E + 1);
    uint32_t* kept = (uint32_t*)gs + a.n_groups;
    const int per = E / a.n_groups;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (expert_of<LPT>(v, sub) < E) keys[expert_of<LPT>(v, sub)] = key[v];
    __syncthreads();
    for (int g = sub; g < a.n_groups; g += LPT) {
      uint32_t first = kMasked, second = kMasked;
      for (int i = 0; i < per; ++i) {
        const uint32_t q = keys[g * per + i];
        second = max(second, min(first, q));
        first = max(first, q);
      }
      // a masked expert adds nothing; a group of masked experts is last
      const auto back = [](uint32_t q) { return __uint_as_float(q ^ ((q >> 31) ? 0x80000000u : 0xffffffffu)); };
      float s = first == kMasked ? -INFINITY : back(first);
      if (a.group_top == 2 && second != kMasked) s += back(second);
      gs[g] = s;
    }
    __syncthreads();
    for (int g = sub; g < a.n_groups; g += LPT) {
      const float mine = gs[g];
      int before = 0;
      for (int h = 0; h < a.n_groups; ++h) before += gs[h] > mine || (gs[h] == mine && h < g);
      kept[g] = before < a.top_groups;
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = expert_of<LPT>(v, sub);
      if (e < E && !kept[e / per]) key[v] = kMasked;
    }
  }

  for (int j = 0; j < k; ++j) {
    uint32_t best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    best = across<LPT>(best, [](uint32_t p, uint32_t q) { return max(p, q); });
    uint32_t at = ~0u;
#pragma unroll
    for (int v = 0; v < V; ++v) at = min(at, key[v] == best ? (uint32_t)expert_of<LPT>(v, sub) : ~0u);
    at = across<LPT>(at, [](uint32_t p, uint32_t q) { return min(p, q); });
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = (uint32_t)expert_of<LPT>(v, sub) == at ? kTaken : key[v];
    if (sub == 0) ids[j] = at | (best == kMasked ? 0x80000000u : 0u);
  }
  __syncthreads();

  // weights: lane `sub` takes slots sub, sub + LPT, ...
  // (an expert that was left when nothing else was has weight 0, but NaN stays)
  const auto chosen = [&](uint32_t id) {
    const float z = to_f32(row[id & 0x7fffffffu]);
    return id >> 31 && z == z ? 0.0f : score(z);
  };
  float sum = 0.0f;
  for (int j = sub; j < k; j += LPT) sum += chosen(ids[j]);
  sum = across<LPT>(sum, [](float p, float q) { return p + q; });
  for (int j = sub; j < k && live; j += LPT) {
    const uint32_t id = ids[j];
    const float s = chosen(id);
    const float w = a.renorm ? (s == 0.0f ? 0.0f : a.scale * s / sum) : a.scale * s;
    a.ids[t * k + j] = (int32_t)(id & 0x7fffffffu);
    a.weights[t * k + j] = w;
  }
}

// Gradient.  With w the weights, d their gradients and dot = sum of w d:
//   softmax, renormalised    dx_j = w_j (d_j - dot / scale) on the chosen, 0 elsewhere
//                            (the sum over all experts cancels)
//   softmax                  dx_i = w_i d_i [i chosen] - p_i dot
//   sigmoid, renormalised    dx_j = w_j (1 - s_j) (d_j - dot / scale)
//   sigmoid                  dx_j = w_j (1 - s_j) d_j
// One wavefront per token: the chosen experts' terms are put at their places
// in LDS, then the row is written once; the logits are read only where the
// formula has them.  T * E * 2 or 4 bytes are written, and as many read for
// the plain softmax: 8191 tokens of 128 fp32 logits 6.5 us, of which the bytes
// (8.4 MB) are 1.6 and a launch about 2; 16,384 tokens 9.5 us.
struct RouteGradArgs {
  const void* logits;
  int64_t T, stride;
  int32_t E, k, sigmoid, renorm;
  float scale;
  const int32_t* ids;
  const float* weights;
  const float* d_weights;
  void* d_logits;
  int32_t* status;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(RouteGradArgs a) {
  constexpr int kTok = kThreads / 64;
  extern __shared__ float terms[];
  const int E = a.E, k = a.k, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int64_t t = block_index() * kTok + wave;
  float* mine = terms + wave * E;
  const bool live = t < a.T;
  const T* row = (const T*)a.logits + (live ? t : a.T - 1) * a.stride;
  for (int e = lane; e < E; e += 64) mine[e] = 0.0f;
  __syncthreads();
  float dot = 0.0f;
  for (int j = lane; j < k && live; j += 64) {
    const float w = a.weights[t * k + j], d = a.d_weights[t * k + j];
    dot += w == 0.0f ? 0.0f : w * d;   // a weight of 0 passes nothing on, infinities and NaN neither
  }
  dot = across<64>(dot, [](float p, float q) { return p + q; });
  for (int j = lane; j < k && live; j += 64) {
    const int id = a.ids[t * k + j];
    if (id < 0 || id >= E) {
      report(a.status, VP_ERR_INVALID_ARGUMENT);
      continue;
    }
    const float w = a.weights[t * k + j];
    float g = w == 0.0f ? 0.0f : w * (a.renorm ? a.d_weights[t * k + j] - dot / a.scale : a.d_weights[t * k + j]);
    if (a.sigmoid && w != 0.0f) g *= sigmoid(-to_f32(row[id]));
    mine[id] = g;
  }
  __syncthreads();
  if (!live) return;
  T* out = (T*)a.d_logits + t * E;
  if (a.sigmoid || a.renorm) {
    for (int e = lane; e < E; e += 64) out[e] = from_f32<T>(mine[e]);
    return;
  }
  float top = -INFINITY, sum = 0.0f;
  for (int e = lane; e < E; e += 64) top = fmaxf(top, to_f32(row[e]));
  top = across<64>(top, [](float p, float q) { return fmaxf(p, q); });
  if (top == -INFINITY) {   // every expert masked: all weights are 0
    for (int e = lane; e < E; e += 64) out[e] = from_f32<T>(0.0f);
    return;
  }
  for (int e = lane; e < E; e += 64) sum += expf(to_f32(row[e]) - top);
  sum = across<64>(sum, [](float p, float q) { return p + q; });
  const float part = dot / sum;
  for (int e = lane; e < E; e += 64) out[e] = from_f32<T>(mine[e] - expf(to_f32(row[e]) - top) * part);
}

// First row of every local expert of rank `self` in the expert-major output:
// the running sums over the experts of the sources' counts.  One workgroup;
// at most 4,096 counts of each source, E of them read: 3.8 us for 16 ranks of
// 8 experts, 6.0 for 4,096 experts of one, latency of a load and a scan.
constexpr int kOffsetThreads = 1024;
__global__ void __launch_bounds__(kOffsetThreads) offsets_kernel(const int32_t* counts, int N, int E, int self,
                                                                 int64_t* offsets, int32_t* status) {
  extern __shared__ int64_t sums[];
  __shared__ int64_t part[kOffsetThreads];
  const int L = E / N, tid = threadIdx.x;
  for (int m = tid; m < L; m += kOffsetThreads) sums[m] = 0;
  __syncthreads();
  for (int i = tid; i < N * L; i += kOffsetThreads) {
    const int src = i / L, m = i - src * L;
    const int c = counts[(int64_t)src * E + (int64_t)self * L + m];
    if (c < 0) report(status, VP_ERR_INVALID_ARGUMENT);
    atomicAdd((unsigned long long*)&sums[m], (unsigned long long)(int64_t)c);   // whole numbers: any order
  }
  __syncthreads();
  // each thread a run of experts, then a scan over the threads' totals
  const int run = (L + kOffsetThreads - 1) / kOffsetThreads, m0 = min(tid * run, L), m1 = min(m0 + run, L);
  int64_t s = 0;
  for (int m = m0; m < m1; ++m) s += sums[m];
  part[tid] = s;
  __syncthreads();
  for (int d = 1; d < kOffsetThreads; d <<= 1) {
    const int64_t add = tid >= d ? part[tid - d] : 0;
    __syncthreads();
    part[tid] += add;
    __syncthreads();
  }
  int64_t at = part[tid] - s;
  for (int m = m0; m < m1; ++m) {
    offsets[m] = at;
    at += sums[m];
  }
  if (tid == kOffsetThreads - 1) offsets[L] = part[tid];
}

}  // namespace

// Lanes that share a token.  A wavefront per token against sixteen lanes, us: 96 tokens of 256 experts 5.2 / 7.7, 4096
// 7.5 / 8.2, 8192 11.3 / 9.3; of 128 experts 2048 5.3 / 5.3, 4096 7.2 / 5.4.
int32_t route_lanes(int64_t T, int32_t E) { return E > 256 || T <= (E <= 128 ? 2048 : 4096) ? 64 : 16; }

namespace {

template <typename T> void launch_route_as(const RouteArgs& a, hipStream_t s) {
  const auto go = [&](auto kernel, int lpt, int threads) {
    const int tok = threads / lpt;
    const size_t lds = 4 * (size_t)tok * (a.k + 1 + (a.n_groups > 1 ? a.E + 1 + 2 * a.n_groups : 0));
    hipLaunchKernelGGL(kernel, grid_of((a.T + tok - 1) / tok), dim3(threads), lds, s, a);
  };
  const bool few = route_lanes(a.T, a.E) == 64;
  if (few && a.E <= 64) go(route_kernel<T, 64, 1>, 64, kThreads);
  else if (few && a.E <= 256) go(route_kernel<T, 64, 4>, 64, kThreads);
  else if (a.E <= 64) go(route_kernel<T, 16, 4>, 16, kThreads);
  else if (a.E <= 128) go(route_kernel<T, 16, 8>, 16, kThreads);
  else if (a.E <= 256) go(route_kernel<T, 16, 16>, 16, kThreads);
  else if (a.E <= 1024) go(route_kernel<T, 64, 16>, 64, kThreads);
  else go(route_kernel<T, 64, 64>, 64, 64);   // one token: its keys take 16 KB of LDS
}

}  // namespace

vp_status launch_route(const void* logits, int32_t dtype, int64_t T, int32_t E, int64_t stride,
                       const vp_route_params& p, const float* bias, int32_t* ids, float* weights, void* stream) {
  const RouteArgs a{logits, T, stride, E, p.top_k, p.score == VP_SCORE_SIGMOID, p.n_groups, p.top_groups, p.group_top,
                    p.renorm, p.scale, bias, ids, weights};
  if (T > 0) {
    if (dtype == VP_F32) launch_route_as<float>(a, (hipStream_t)stream);
    else if (dtype == VP_BF16) launch_route_as<Bf16>(a, (hipStream_t)stream);
    else launch_route_as<F16>(a, (hipStream_t)stream);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "route launch failed");
  return VP_OK;
}

vp_status launch_route_grad(const void* logits, int32_t dtype, int64_t T, int32_t E, int64_t stride,
                            const vp_route_params& p, const int32_t* ids, const float* weights,
                            const float* d_weights, void* d_logits, int32_t* status, void* stream) {
  const RouteGradArgs a{logits, T, stride, E, p.top_k, p.score == VP_SCORE_SIGMOID, p.renorm, p.scale, ids, weights,
                        d_weights, d_logits, status};
  if (T > 0) {
    const dim3 grid = grid_of((T + kThreads / 64 - 1) / (kThreads / 64));
    const size_t lds = (size_t)(kThreads / 64) * E * 4;
    hipStream_t s = (hipStream_t)stream;
    if (dtype == VP_F32) hipLaunchKernelGGL(route_grad_kernel<float>, grid, dim3(kThreads), lds, s, a);
    else if (dtype == VP_BF16) hipLaunchKernelGGL(route_grad_kernel<Bf16>, grid, dim3(kThreads), lds, s, a);
    else hipLaunchKernelGGL(route_grad_kernel<F16>, grid, dim3(kThreads), lds, s, a);
  }
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "route gradient launch failed");
  return VP_OK;
}

vp_status launch_expert_offsets(const int32_t* counts, int32_t N, int32_t E, int32_t self, int64_t* offsets,
                                int32_t* status, void* stream) {
  hipLaunchKernelGGL(offsets_kernel, dim3(1), dim3(kOffsetThreads), (size_t)(E / N) * 8, (hipStream_t)stream, counts,
                     N, E, self, offsets, status);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "offsets launch failed");
  return VP_OK;
}

vp_status take_unclaimed_route(int32_t* out, void* stream) {
  hipLaunchKernelGGL(take_unclaimed_kernel, dim3(1), dim3(1), 0, (hipStream_t)stream, out);
  if (hipGetLastError() != hipSuccess) return set_error(VP_ERR_HIP, "status launch failed");
  return VP_OK;
}

}  // namespace vp
