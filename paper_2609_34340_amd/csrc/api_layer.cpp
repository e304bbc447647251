// C-ABI entry points of the layer operators: argument checks.
#include <cmath>

#include "internal.h"

using vp::set_error;

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 31, kMaxStride = int64_t(1) << 22;
constexpr int32_t kMaxExperts = 4096, kMaxTopK = 64, kMaxGroups = 64, kMaxWidth = 1 << 20;

bool is_float(int32_t d) { return d == VP_F32 || d == VP_BF16 || d == VP_F16; }
bool is_half(int32_t d) { return d == VP_BF16 || d == VP_F16; }
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
// Rows of `width` bytes, `stride` apart, moved in 16-byte vectors.
bool vector_rows(const void* p, int64_t width, int64_t stride) {
  return aligned(p) && width % 16 == 0 && stride % 16 == 0 && stride >= width;
}

vp_status check_route(int32_t dtype, int64_t T, int32_t E, int64_t stride, const vp_route_params* p) {
  if (!p) return set_error(VP_ERR_INVALID_ARGUMENT, "null route parameters");
  if (!is_float(dtype)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown element type");
  if (T < 0 || E < 1 || stride < E || p->top_k < 1 || p->top_k > E)
    return set_error(VP_ERR_INVALID_ARGUMENT, "bad routing sizes");
  if (p->score != VP_SCORE_SOFTMAX && p->score != VP_SCORE_SIGMOID)
    return set_error(VP_ERR_INVALID_ARGUMENT, "unknown score");
  if (p->n_groups < 1 || E % p->n_groups != 0 || p->top_groups < 1 || p->top_groups > p->n_groups ||
      (p->group_top != 1 && p->group_top != 2) || (p->renorm != 0 && p->renorm != 1))
    return set_error(VP_ERR_INVALID_ARGUMENT, "bad routing groups");
  if (p->top_k > p->top_groups * (E / p->n_groups))
    return set_error(VP_ERR_INVALID_ARGUMENT, "the kept groups hold fewer than top_k experts");
  if (!(p->scale > 0.0f) || !std::isfinite(p->scale))
    return set_error(VP_ERR_INVALID_ARGUMENT, "scale must be positive and finite");
  if (E > kMaxExperts || p->top_k > kMaxTopK || p->n_groups > kMaxGroups || T * p->top_k >= kMaxRows || T >= kMaxRows)
    return set_error(VP_ERR_UNSUPPORTED, "more than 4096 experts, top 64, 64 groups or 2^31 assignments");
  return VP_OK;
}

vp_status check_experts(int32_t dtype, const int64_t* offsets, int64_t R, int32_t L, int32_t N, int32_t K) {
  if (!is_half(dtype)) return set_error(VP_ERR_INVALID_ARGUMENT, "the experts' rows are bf16 or fp16");
  if (R < 0 || L < 1 || N < 1 || K < 1) return set_error(VP_ERR_INVALID_ARGUMENT, "bad product sizes");
  if (!offsets) return set_error(VP_ERR_INVALID_ARGUMENT, "null pointer");
  if (N % 8 != 0 || K % 8 != 0) return set_error(VP_ERR_UNSUPPORTED, "N and K must be multiples of 8");
  if (R >= kMaxRows || L > kMaxExperts || N > kMaxWidth || K > kMaxWidth)
    return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 rows, 4096 experts or 2^20 columns");
  return VP_OK;
}

// A tile of a gated product spans both halves of an expert's weights.
vp_status check_gated(int32_t gated, int32_t N, int64_t row_bytes) {
  if (gated != 0 && gated != 1) return set_error(VP_ERR_INVALID_ARGUMENT, "gated is 0 or 1");
  if (gated && N % 16 != 0) return set_error(VP_ERR_UNSUPPORTED, "a gated product's N must be a multiple of 16");
  if (gated && ((int64_t)N / 2 + 256) * row_bytes >= int64_t(1) << 30)
    return set_error(VP_ERR_UNSUPPORTED, "half of a gated expert's weights must be below 1 GiB");
  return VP_OK;
}

// `width` bytes of each row, moved in 16-byte vectors.
vp_status check_rows(const void* p, int64_t width, int64_t stride, int64_t R, const char* name) {
  if (R > 0 && !p) return set_error(VP_ERR_INVALID_ARGUMENT, std::string("null ") + name);
  if (!vector_rows(p, width, stride))
    return set_error(VP_ERR_INVALID_ARGUMENT, std::string(name) + ": rows must be 16-byte vectors, aligned, within the stride");
  return VP_OK;
}

// Of a product, whose tiles address their rows by 32-bit offsets.
vp_status check_operand(const void* p, int64_t width, int64_t stride, int64_t R, const char* name) {
  const vp_status st = check_rows(p, width, stride, R, name);
  if (st != VP_OK) return st;
  if (stride > kMaxStride) return set_error(VP_ERR_UNSUPPORTED, std::string(name) + ": stride above 4 MiB");
  return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_route(const void* logits, int32_t dtype, int64_t T, int32_t E, int64_t logits_stride,
                   const vp_route_params* p, const float* bias, int32_t* ids, float* weights, void* stream) {
  vp_status st = check_route(dtype, T, E, logits_stride, p);
  if (st != VP_OK) return st;
  if (T > 0 && (!logits || !ids || !weights)) return set_error(VP_ERR_INVALID_ARGUMENT, "null pointer");
  if (T == 0) return VP_OK;
  return vp::launch_route(logits, dtype, T, E, logits_stride, *p, bias, ids, weights, stream);
}

vp_status vp_route_grad(const void* logits, int32_t dtype, int64_t T, int32_t E, int64_t logits_stride,
                        const vp_route_params* p, const int32_t* ids, const float* weights, const float* d_weights,
                        void* d_logits, int32_t* dev_status, void* stream) {
  vp_status st = check_route(dtype, T, E, logits_stride, p);
  if (st != VP_OK) return st;
  if (T > 0 && (!logits || !ids || !weights || !d_weights || !d_logits))
    return set_error(VP_ERR_INVALID_ARGUMENT, "null pointer");
  if (T == 0) return VP_OK;
  return vp::launch_route_grad(logits, dtype, T, E, logits_stride, *p, ids, weights, d_weights, d_logits, dev_status,
                               stream);
}

vp_status vp_expert_offsets(const int32_t* counts, int32_t n_ranks, int32_t E, int32_t self_rank, int64_t* offsets,
                            int32_t* dev_status, void* stream) {
  if (n_ranks < 1 || n_ranks > vp::kMaxRanks || E < 1 || E % n_ranks != 0 || E > kMaxExperts || self_rank < 0 ||
      self_rank >= n_ranks)
    return set_error(VP_ERR_INVALID_ARGUMENT, "bad offsets sizes (E a multiple of N, <= 4096)");
  if (!counts || !offsets) return set_error(VP_ERR_INVALID_ARGUMENT, "null pointer");
  return vp::launch_expert_offsets(counts, n_ranks, E, self_rank, offsets, dev_status, stream);
}

vp_status vp_expert_matmul(const void* x, int64_t x_stride, int32_t dtype, const void* w, const int64_t* offsets,
                           int64_t R, int32_t L, int32_t N, int32_t K, int32_t gated, void* y, int64_t y_stride,
                           void* pre, int64_t pre_stride, int32_t* dev_status, void* stream) {
  vp_status st = check_experts(dtype, offsets, R, L, N, K);
  if (st != VP_OK) return st;
  if ((st = check_gated(gated, N, (int64_t)K * 2)) != VP_OK) return st;
  if (!gated && pre) return set_error(VP_ERR_INVALID_ARGUMENT, "pre belongs to a gated product");
  if ((st = check_operand(x, (int64_t)K * 2, x_stride, R, "x")) != VP_OK) return st;
  if ((st = check_operand(w, (int64_t)K * 2, (int64_t)K * 2, 1, "w")) != VP_OK) return st;
  if ((st = check_operand(y, (int64_t)(gated ? N / 2 : N) * 2, y_stride, R, "y")) != VP_OK) return st;
  if (pre && (st = check_operand(pre, (int64_t)N * 2, pre_stride, R, "pre")) != VP_OK) return st;
  if (R == 0) return VP_OK;
  const vp::ExpertLaunch a{vp::kExpertForward, gated != 0, false, dtype, x, w, x_stride, (int64_t)K * 2, offsets, R, L,
                           N, K, y, pre, y_stride, pre_stride, dev_status};
  return vp::launch_expert_product(a, stream);
}

vp_status vp_expert_matmul_grad_x(const void* dy, int64_t dy_stride, int32_t dtype, const void* w,
                                  const int64_t* offsets, int64_t R, int32_t L, int32_t N, int32_t K, void* dx,
                                  int64_t dx_stride, int32_t* dev_status, void* stream) {
  vp_status st = check_experts(dtype, offsets, R, L, N, K);
  if (st != VP_OK) return st;
  if ((st = check_operand(dy, (int64_t)N * 2, dy_stride, R, "dy")) != VP_OK) return st;
  if ((st = check_operand(w, (int64_t)K * 2, (int64_t)K * 2, 1, "w")) != VP_OK) return st;
  if ((st = check_operand(dx, (int64_t)K * 2, dx_stride, R, "dx")) != VP_OK) return st;
  if (R == 0) return VP_OK;
  const vp::ExpertLaunch a{vp::kExpertGradX, false, false, dtype, dy, w, dy_stride, (int64_t)K * 2, offsets, R, L, N, K,
                           dx, nullptr, dx_stride, 0, dev_status};
  return vp::launch_expert_product(a, stream);
}

vp_status vp_expert_matmul_grad_w(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int32_t dtype,
                                  const int64_t* offsets, int64_t R, int32_t L, int32_t N, int32_t K, float* dw,
                                  int32_t* dev_status, void* stream) {
  vp_status st = check_experts(dtype, offsets, R, L, N, K);
  if (st != VP_OK) return st;
  if ((st = check_operand(dy, (int64_t)N * 2, dy_stride, R, "dy")) != VP_OK) return st;
  if ((st = check_operand(x, (int64_t)K * 2, x_stride, R, "x")) != VP_OK) return st;
  if ((st = check_operand(dw, (int64_t)K * 4, (int64_t)K * 4, 1, "dw")) != VP_OK) return st;
  const vp::ExpertLaunch a{vp::kExpertGradW, false, false, dtype, dy, x, dy_stride, x_stride, offsets, R, L, N, K, dw,
                           nullptr, (int64_t)K * 4, 0, dev_status};
  return vp::launch_expert_product(a, stream);
}

vp_status vp_expert_gate_grad(const void* dh, int64_t dh_stride, const void* pre, int64_t pre_stride, int32_t dtype,
                              const int64_t* offsets, int64_t R, int32_t L, int32_t I, void* dpre,
                              int64_t dpre_stride, int32_t* dev_status, void* stream) {
  vp_status st = check_experts(dtype, offsets, R, L, I, 8);
  if (st != VP_OK) return st;
  if ((st = check_rows(dh, (int64_t)I * 2, dh_stride, R, "dh")) != VP_OK) return st;
  if ((st = check_rows(pre, (int64_t)I * 4, pre_stride, R, "pre")) != VP_OK) return st;
  if ((st = check_rows(dpre, (int64_t)I * 4, dpre_stride, R, "dpre")) != VP_OK) return st;
  if (R == 0) return VP_OK;
  return vp::launch_expert_gate_grad(dh, dh_stride, pre, pre_stride, dtype, R, I, offsets, L, dpre, dpre_stride,
                                     dev_status, stream);
}

namespace {

vp_status check_merge(int32_t dtype, int64_t T, int32_t k, int64_t H, const float* weights) {
  if (!is_float(dtype)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown element type");
  if (T < 0 || k < 1 || k > 255 || H < 1) return set_error(VP_ERR_INVALID_ARGUMENT, "bad merge sizes (k <= 255)");
  if (T > 0 && !weights) return set_error(VP_ERR_INVALID_ARGUMENT, "null weights");
  if (T >= kMaxRows || H > kMaxWidth) return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 tokens or 2^20 columns");
  return VP_OK;
}

}  // namespace

vp_status vp_merge(const void* rows, int32_t dtype, int64_t T, int32_t k, int64_t H, int64_t row_stride,
                   const float* weights, const void* residual, int64_t residual_stride, void* out, int64_t out_stride,
                   void* stream) {
  vp_status st = check_merge(dtype, T, k, H, weights);
  if (st != VP_OK) return st;
  const int64_t width = H * vp::dtype_size(dtype);
  if ((st = check_rows(rows, width, row_stride, T, "rows")) != VP_OK) return st;
  if ((st = check_rows(out, width, out_stride, T, "out")) != VP_OK) return st;
  if (residual && (st = check_rows(residual, width, residual_stride, T, "residual")) != VP_OK) return st;
  if (T == 0) return VP_OK;
  return vp::launch_merge(rows, dtype, T, k, H, row_stride, weights, residual, residual_stride, out, out_stride,
                          stream);
}

vp_status vp_merge_grad(const void* d_out, int32_t dtype, int64_t T, int32_t k, int64_t H, int64_t d_out_stride,
                        const void* rows, int64_t row_stride, const float* weights, void* d_rows,
                        int64_t d_rows_stride, float* d_weights, void* stream) {
  vp_status st = check_merge(dtype, T, k, H, weights);
  if (st != VP_OK) return st;
  const int64_t width = H * vp::dtype_size(dtype);
  if ((st = check_rows(d_out, width, d_out_stride, T, "d_out")) != VP_OK) return st;
  if ((st = check_rows(rows, width, row_stride, T, "rows")) != VP_OK) return st;
  if ((st = check_rows(d_rows, width, d_rows_stride, T, "d_rows")) != VP_OK) return st;
  if (T > 0 && !d_weights) return set_error(VP_ERR_INVALID_ARGUMENT, "null d_weights");
  if (T == 0) return VP_OK;
  return vp::launch_merge_grad(d_out, dtype, T, k, H, d_out_stride, rows, row_stride, weights, d_rows, d_rows_stride,
                               d_weights, stream);
}

int64_t vp_mx_row_bytes(int64_t K) { return K < 32 || K % 32 != 0 ? 0 : vp::mx_row_bytes(K); }

namespace {

vp_status check_mx(int32_t dtype, int64_t rows, int64_t K) {
  if (!is_float(dtype)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown element type");
  if (rows < 0 || K < 1) return set_error(VP_ERR_INVALID_ARGUMENT, "bad block sizes");
  if (K % 32 != 0 || K > kMaxWidth || rows >= kMaxRows)
    return set_error(VP_ERR_UNSUPPORTED, "K must be a multiple of 32 up to 2^20, rows below 2^31");
  return VP_OK;
}

}  // namespace

vp_status vp_mx_quantize(const void* x, int32_t dtype, int64_t rows, int64_t K, int64_t x_stride, void* q,
                         int64_t q_stride, void* stream) {
  vp_status st = check_mx(dtype, rows, K);
  if (st != VP_OK) return st;
  if ((st = check_rows(x, K * vp::dtype_size(dtype), x_stride, rows, "x")) != VP_OK) return st;
  if ((st = check_rows(q, vp::mx_row_bytes(K), q_stride, rows, "q")) != VP_OK) return st;
  if (rows == 0) return VP_OK;
  return vp::launch_mx_quantize(x, dtype, rows, K, x_stride, q, q_stride, stream);
}

vp_status vp_mx_dequantize(const void* q, int64_t rows, int64_t K, int64_t q_stride, void* out, int32_t dtype,
                           int64_t out_stride, void* stream) {
  vp_status st = check_mx(dtype, rows, K);
  if (st != VP_OK) return st;
  if ((st = check_rows(q, vp::mx_row_bytes(K), q_stride, rows, "q")) != VP_OK) return st;
  if ((st = check_rows(out, K * vp::dtype_size(dtype), out_stride, rows, "out")) != VP_OK) return st;
  if (rows == 0) return VP_OK;
  return vp::launch_mx_dequantize(q, rows, K, q_stride, out, dtype, out_stride, stream);
}

vp_status vp_expert_matmul_mx(const void* xq, int64_t xq_stride, const void* wq, const int64_t* offsets, int64_t R,
                              int32_t L, int32_t N, int32_t K, int32_t gated, void* y, int32_t dtype,
                              int64_t y_stride, int32_t* dev_status, void* stream) {
  vp_status st = check_experts(dtype, offsets, R, L, N, K);
  if (st != VP_OK) return st;
  if (K % 32 != 0) return set_error(VP_ERR_UNSUPPORTED, "K must be a multiple of 32");
  const int64_t rb = vp::mx_row_bytes(K);
  if ((st = check_gated(gated, N, rb)) != VP_OK) return st;
  if ((st = check_operand(xq, rb, xq_stride, R, "xq")) != VP_OK) return st;
  if ((st = check_operand(wq, rb, rb, 1, "wq")) != VP_OK) return st;
  if ((st = check_operand(y, (int64_t)(gated ? N / 2 : N) * 2, y_stride, R, "y")) != VP_OK) return st;
  if (R == 0) return VP_OK;
  const vp::ExpertLaunch a{vp::kExpertForward, gated != 0, true, dtype, xq, wq, xq_stride, rb, offsets, R, L, N, K, y,
                           nullptr, y_stride, 0, dev_status};
  return vp::launch_expert_product(a, stream);
}

vp_status vp_take_status(int32_t* dev_status, void* stream) {
  if (!dev_status) return set_error(VP_ERR_INVALID_ARGUMENT, "null pointer");
  const vp_status st = vp::take_unclaimed_route(dev_status, stream);
  return st != VP_OK ? st : vp::take_unclaimed_experts(dev_status, stream);
}

int32_t vp_expert_kernel(int32_t direction, int32_t mx, int32_t gated, int64_t R, int32_t L, int32_t N, int32_t K) {
  static const int64_t some_offsets = 0;   // only for the check
  if (direction < 0 || direction > 2 || (mx != 0 && mx != 1) || (gated != 0 && gated != 1)) return -1;
  if (direction != vp::kExpertForward && (mx || gated)) return -1;
  if (check_experts(VP_BF16, &some_offsets, R, L, N, K) != VP_OK || (mx && K % 32 != 0)) return -1;
  const int64_t w_row = mx ? vp::mx_row_bytes(K) : (int64_t)K * 2;
  if (check_gated(gated, N, w_row) != VP_OK) return -1;
  vp::ExpertLaunch a{};
  a.mode = direction;
  a.gated = gated != 0;
  a.mx = mx != 0;
  a.dtype = VP_BF16;
  a.b_stride = w_row;
  a.R = R;
  a.L = L;
  a.N = N;
  a.K = K;
  return vp::expert_kind(a);
}

int32_t vp_route_lanes(int64_t T, int32_t E) {
  return T < 0 || E < 1 || E > kMaxExperts ? -1 : vp::route_lanes(T, E);
}

}  // extern "C"
