// C-ABI entry points of norm, dropout and the dense products: argument checks.
#include <cmath>

#include "internal.h"

using vp::set_error;

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 31, kMaxStride = int64_t(1) << 22;
constexpr int64_t kMaxWidth = 1 << 20;

bool is_float(int32_t d) { return d == VP_F32 || d == VP_BF16 || d == VP_F16; }
bool is_half(int32_t d) { return d == VP_BF16 || d == VP_F16; }
bool is_act(int32_t a) { return a >= VP_ACT_NONE && a <= VP_ACT_GELU_TANH; }

vp_status check_sizes(int32_t dtype, int64_t T, int64_t H) {
  if (!is_float(dtype)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown element type");
  if (T < 0 || H < 1) return set_error(VP_ERR_INVALID_ARGUMENT, "bad sizes");
  if (T >= kMaxRows || H > kMaxWidth) return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 rows or 2^20 columns");
  return VP_OK;
}

// `width` bytes of each of T rows, in multiples of `unit`.
vp_status check_rows(const void* p, int64_t width, int64_t stride, int64_t unit, int64_t T, const char* name) {
  if (T > 0 && !p) return set_error(VP_ERR_INVALID_ARGUMENT, std::string("null ") + name);
  if ((uintptr_t)p % unit != 0 || stride % unit != 0 || stride < width)
    return set_error(VP_ERR_INVALID_ARGUMENT, std::string(name) + ": rows must be aligned and within the stride");
  return VP_OK;
}

vp_status check_vector(const void* p, int32_t type, int32_t dtype, const char* name) {
  if (!p) return VP_OK;
  if (type != VP_F32 && type != dtype)
    return set_error(VP_ERR_INVALID_ARGUMENT, std::string(name) + " must be fp32 or of the rows' type");
  if ((uintptr_t)p % vp::dtype_size(type) != 0)
    return set_error(VP_ERR_INVALID_ARGUMENT, std::string(name) + " must be aligned");
  return VP_OK;
}

vp_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return VP_OK;
  if (!ws || ((uintptr_t)ws & 15) != 0) return set_error(VP_ERR_INVALID_ARGUMENT, "workspace missing or unaligned");
  if (have < need) return set_error(VP_ERR_INVALID_ARGUMENT, "workspace too small");
  return VP_OK;
}

vp_status check_product(int32_t dtype, int64_t R, int32_t N, int32_t K) {
  if (!is_half(dtype)) return set_error(VP_ERR_INVALID_ARGUMENT, "dense products take bf16 or fp16");
  if (R < 0 || N < 1 || K < 1) return set_error(VP_ERR_INVALID_ARGUMENT, "bad product sizes");
  if (N % 8 != 0 || K % 8 != 0) return set_error(VP_ERR_UNSUPPORTED, "N and K must be multiples of 8");
  if (R >= kMaxRows || N > kMaxWidth || K > kMaxWidth)
    return set_error(VP_ERR_UNSUPPORTED, "more than 2^31 rows or 2^20 columns");
  return VP_OK;
}

// Of a product: 16-byte vectors, whose tiles address them by 32-bit offsets.
vp_status check_operand(const void* p, int64_t width, int64_t stride, int64_t R, const char* name) {
  const vp_status st = check_rows(p, width, stride, 16, R, name);
  if (st != VP_OK) return st;
  if (stride > kMaxStride) return set_error(VP_ERR_UNSUPPORTED, std::string(name) + ": stride above 4 MiB");
  return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_layer_norm(const void* x, int32_t dtype, int64_t T, int64_t H, int64_t x_stride, const void* weight,
                        const void* bias, int32_t param_dtype, float eps, int32_t center, void* y, int64_t y_stride,
                        float* stats, void* stream) {
  vp_status st = check_sizes(dtype, T, H);
  if (st != VP_OK) return st;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(VP_ERR_INVALID_ARGUMENT, "eps must be finite and not negative");
  if (center != 0 && center != 1) return set_error(VP_ERR_INVALID_ARGUMENT, "center is 0 or 1");
  const int64_t size = vp::dtype_size(dtype);
  if ((st = check_rows(x, H * size, x_stride, size, T, "x")) != VP_OK) return st;
  if ((st = check_rows(y, H * size, y_stride, size, T, "y")) != VP_OK) return st;
  if ((st = check_vector(weight, param_dtype, dtype, "weight")) != VP_OK) return st;
  if ((st = check_vector(bias, param_dtype, dtype, "bias")) != VP_OK) return st;
  if ((st = check_vector(stats, VP_F32, dtype, "stats")) != VP_OK) return st;
  if (T == 0) return VP_OK;
  vp::NormLaunch a{};
  a.dtype = dtype;
  a.param_dtype = param_dtype;
  a.center = center != 0;
  a.T = T;
  a.H = H;
  a.x = x;
  a.x_stride = x_stride;
  a.weight = weight;
  a.bias = bias;
  a.eps = eps;
  a.out = y;
  a.out_stride = y_stride;
  a.stats = stats;
  return vp::launch_layer_norm(a, stream);
}

size_t vp_layer_norm_grad_workspace(int64_t T, int64_t H) {
  return check_sizes(VP_F32, T, H) != VP_OK ? 0 : vp::layer_norm_grad_workspace(T, H);
}

vp_status vp_layer_norm_grad(const void* d_out, int64_t d_out_stride, const void* x, int64_t x_stride, int32_t dtype,
                             int64_t T, int64_t H, const float* stats, const void* weight, int32_t param_dtype,
                             int32_t center, const void* residual, int64_t residual_stride, void* d_x,
                             int64_t d_x_stride, float* d_weight, float* d_bias, void* ws, size_t ws_bytes,
                             void* stream) {
  vp_status st = check_sizes(dtype, T, H);
  if (st != VP_OK) return st;
  if (center != 0 && center != 1) return set_error(VP_ERR_INVALID_ARGUMENT, "center is 0 or 1");
  const int64_t size = vp::dtype_size(dtype);
  if ((st = check_rows(d_out, H * size, d_out_stride, size, T, "d_out")) != VP_OK) return st;
  if ((st = check_rows(x, H * size, x_stride, size, T, "x")) != VP_OK) return st;
  if ((st = check_rows(d_x, H * size, d_x_stride, size, T, "d_x")) != VP_OK) return st;
  if (residual && (st = check_rows(residual, H * size, residual_stride, size, T, "residual")) != VP_OK) return st;
  if (T > 0 && !stats) return set_error(VP_ERR_INVALID_ARGUMENT, "null stats");
  if ((st = check_vector(stats, VP_F32, dtype, "stats")) != VP_OK) return st;
  if ((st = check_vector(weight, param_dtype, dtype, "weight")) != VP_OK) return st;
  if ((st = check_vector(d_weight, VP_F32, dtype, "d_weight")) != VP_OK) return st;
  if ((st = check_vector(d_bias, VP_F32, dtype, "d_bias")) != VP_OK) return st;
  if (d_weight || d_bias) {
    if ((st = check_workspace(ws, ws_bytes, vp::layer_norm_grad_workspace(T, H))) != VP_OK) return st;
  }
  vp::NormLaunch a{};
  a.dtype = dtype;
  a.param_dtype = param_dtype;
  a.center = center != 0;
  a.T = T;
  a.H = H;
  a.d_out = d_out;
  a.d_out_stride = d_out_stride;
  a.x = x;
  a.x_stride = x_stride;
  a.given = stats;
  a.weight = weight;
  a.residual = residual;
  a.residual_stride = residual_stride;
  a.out = d_x;
  a.out_stride = d_x_stride;
  a.d_weight = d_weight;
  a.d_bias = d_bias;
  a.ws = ws;
  return vp::launch_layer_norm_grad(a, stream);
}

vp_status vp_dropout(const void* x, int32_t dtype, int64_t T, int64_t H, int64_t x_stride, double p, uint64_t seed,
                     const int64_t* step, const void* residual, int64_t residual_stride, void* out,
                     int64_t out_stride, void* stream) {
  vp_status st = check_sizes(dtype, T, H);
  if (st != VP_OK) return st;
  if (!(p >= 0.0 && p <= 1.0)) return set_error(VP_ERR_INVALID_ARGUMENT, "p must be between 0 and 1");
  if ((uintptr_t)step % 8 != 0) return set_error(VP_ERR_INVALID_ARGUMENT, "step must be aligned");
  const int64_t size = vp::dtype_size(dtype);
  if ((st = check_rows(x, H * size, x_stride, size, T, "x")) != VP_OK) return st;
  if ((st = check_rows(out, H * size, out_stride, size, T, "out")) != VP_OK) return st;
  if (residual && (st = check_rows(residual, H * size, residual_stride, size, T, "residual")) != VP_OK) return st;
  if (T == 0) return VP_OK;
  return vp::launch_dropout(x, dtype, T, H, x_stride, (uint32_t)std::floor(p * 65536.0 + 0.5), seed, step, residual,
                            residual_stride, out, out_stride, stream);
}

size_t vp_linear_workspace(int32_t direction, int64_t R, int32_t N, int32_t K) {
  if (direction < vp::kExpertForward || direction > vp::kExpertGradW || check_product(VP_BF16, R, N, K) != VP_OK) return 0;
  return vp::linear_workspace(direction, R, N, K);
}

int32_t vp_linear_kernel(int32_t direction, int64_t R, int32_t N, int32_t K, int32_t* parts) {
  if (direction < vp::kExpertForward || direction > vp::kExpertGradW || check_product(VP_BF16, R, N, K) != VP_OK) return -1;
  return vp::linear_kind(direction, R, N, K, parts);
}

vp_status vp_linear(const void* x, int64_t x_stride, int32_t dtype, const void* w, int64_t w_stride, int64_t R,
                    int32_t N, int32_t K, const void* bias, int32_t bias_dtype, int32_t act, const void* residual,
                    int64_t residual_stride, void* y, int32_t out_dtype, int64_t y_stride, void* pre,
                    int64_t pre_stride, void* ws, size_t ws_bytes, void* stream) {
  vp_status st = check_product(dtype, R, N, K);
  if (st != VP_OK) return st;
  if (!is_act(act)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown activation");
  if (out_dtype != VP_F32 && out_dtype != dtype)
    return set_error(VP_ERR_INVALID_ARGUMENT, "results are fp32 or of the rows' type");
  const int64_t out = (int64_t)N * vp::dtype_size(out_dtype);
  if ((st = check_operand(x, (int64_t)K * 2, x_stride, R, "x")) != VP_OK) return st;
  if ((st = check_operand(w, (int64_t)K * 2, w_stride, N, "w")) != VP_OK) return st;
  if ((st = check_operand(y, out, y_stride, R, "y")) != VP_OK) return st;
  if (residual && (st = check_operand(residual, out, residual_stride, R, "residual")) != VP_OK) return st;
  if (pre && (st = check_operand(pre, (int64_t)N * 2, pre_stride, R, "pre")) != VP_OK) return st;
  if ((st = check_vector(bias, bias_dtype, dtype, "bias")) != VP_OK) return st;
  if (((uintptr_t)bias & 15) != 0) return set_error(VP_ERR_INVALID_ARGUMENT, "bias must be 16-byte aligned");
  if ((st = check_workspace(ws, ws_bytes, vp::linear_workspace(vp::kExpertForward, R, N, K))) != VP_OK) return st;
  if (R == 0) return VP_OK;
  vp::LinearLaunch a{};
  a.mode = vp::kExpertForward;
  a.dtype = dtype;
  a.bias_dtype = bias_dtype;
  a.out_dtype = out_dtype;
  a.act = act;
  a.a = x;
  a.a_stride = x_stride;
  a.b = w;
  a.b_stride = w_stride;
  a.R = R;
  a.N = N;
  a.K = K;
  a.bias = bias;
  a.residual = residual;
  a.residual_stride = residual_stride;
  a.out = y;
  a.out_stride = y_stride;
  a.pre = pre;
  a.pre_stride = pre_stride;
  a.ws = ws;
  return vp::launch_linear(a, stream);
}

size_t vp_linear_act_grad_workspace(int64_t R, int64_t N) {
  return check_sizes(VP_F32, R, N) != VP_OK ? 0 : vp::act_grad_workspace(R, N);
}

vp_status vp_linear_act_grad(const void* d_y, int64_t d_y_stride, const void* pre, int64_t pre_stride, int32_t dtype,
                             int64_t R, int64_t N, int32_t act, void* d_pre, int64_t d_pre_stride, float* d_bias,
                             void* ws, size_t ws_bytes, void* stream) {
  vp_status st = check_sizes(dtype, R, N);
  if (st != VP_OK) return st;
  if (!is_act(act)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown activation");
  if (!d_pre && !d_bias) return set_error(VP_ERR_INVALID_ARGUMENT, "neither d_pre nor d_bias");
  if (R > 0 && (act == VP_ACT_NONE) != (pre == nullptr))
    return set_error(VP_ERR_INVALID_ARGUMENT, "an activation's gradient needs pre, and only that does");
  const int64_t size = vp::dtype_size(dtype);
  if ((st = check_rows(d_y, N * size, d_y_stride, size, R, "d_y")) != VP_OK) return st;
  if (pre && (st = check_rows(pre, N * size, pre_stride, size, R, "pre")) != VP_OK) return st;
  if (d_pre && (st = check_rows(d_pre, N * size, d_pre_stride, size, R, "d_pre")) != VP_OK) return st;
  if ((st = check_vector(d_bias, VP_F32, dtype, "d_bias")) != VP_OK) return st;
  if (d_bias && (st = check_workspace(ws, ws_bytes, vp::act_grad_workspace(R, N))) != VP_OK) return st;
  if (R == 0 && !d_bias) return VP_OK;
  return vp::launch_act_grad(d_y, d_y_stride, pre, pre_stride, dtype, R, N, act, d_pre, d_pre_stride, d_bias, ws, stream);
}

vp_status vp_linear_grad_x(const void* d_y, int64_t d_y_stride, int32_t dtype, const void* w, int64_t w_stride,
                           int64_t R, int32_t N, int32_t K, int32_t act, const void* pre, int64_t pre_stride,
                           const void* residual, int64_t residual_stride, void* d_x, int64_t d_x_stride, void* ws,
                           size_t ws_bytes, void* stream) {
  vp_status st = check_product(dtype, R, N, K);
  if (st != VP_OK) return st;
  if (!is_act(act)) return set_error(VP_ERR_INVALID_ARGUMENT, "unknown activation");
  if (R > 0 && (act == VP_ACT_NONE) != (pre == nullptr))
    return set_error(VP_ERR_INVALID_ARGUMENT, "an activation's gradient needs pre, and only that does");
  if ((st = check_operand(d_y, (int64_t)N * 2, d_y_stride, R, "d_y")) != VP_OK) return st;
  if ((st = check_operand(w, (int64_t)K * 2, w_stride, N, "w")) != VP_OK) return st;
  if ((st = check_operand(d_x, (int64_t)K * 2, d_x_stride, R, "d_x")) != VP_OK) return st;
  if (pre && (st = check_operand(pre, (int64_t)K * 2, pre_stride, R, "pre")) != VP_OK) return st;
  if (residual && (st = check_operand(residual, (int64_t)K * 2, residual_stride, R, "residual")) != VP_OK) return st;
  if ((st = check_workspace(ws, ws_bytes, vp::linear_workspace(vp::kExpertGradX, R, N, K))) != VP_OK) return st;
  if (R == 0) return VP_OK;
  vp::LinearLaunch a{};
  a.mode = vp::kExpertGradX;
  a.dtype = a.out_dtype = dtype;
  a.act = act;
  a.a = d_y;
  a.a_stride = d_y_stride;
  a.b = w;
  a.b_stride = w_stride;
  a.R = R;
  a.N = N;
  a.K = K;
  a.slope = pre;
  a.slope_stride = pre_stride;
  a.residual = residual;
  a.residual_stride = residual_stride;
  a.out = d_x;
  a.out_stride = d_x_stride;
  a.ws = ws;
  return vp::launch_linear(a, stream);
}

vp_status vp_linear_grad_w(const void* d_y, int64_t d_y_stride, const void* x, int64_t x_stride, int32_t dtype,
                           int64_t R, int32_t N, int32_t K, float* d_w, void* ws, size_t ws_bytes, void* stream) {
  vp_status st = check_product(dtype, R, N, K);
  if (st != VP_OK) return st;
  if ((st = check_operand(d_y, (int64_t)N * 2, d_y_stride, R, "d_y")) != VP_OK) return st;
  if ((st = check_operand(x, (int64_t)K * 2, x_stride, R, "x")) != VP_OK) return st;
  if ((st = check_operand(d_w, (int64_t)K * 4, (int64_t)K * 4, 1, "d_w")) != VP_OK) return st;
  if ((st = check_workspace(ws, ws_bytes, vp::linear_workspace(vp::kExpertGradW, R, N, K))) != VP_OK) return st;
  vp::LinearLaunch a{};
  a.mode = vp::kExpertGradW;
  a.dtype = dtype;
  a.out_dtype = VP_F32;
  a.a = d_y;
  a.a_stride = d_y_stride;
  a.b = x;
  a.b_stride = x_stride;
  a.R = R;
  a.N = N;
  a.K = K;
  a.out = d_w;
  a.out_stride = (int64_t)K * 4;
  a.ws = ws;
  return vp::launch_linear(a, stream);
}

}  // extern "C"
