// C ABI of the operators around the linear backward: argument checks, workspace layouts and the launches
// behind each call.
#include "block_host.h"
#include "call_checks.h"

namespace hot {

namespace {

bool fn_ok(hot_act_fn f) { return f >= HOT_ACT_NONE && f <= HOT_ACT_SILU; }

size_t activation_sums_bytes(int64_t rows, int64_t cols) {
  return (size_t)activation_sum_rows(rows, cols) * round_up(cols, 32) * 4;
}
size_t norm_sums_bytes(int64_t rows, int64_t cols) {
  return (size_t)layer_norm_sum_rows(rows, cols, HOT_BF16) * 2 * round_up(cols, 32) * 4;
}

}  // namespace
}  // namespace hot

using namespace hot;

extern "C" {

size_t hot_checkpoint_bytes(int64_t rows, int64_t cols) { return size_ok(rows, cols) ? ckpt_layout(rows, cols).total : 0; }

hot_status hot_checkpoint_write(const void* x, hot_type type, int64_t rows, int64_t cols, void* ckpt, void* stream) {
  if (!x || !ckpt || !type_ok(type)) return HOT_ERR_ARG;
  if (!size_ok(rows, cols)) return HOT_ERR_SHAPE;
  Buffers b;
  b.in(x, bytes_of(type, rows, cols));
  b.out(ckpt, (int64_t)ckpt_layout(rows, cols).total);
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  HOT_STAGE(kStCkptWrite, launch_activation(HOT_ACT_NONE, x, type, rows, cols, nullptr, ckpt, s));
  return HOT_OK;
}

hot_status hot_checkpoint_read(const void* ckpt, int64_t rows, int64_t cols, void* x, hot_type type, void* stream) {
  if (!x || !ckpt || !type_ok(type)) return HOT_ERR_ARG;
  if (!size_ok(rows, cols)) return HOT_ERR_SHAPE;
  Buffers b;
  b.in(ckpt, (int64_t)ckpt_layout(rows, cols).total);
  b.out(x, bytes_of(type, rows, cols));
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  HOT_STAGE(kStCkptRead, launch_checkpoint_read(ckpt, rows, cols, x, type, s));
  return HOT_OK;
}

hot_status hot_activation_forward(hot_act_fn fn, const void* x, hot_type type, int64_t rows, int64_t cols, void* y,
                                  void* ckpt, void* stream) {
  if (!x || !y || !type_ok(type) || !fn_ok(fn) || fn == HOT_ACT_NONE) return HOT_ERR_ARG;
  if (!size_ok(rows, cols)) return HOT_ERR_SHAPE;
  Buffers b;
  b.in(x, bytes_of(type, rows, cols));
  b.out(y, bytes_of(type, rows, cols));
  b.out(ckpt, (int64_t)ckpt_layout(rows, cols).total);
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  HOT_STAGE(kStActForward, launch_activation(fn, x, type, rows, cols, y, ckpt, s));
  return HOT_OK;
}

size_t hot_activation_backward_workspace_bytes(int64_t rows, int64_t cols) {
  return size_ok(rows, cols) ? activation_sums_bytes(rows, cols) : 0;
}

hot_status hot_activation_backward(hot_act_fn fn, const void* g_y, hot_type type, const void* x, const void* ckpt,
                                   int64_t rows, int64_t cols, void* g_x, float* g_bias, void* ws, size_t ws_bytes,
                                   void* stream) {
  if (!g_y || !g_x || !type_ok(type) || !fn_ok(fn) || !x == !ckpt) return HOT_ERR_ARG;
  if (g_bias && (!ws || !aligned256(ws))) return HOT_ERR_ARG;
  if (!size_ok(rows, cols)) return HOT_ERR_SHAPE;
  const size_t need = g_bias ? activation_sums_bytes(rows, cols) : 0;
  Buffers b;
  b.in(g_y, bytes_of(type, rows, cols));
  b.in(x, bytes_of(type, rows, cols));
  b.in(ckpt, (int64_t)ckpt_layout(rows, cols).total);
  b.out(g_x, bytes_of(type, rows, cols));
  b.out(g_bias, cols * 4);
  if (g_bias) b.out(ws, (int64_t)need);
  if (!b.ok()) return HOT_ERR_ARG;
  if (g_bias && ws_bytes < need) return HOT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const int64_t pitch = round_up(cols, 32);
  const int sums = activation_sum_rows(rows, cols);
  float* const partials = !g_bias || sums == 1 ? g_bias : (float*)ws;
  HOT_STAGE(kStActBackward, launch_activation_grad(fn, g_y, type, x, ckpt, rows, cols, g_x, partials, pitch, s));
  if (partials != g_bias) HOT_STAGE(kStColumnSums, launch_column_sums(partials, sums, pitch, cols, g_bias, nullptr, s));
  return HOT_OK;
}

hot_status hot_layer_norm_forward(const void* x, hot_type x_type, const void* residual, const float* gamma,
                                  const float* beta, float eps, int64_t rows, int64_t cols, void* h, void* y,
                                  hot_type y_type, float* mean, float* rstd, void* ckpt, void* stream) {
  if (!x || !y || !mean || !rstd || !residual != !h || !type_ok(x_type) || !type_ok(y_type)) return HOT_ERR_ARG;
  if (x_type == HOT_BF16 && y_type != HOT_BF16) return HOT_ERR_ARG;
  if (!(eps >= 0.0f)) return HOT_ERR_ARG;
  if (!size_ok(rows, cols) || cols > kMaxNormCols) return HOT_ERR_SHAPE;
  Buffers b;
  b.in(x, bytes_of(x_type, rows, cols));
  b.in(residual, bytes_of(x_type, rows, cols));
  b.in(gamma, cols * 4);
  b.in(beta, cols * 4);
  b.out(h, bytes_of(x_type, rows, cols));
  b.out(y, bytes_of(y_type, rows, cols));
  b.out(mean, rows * 4);
  b.out(rstd, rows * 4);
  b.out(ckpt, (int64_t)ckpt_layout(rows, cols).total);
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  const NormForward a{x, residual, gamma, beta, eps, rows, cols, x_type, y_type, h, y, ckpt, mean, rstd};
  HOT_STAGE(kStNormForward, launch_layer_norm(a, s));
  return HOT_OK;
}

size_t hot_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
  return size_ok(rows, cols) && cols <= kMaxNormCols ? norm_sums_bytes(rows, cols) : 0;
}

hot_status hot_layer_norm_backward(const void* g_y, hot_type y_type, const void* h, const void* ckpt, hot_type x_type,
                                   const float* gamma, const float* mean, const float* rstd, const void* g_residual,
                                   int64_t rows, int64_t cols, void* g_x, float* g_gamma, float* g_beta, void* ws,
                                   size_t ws_bytes, void* stream) {
  if (!g_y || !mean || !rstd || !g_x || !h == !ckpt || !g_gamma != !g_beta) return HOT_ERR_ARG;
  if (!type_ok(x_type) || !type_ok(y_type) || (x_type == HOT_BF16 && y_type != HOT_BF16)) return HOT_ERR_ARG;
  if (g_gamma && (!ws || !aligned256(ws))) return HOT_ERR_ARG;
  if (!size_ok(rows, cols) || cols > kMaxNormCols) return HOT_ERR_SHAPE;
  const size_t need = g_gamma ? norm_sums_bytes(rows, cols) : 0;
  Buffers b;
  b.in(g_y, bytes_of(y_type, rows, cols));
  b.in(h, bytes_of(x_type, rows, cols));
  b.in(ckpt, (int64_t)ckpt_layout(rows, cols).total);
  b.in(gamma, cols * 4);
  b.in(mean, rows * 4);
  b.in(rstd, rows * 4);
  b.in(g_residual, bytes_of(x_type, rows, cols));
  b.out(g_x, bytes_of(x_type, rows, cols));
  b.out(g_gamma, cols * 4);
  b.out(g_beta, cols * 4);
  if (g_gamma) b.out(ws, (int64_t)need);
  if (!b.ok()) return HOT_ERR_ARG;
  if (g_gamma && ws_bytes < need) return HOT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const int64_t pitch = round_up(cols, 32);
  const int sums = layer_norm_sum_rows(rows, cols, x_type);
  const bool apart = g_gamma && sums > 1;
  NormBackward a{g_y, h, ckpt, g_residual, gamma, mean, rstd, rows, cols, x_type, y_type, g_x, g_gamma, g_beta, 0};
  if (apart) {
    a.sum_gamma = (float*)ws;
    a.sum_beta = a.sum_gamma + pitch;
    a.sum_pitch = 2 * pitch;
  }
  HOT_STAGE(kStNormBackward, launch_layer_norm_grad(a, s));
  if (apart) HOT_STAGE(kStColumnSums, launch_column_sums(a.sum_gamma, sums, 2 * pitch, cols, g_gamma, g_beta, s));
  return HOT_OK;
}

size_t hot_linear_forward_workspace_bytes(hot_type type, int64_t L, int64_t O, int64_t I) {
  if (!type_ok(type) || !size_ok(L, I) || !size_ok(L, O)) return 0;
  return linear_scratch_bytes(type, L, O, I);
}

hot_status hot_linear_forward(const void* x, const void* w, hot_type type, const float* bias, const void* residual,
                              int64_t L, int64_t O, int64_t I, hot_act_fn fn, void* y, hot_type y_type, void* ckpt,
                              void* ws, size_t ws_bytes, void* stream) {
  if (!x || !w || !y || !type_ok(type) || !type_ok(y_type) || !fn_ok(fn)) return HOT_ERR_ARG;
  if (type == HOT_F32 && y_type != HOT_F32) return HOT_ERR_ARG;
  if (!size_ok(L, I) || !size_ok(L, O)) return HOT_ERR_SHAPE;
  const size_t need = linear_scratch_bytes(type, L, O, I);
  if (need && (!ws || !aligned256(ws))) return HOT_ERR_ARG;
  Buffers b;
  b.in(x, bytes_of(type, L, I));
  b.in(w, bytes_of(type, O, I));
  b.in(bias, O * 4);
  b.in(residual, bytes_of(y_type, L, O));
  b.out(y, bytes_of(y_type, L, O));
  b.out(ckpt, (int64_t)ckpt_layout(L, O).total);
  if (need) b.out(ws, (int64_t)need);
  if (!b.ok()) return HOT_ERR_ARG;
  if (ws_bytes < need) return HOT_ERR_WORKSPACE;
  const LinearForward a{x, w, bias, residual, L, O, I, fn, type, y_type, y, ckpt, need ? ws : nullptr};
  if (launch_linear(a, (hipStream_t)stream) != hipSuccess) return HOT_ERR_DEVICE;
  return HOT_OK;
}

hot_status hot_debug_linear_plan(hot_type type, hot_type y_type, int64_t L, int64_t O, int64_t I, int32_t with_ckpt,
                                 hot_linear_plan* plan) {
  if (!plan || !type_ok(type) || !type_ok(y_type) || (type == HOT_F32 && y_type != HOT_F32)) return HOT_ERR_ARG;
  if (!size_ok(L, I) || !size_ok(L, O)) return HOT_ERR_SHAPE;
  describe_linear(type, y_type, L, O, I, with_ckpt != 0, plan);
  return HOT_OK;
}

}  // extern "C"
