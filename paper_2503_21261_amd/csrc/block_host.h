// Host-side declarations of the operators around the linear backward: layouts and launchers.
#pragma once
#include "hot_host.h"

namespace hot {

// A checkpoint of [rows x cols]: rows x pitch codes, then (from a multiple of 256) one exponent per 32 codes.
struct CkptLayout {
  int64_t pitch;
  size_t exps, total;
};
inline CkptLayout ckpt_layout(int64_t rows, int64_t cols) {
  CkptLayout k;
  k.pitch = round_up(cols, 32);
  k.exps = (size_t)round_up(rows * k.pitch, 256);
  k.total = k.exps + (size_t)(rows * (k.pitch / 32));
  return k;
}

// Lanes of one launch: a launch of 2^32 or more is refused, so the longest tensors take several.
constexpr int64_t kMaxLaunch = 1ll << 31;

// Whether an output of `rows` rows of `pitch` bytes is stored with the streaming hint: what the L2s (32 MB) could not hold anyway, in
// rows of whole lines.
inline bool stream_output(int64_t rows, int64_t pitch) { return rows * pitch > (32 << 20) && pitch % 128 == 0; }

// Rows of partial sums that a column sum over `rows` rows leaves, and its width: the gradient kernels
// write one such row per row group, `column_sums` adds them; a single row is the sum, and goes where that belongs.
constexpr int kMaxSumRows = 1024;
int activation_sum_rows(int64_t rows, int64_t cols);
int layer_norm_sum_rows(int64_t rows, int64_t cols, hot_type x_type);   // bfloat16: as many as fp32 or more

// x -> y = f(x) (y may be null) and the checkpoint of x (ckpt may be null).
hipError_t launch_activation(int fn, const void* x, hot_type type, int64_t rows, int64_t cols, void* y, void* ckpt,
                             hipStream_t s);
hipError_t launch_checkpoint_read(const void* ckpt, int64_t rows, int64_t cols, void* x, hot_type type, hipStream_t s);
// g_x = g_y f'(x), x from `x` or from `ckpt`; partials (activation_sum_rows() rows, `pitch` floats apart, may be null): sums of g_x.
hipError_t launch_activation_grad(int fn, const void* g_y, hot_type type, const void* x, const void* ckpt, int64_t rows,
                                  int64_t cols, void* g_x, float* partials, int64_t pitch, hipStream_t s);
// out[c] = sum over r of partials[r * width + c]; the second half of a row, where there is one, goes to out2.
hipError_t launch_column_sums(const float* partials, int rows, int64_t width, int64_t cols, float* out, float* out2,
                              hipStream_t s);

constexpr int64_t kMaxNormCols = 16384;
struct NormForward {
  const void *x, *residual;
  const float *gamma, *beta;
  float eps;
  int64_t rows, cols;
  hot_type x_type, y_type;
  void *h, *y, *ckpt;
  float *mean, *rstd;
};
hipError_t launch_layer_norm(const NormForward& a, hipStream_t s);
struct NormBackward {
  const void *g_y, *h, *ckpt, *g_residual;
  const float *gamma, *mean, *rstd;
  int64_t rows, cols;
  hot_type x_type, y_type;
  void* g_x;
  // Row b of sums of workgroup b, at sum_gamma + b * sum_pitch and sum_beta + b * sum_pitch (null: no parameter gradients)
  float *sum_gamma, *sum_beta;
  int64_t sum_pitch;
};
hipError_t launch_layer_norm_grad(const NormBackward& a, hipStream_t s);

// y = f(x.w^T + bias) + residual, and the checkpoint of x.w^T + bias.
struct LinearForward {
  const void *x, *w;
  const float* bias;
  const void* residual;
  int64_t L, O, I;
  int fn;
  hot_type type, y_type;
  void *y, *ckpt, *ws;
};
size_t linear_scratch_bytes(hot_type type, int64_t L, int64_t O, int64_t I);
hipError_t launch_linear(const LinearForward& a, hipStream_t s);
void describe_linear(hot_type type, hot_type y_type, int64_t L, int64_t O, int64_t I, bool kept, hot_linear_plan* out);

}  // namespace hot
