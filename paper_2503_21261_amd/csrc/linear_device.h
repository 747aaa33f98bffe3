// What the kernels of the forward product share: the epilogue of eight consecutive outputs of a row.
#pragma once
#include "block_device.h"

namespace hot {

struct LinearOut {
  const float* bias;
  const void* residual;
  void* y;
  CkptView k;        // codes null: no checkpoint
  int64_t L;
  int O;
  int fn;
};

__device__ __forceinline__ void act_any(int fn, float (&v)[8]) {
  switch (fn) {   // uniform
#define HOT_CASE(F)                                     \
  case F:                                               \
    _Pragma("unroll") for (int i = 0; i < 8; ++i) v[i] = act_value<F>(v[i]); \
    break;
    HOT_CASE(HOT_ACT_RELU)
    HOT_CASE(HOT_ACT_GELU)
    HOT_CASE(HOT_ACT_GELU_TANH)
    HOT_CASE(HOT_ACT_SILU)
#undef HOT_CASE
    default: break;
  }
}

// v: x.w^T at (row, c .. c + 7); n = how many of the eight columns exist (may be 0 or less, for a lane of a checkpoint
// group past the last column, whose codes are zero).  With a checkpoint the four lanes of a group call this together.
template <class TY>
__device__ __forceinline__ void linear_finish8(const LinearOut& o, int64_t row, int c, int n, float (&v)[8]) {
  if (o.bias) {
    float b[8] = {};
    if (n > 0) load_values(o.bias + c, n, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += b[i];
  }
  if (o.k.codes) {
    if (n < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
    }
    ckpt_store8(o.k, row * o.k.pitch + c, v);
  }
  act_any(o.fn, v);
  if (n <= 0) return;
  const int64_t at = row * o.O + c;
  if (o.residual) {
    float r[8];
    load_values((const TY*)o.residual + at, n, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  store8((TY*)o.y + at, v, n);
}

}  // namespace hot
