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

// Bias of eight outputs (0 past the last one).
__device__ __forceinline__ void load_bias8(const LinearOut& o, int c, int n, float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = 0.0f;
  if (o.bias && n > 0) load_values(o.bias + c, n, b);
}

// v: x.w^T at (row, c .. c + 7), b: its bias; n = how many of the eight columns exist (may be 0 or less, for a lane of a
// checkpoint group past the last column, whose codes are zero).  With a checkpoint the four lanes of a group call
// this together.
template <class TY>
__device__ __forceinline__ void linear_finish8(const LinearOut& o, int64_t row, int c, int n, const float (&b)[8], float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += b[i];
  if (o.k.codes) {
    if (rarely(n < 8)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
    }
    if (c < (int)o.k.pitch) ckpt_store8(o.k, row * o.k.pitch + c, v);
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

// Workgroup -> tile: workgroups go to the eight XCDs in turn, each with an L2 of its own.  Ids are dealt so that an XCD
// walks a contiguous run of positions, and positions go in bands of eight tile rows, tile row fastest: the tiles it works on
// at a time share their operands in its L2.
__device__ __forceinline__ int xcd_contiguous(int id, int total) {
  const int per_xcd = total / 8;
  return id < per_xcd * 8 ? (id % 8) * per_xcd + id / 8 : id;
}
__device__ __forceinline__ void tile_at(int p, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int band = 8 * tiles_n, first = p / band * 8, in = p % band;
  const int rows = tiles_m - first < 8 ? tiles_m - first : 8;
  tm = first + in % rows;
  tn = in / rows;
}

}  // namespace hot
