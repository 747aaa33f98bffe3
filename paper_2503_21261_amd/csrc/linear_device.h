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
  int stream;        // y is stored with the streaming hint
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
    if (c < (int)o.k.pitch) {
      if (o.stream) ckpt_store8<true>(o.k, row * o.k.pitch + c, v);
      else ckpt_store8(o.k, row * o.k.pitch + c, v);
    }
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
  // Streamed: 16384 x 11008 x 4096 bfloat16 1130 -> 1070 us, with GELU and checkpoint 1215 -> 1155; 50432 x 2304 x 768 fp32 525 -> 504.
  if (!o.stream) {
    store8((TY*)o.y + at, v, n);
  } else if (sizeof(TY) == 2 || __builtin_amdgcn_ballot_w64(n < 8)) {
    store8<true>((TY*)o.y + at, v, n);
  } else {
    // fp32, both lanes of a pair (a streamed row is whole groups of 32 columns): they exchange halves, so that each store of theirs is
    // 32 bytes in a row (12608 x 2304 x 768 142 us, 148 with four of every eight columns a store)
    const bool odd = threadIdx.x & 1;
    f4_any first, second;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float other = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(odd ? v[i] : v[i + 4]), 0xB1, 0xF, 0xF, true));
      first[i] = odd ? other : v[i];
      second[i] = odd ? v[i + 4] : other;
    }
    float* const p = (float*)o.y + at + (odd ? -4 : 0);
    __builtin_nontemporal_store(first, (f4_any*)p);
    __builtin_nontemporal_store(second, (f4_any*)(p + 8));
  }
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
