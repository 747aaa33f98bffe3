// Host-side declarations of the low-rank adapters: layouts and launchers.
#pragma once
#include "hot_host.h"

namespace hot {

constexpr int64_t kMaxRank = 128;
constexpr int kMaxSlices = 32;

// Rows of a batch and the adapters of their requests: rows offsets[s] .. offsets[s + 1] - 1 belong to adapter index[s].
struct AdapterBatch {
  const int32_t *offsets, *index;   // device; null: all rows belong to adapter 0
  int segments, adapters;
  int64_t L;
};

// out[l][j] = sum over k of q[l][k] w[adapter(l)][j][k], in `slices` slices of the sum, each [L][pitch] fp32.
struct AdapterShrink {
  AdapterBatch b;
  const void *q, *w;
  float* out;
  int64_t K, w_pitch, w_stride, w_step;   // w: elements from j to j + 1, from adapter to adapter, and a step's distance in units of its length
  int rank, pitch, slices;
  int64_t slice;                    // columns of a slice
  float* u;                         // the sums again, [L][rank] (zeros where a row has no adapter), without slices; or null
};
// y[l][n] = base[l][n] + scale[adapter(l)] * sum over j of p[l][j] w[adapter(l)][n][j], p the sum of the slices.
struct AdapterExpand {
  AdapterBatch b;
  const float* p;
  const void *w, *base;
  const float* scale;
  void* y;
  float* u;                         // p itself, [L][rank]; null: not wanted
  int64_t N, w_pitch, w_stride;
  int rank, pitch, slices;
  int w_cols;                       // elements of a row of w: rank, or more with zeros behind
};
// u and g_u (the sum of its slices) for the sums over rows: [steps of 32 rows][parts][ranks rounded up to 16][32], rows in the order of their
// adapters, and that order itself.
struct AdapterPack {
  AdapterBatch b;
  const float *g_u, *u;
  void *g_out, *u_out;
  const int32_t *order, *start, *first;   // segments in the order of their adapters, their first positions, the adapters' (null without offsets)
  int32_t* rows;                    // rows of the positions
  int rank, g_pitch, slices;
};
// One product of sums over rows: part[slot][j][n] = sum over the part's rows of p[j][l] q[l][n].
struct AdapterOuterOperand {
  const void *p, *q;
  float* part;
  int64_t N;
  int scaled;                       // p times the adapter's scale
};
struct AdapterOuter {
  AdapterBatch b;
  AdapterOuterOperand a[2];
  const float* scale;
  const int32_t *first, *rows;
  int rank, parts;
};
struct AdapterReduce {
  const int32_t* first;
  int64_t L, I, O;
  const float *part_a, *part_b;
  float *g_a, *g_b;
  int rank, parts, adapters;
};
// Before a backward call: segments sorted by adapter, and both weights transposed.
struct AdapterPrepare {
  AdapterBatch b;
  const void *a, *w;                // a [adapters][rank][I], w [adapters][O][rank]
  void *at, *wt;                    // [adapters][I][rank_pitch], [adapters][steps of 128 bytes of O][rank][step]
  int64_t I, O;
  int rank, rank_pitch;
  int64_t wt_stride;
  int32_t *order, *start, *first;
};

struct AdapterPlan {
  bool rows;                        // a wave works on one row, not on a tile of them
  int tile;                         // rows of a workgroup of the first product
  int pitch;                        // floats of a row of p
  int slices_forward, slices_backward, parts;
  int64_t slice_forward, slice_backward;
  int rank_pitch;
  int64_t positions;                // of the packed factors
  size_t at, wt, sorted, packed, part_a, part_b, forward, backward;   // offsets into the workspace, and its sizes
};
AdapterPlan adapter_plan(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters, int64_t segments);

hipError_t launch_adapter_shrink(const AdapterShrink& a, int tile, hot_type type, hipStream_t s);
hipError_t launch_adapter_expand(const AdapterExpand& a, bool rows, hot_type type, hipStream_t s);
hipError_t launch_adapter_prepare(const AdapterPrepare& a, hot_type type, hipStream_t s);
hipError_t launch_adapter_pack(const AdapterPack& a, hot_type type, hipStream_t s);
hipError_t launch_adapter_outer(const AdapterOuter& a, hot_type type, hipStream_t s);
hipError_t launch_adapter_reduce(const AdapterReduce& a, hipStream_t s);

}  // namespace hot
