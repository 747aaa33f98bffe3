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
  int64_t K, w_stride;              // w: [rank][K], or packed tiles; elements from adapter to adapter
  int w_packed, rank, pitch, slices;
  int64_t slice;                    // columns of a slice
  // Without slices: the sums again, [L][rank] (zeros where a row has no adapter); and scaled, as the expansion takes them; or null.
  float* u;
  void* packed;
  const float* scale;
  int chunks;                       // chunks of 32 ranks of those; 0: one that holds 16 ranks and their second parts
};
// y[l][n] = base[l][n] + scale[adapter(l)] * sum over j of p[l][j] w[adapter(l)][n][j], p the sum of the slices.
struct AdapterExpand {
  AdapterBatch b;
  const float* p;
  const void *w, *base;
  const float* scale;
  void* y;
  float* u;                         // p itself, [L][rank]; null: not wanted
  const void* packed;               // scale * p in the order of the lanes; null: there are slices
  int64_t N, w_pitch, w_stride;
  int rank, pitch, slices;
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
// One product of sums over rows: part[slot][j][n] = scale[adapter] times the sum over the part's rows of p[j][l] q[l][n].
struct AdapterOuterOperand {
  const void *p, *q;
  float* part;
  int64_t N;
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
// Before the first product: weights packed in the order of its lanes; in a backward call also segments sorted by adapter, and the transpose
// of the second product's weights.
struct AdapterPrepare {
  AdapterBatch b;
  const void *a, *w;                // a [adapters][rank][I]; w [adapters][rank * K], element (j, k) at j * by_j + k * by_k
  void *at, *wt;                    // [adapters][I][rank] (null: not wanted), [adapters][wt_stride]
  int64_t I, K, by_j, by_k, wt_stride;
  int rank;
  int32_t *order, *start, *first;   // null: not wanted
};

struct AdapterPlan {
  bool rows;                        // a wave works on one row, not on a tile of them
  bool pack_forward;                // the forward call packs its weights
  int tile;                         // rows of a workgroup of the first product
  int pitch;                        // floats of a row of p
  int chunks;
  int slices_forward, slices_backward, parts;
  int64_t slice_forward, slice_backward, wt_stride;
  int64_t positions;                // of the packed factors of the sums over rows
  size_t factors, wt, at, sorted, packed, part_a, part_b, forward, backward;   // offsets into the workspace, and its sizes
};
AdapterPlan adapter_plan(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters, int64_t segments);

hipError_t launch_adapter_shrink(const AdapterShrink& a, int tile, hot_type type, hipStream_t s);
hipError_t launch_adapter_expand(const AdapterExpand& a, bool rows, hot_type type, hipStream_t s);
hipError_t launch_adapter_prepare(const AdapterPrepare& a, hot_type type, hipStream_t s);
hipError_t launch_adapter_pack(const AdapterPack& a, hot_type type, hipStream_t s);
hipError_t launch_adapter_outer(const AdapterOuter& a, hot_type type, hipStream_t s);
hipError_t launch_adapter_reduce(const AdapterReduce& a, hipStream_t s);

}  // namespace hot
