// Log probabilities of given tokens, the entropy of each row's distribution, its likeliest tokens, and the gradient of the logits:
//   m = max z, S = sum exp(z - m), log p = z - m - log S, H = -sum p log p = log S - sum exp(z - m) (z - m) / S,
//   g_z = g_logp (1[target] - p) - g_H p (log p + H).
//
// Bound by memory: the forward call reads the logits once (running maximum and sums, rescaled every 32 elements of a lane), the
// gradient reads them and writes as much.
#include "block_device.h"
#include "block_host.h"
#include "tune_host.h"

namespace hot {

namespace {

constexpr int kLanes = 256, kSpan = kLanes * 8;      // elements that a workgroup loads at once: eight a lane
constexpr int kMaxParts = 64, kMaxTop = 32, kCandidates = 256;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.402823466e+38f;
constexpr float kFloor = -300.0f;                    // e^-300 is 0: keeps 0 x -inf out of a sum

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Sums of a part of a row: m = max z, s = sum e^(z - m), w = sum e^(z - m) (z - m).  An infinity or a NaN makes s and w NaN.
struct Sums {
  float m, s, w;
};
// Sums relative to one maximum from those relative to another; a part that held nothing but -inf has s = 0.
__device__ __forceinline__ void rescale(Sums& a, float m) {
  const float d = a.m - m;
  const float shift = d == d ? fmaxf(d, kFloor) : 0.0f, f = exp_of(shift);
  a.w = f * fmaf(shift, a.s, a.w);
  a.s *= f;
  a.m = m;
}

__device__ __forceinline__ float lane_max64(float v) {
  v = fmaxf(v, lane_xor<1>(v));
  v = fmaxf(v, lane_xor<2>(v));
  v = fmaxf(v, lane_xor<4>(v));
  v = fmaxf(v, lane_xor<8>(v));
  v = fmaxf(v, lane_xor<16>(v));
  return fmaxf(v, lane_xor<32>(v));
}

// Values in the order of the likeliest tokens: a NaN first, then by value (-0 is 0).  Among equals the lower token comes first.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  if (z != z) return 0xFFFFFFFFu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ bool before(uint32_t ka, int ia, uint32_t kb, int ib) { return ka > kb || (ka == kb && ia < ib); }

// The first of a wave's lanes' (key, token), in its first N lanes: permutes on the vector pipe for up to 16.
template <int MASK>
__device__ __forceinline__ void first_with(uint32_t& key, int& id) {
  const uint32_t k = lane_xor<MASK>(key);
  const int i = (int)lane_xor<MASK>((uint32_t)id);
  if (before(k, i, key, id)) {
    key = k;
    id = i;
  }
}
__device__ __forceinline__ void first_of_lanes(uint32_t& key, int& id, int n) {
  first_with<1>(key, id);
  first_with<2>(key, id);
  first_with<4>(key, id);
  first_with<8>(key, id);
  if (n > 16) first_with<16>(key, id);
  if (n > 32) first_with<32>(key, id);
}

// What leaves the sums of a whole row.
struct RowResult {
  float m, log_s, entropy;
};
__device__ __forceinline__ RowResult finish(const Sums& a) {
  RowResult r;
  if (a.s == 0.0f) {       // nothing but -inf
    r.m = -INFINITY;
    r.log_s = 0.0f;
    r.entropy = 0.0f;
    return r;
  }
  r.m = a.m;
  r.log_s = kLn2 * __builtin_amdgcn_logf(a.s);
  r.entropy = r.log_s - a.w / a.s;
  return r;
}
__device__ __forceinline__ float log_prob(float z, const RowResult& r) {
  return r.m == -INFINITY ? -INFINITY : (z - r.m) - r.log_s;
}

struct LogProbArgs {
  const void* logits;
  const int64_t* targets;
  float *logp, *entropy, *stats, *top_logp;
  int32_t* top_ids;
  float* part_sums;        // [rows][parts][4]
  float* part_top;         // [rows][parts][top] values, then tokens
  int32_t* part_ids;
  int64_t vocab, first_row;
  int part, parts, top;    // elements of a part (a multiple of kSpan), parts of a row
};

template <class T>
__device__ __forceinline__ void load_logits(const T* row, int64_t at, int64_t end, float (&v)[8]) {
  const int n = (int)min((int64_t)8, end - at);
  load_values(row + at, n, v);
  if (rarely(n < 8)) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= n) v[i] = -INFINITY;
  }
}

// The first `top` of a part in order: values and tokens to out_z, out_id (LDS).  tmax: the lane's largest value but for NaNs;
// nan: whether the part holds one.
template <class T>
__device__ void part_top(const T* row, int64_t first, int64_t end, int top, float tmax, bool nan, float* out_z, int* out_id) {
  __shared__ float s_group[64];
  __shared__ uint32_t s_key[kCandidates];
  __shared__ int s_id[kCandidates];
  __shared__ int s_count;
  __shared__ float s_border;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // The `top`-th largest of the maxima of 64 groups of lanes is at most the `top`-th largest value: a border that few values pass.
  float g = fmaxf(tmax, lane_xor<1>(tmax));
  g = fmaxf(g, lane_xor<2>(g));
  if ((lane & 3) == 0) s_group[wave * 16 + lane / 4] = g;
  if (tid == 0) s_count = 0;
  __syncthreads();
  if (wave == 0) {
    const float mine = s_group[lane];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) {
      const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), i));
      rank += other > mine || (other == mine && i < lane);
    }
    if (rank == top - 1) s_border = mine;
  }
  __syncthreads();
  const float border = s_border;
  if (!nan && border != -INFINITY) {
    if (tmax >= border) {
      for (int64_t at = first + tid * 8; at < end; at += kSpan) {
        float v[8];
        load_logits(row, at, end, v);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (v[i] >= border) {
            const int k = atomicAdd(&s_count, 1);
            if (k < kCandidates) {
              s_key[k] = order_key(v[i]);
              s_id[k] = (int)(at + i);
            }
          }
      }
    }
    __syncthreads();
    const int count = s_count;
    if (count <= kCandidates) {     // uniform; the order in which lanes came does not show in the ranks
      if (tid < count) {
        const uint32_t key = s_key[tid];
        const int id = s_id[tid];
        int rank = 0;
        for (int i = 0; i < count; ++i) rank += before(s_key[i], s_id[i], key, id);
        if (rank < top) {
          out_z[rank] = (float)row[id];
          out_id[rank] = id;
        }
      }
      __syncthreads();
      return;
    }
  }
  // Many values at the border, rows with few finite values or NaNs: one after the other, each the first behind the last one.
  uint32_t last_key = 0xFFFFFFFFu;
  int last_id = -1;
  for (int k = 0; k < top; ++k) {
    uint32_t key = 0;
    int id = 0x7FFFFFFF;
    for (int64_t at = first + tid * 8; at < end; at += kSpan) {
      float v[8];
      load_logits(row, at, end, v);
      const int n = (int)min((int64_t)8, end - at);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t c = order_key(v[i]);
        if (i < n && before(last_key, last_id, c, (int)at + i) && before(c, (int)at + i, key, id)) {
          key = c;
          id = (int)at + i;
        }
      }
    }
    first_of_lanes(key, id, 64);
    __syncthreads();
    if (lane == 0) {
      s_key[wave] = key;
      s_id[wave] = id;
    }
    __syncthreads();
    for (int i = 0; i < kLanes / 64; ++i)
      if (before(s_key[i], s_id[i], key, id)) {
        key = s_key[i];
        id = s_id[i];
      }
    last_key = key;
    last_id = id;
    if (tid == 0) {
      const bool there = id != 0x7FFFFFFF;     // a short part holds fewer than `top`
      out_z[k] = there ? (float)row[id] : -INFINITY;
      out_id[k] = id;
    }
  }
  __syncthreads();
}

template <class T, bool ENTROPY>
__global__ __launch_bounds__(kLanes) void logprob_kernel(const LogProbArgs a) {
  __shared__ Sums s_sums[kLanes / 64];
  __shared__ float s_z[kMaxTop];
  __shared__ int s_token[kMaxTop];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = a.first_row + blockIdx.x / a.parts;
  const int p = blockIdx.x % a.parts;
  const T* const row = (const T*)a.logits + r * a.vocab;
  const int64_t first = (int64_t)p * a.part, end = min(first + a.part, a.vocab);
  const int64_t target = a.targets ? a.targets[r] : -1;
  const bool scored = target >= 0 && target < a.vocab;
  const float z_target = a.parts == 1 && scored ? (float)row[target] : 0.0f;

  Sums t{kLowest, 0.0f, 0.0f};
  float tmax = -INFINITY;
  const auto add = [&](const float (&v)[4][8]) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, v[u][i]);
    tmax = fmaxf(tmax, top);
    if (top > t.m) rescale(t, top);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = v[u][i] - t.m, e = exp_of(d);
        t.s += e;
        if (ENTROPY) t.w = fmaf(e, fmaxf(d, kFloor), t.w);
      }
  };
  int64_t at = first + tid * 8;
  for (; at + 3 * kSpan + 8 <= end; at += 4 * kSpan) {
    Raw8<T> raw[4];
    float v[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) raw[u] = load8(row + at + u * kSpan, 8);
#pragma unroll
    for (int u = 0; u < 4; ++u) widen(raw[u], v[u]);
    add(v);
  }
  if (at < end) {
    float v[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) load_logits(row, at + u * kSpan, end, v[u]);
    add(v);
  }
  const float m = lane_max64(t.m);
  rescale(t, m);
  t.s = lanes_sum<64>(t.s);
  if (ENTROPY) t.w = lanes_sum<64>(t.w);
  if (lane == 0) s_sums[wave] = t;
  __syncthreads();
  float all = kLowest;
#pragma unroll
  for (int i = 0; i < kLanes / 64; ++i) all = fmaxf(all, s_sums[i].m);
  Sums q{all, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kLanes / 64; ++i) {
    Sums o = s_sums[i];
    rescale(o, all);
    q.s += o.s;
    q.w += o.w;
  }
  if (a.top) part_top(row, first, end, a.top, tmax, q.s != q.s, s_z, s_token);
  if (a.parts > 1) {
    const int64_t at = r * a.parts + p;
    if (tid == 0) *(float4*)(a.part_sums + at * 4) = make_float4(q.m, q.s, q.w, 0.0f);
    if (tid < a.top) {
      a.part_top[at * a.top + tid] = s_z[tid];
      a.part_ids[at * a.top + tid] = s_token[tid];
    }
    return;
  }
  const RowResult f = finish(q);
  if (tid == 0) {
    if (a.logp) a.logp[r] = scored ? log_prob(z_target, f) : 0.0f;
    if (a.entropy) a.entropy[r] = f.entropy;
    if (a.stats) *(float2*)(a.stats + 2 * r) = make_float2(f.m, f.log_s);
  }
  if (tid < a.top) {
    a.top_logp[r * a.top + tid] = log_prob(s_z[tid], f);
    a.top_ids[r * a.top + tid] = s_token[tid];
  }
}

// Joins the parts of a row: one wave, a part a lane.  The parts' lists are in order, so the first of the row is the first of the
// lists' heads, `top` times.
template <class T>
__global__ __launch_bounds__(64) void logprob_join_kernel(const LogProbArgs a) {
  __shared__ float s_z[kMaxParts * kMaxTop];
  __shared__ int s_token[kMaxParts * kMaxTop];
  const int lane = threadIdx.x;
  const int64_t r = a.first_row + blockIdx.x;
  const int64_t target = a.targets ? a.targets[r] : -1;
  const bool scored = target >= 0 && target < a.vocab;
  const float z_target = scored ? (float)((const T*)a.logits + r * a.vocab)[target] : 0.0f;
  Sums t{kLowest, 0.0f, 0.0f};
  if (lane < a.parts) {
    const float4 x = *(const float4*)(a.part_sums + (r * a.parts + lane) * 4);
    t = Sums{x.x, x.y, x.z};
  }
  const int held = a.parts * a.top;
  for (int i = lane; i < held; i += 64) {
    s_z[i] = a.part_top[r * held + i];
    s_token[i] = a.part_ids[r * held + i];
  }
  const float m = lane_max64(t.m);
  rescale(t, m);
  t.s = lanes_sum<64>(t.s);
  t.w = lanes_sum<64>(t.w);
  const RowResult f = finish(t);
  if (lane == 0) {
    if (a.logp) a.logp[r] = scored ? log_prob(z_target, f) : 0.0f;
    if (a.entropy) a.entropy[r] = f.entropy;
    if (a.stats) *(float2*)(a.stats + 2 * r) = make_float2(f.m, f.log_s);
  }
  __syncthreads();
  int head = 0;
  for (int k = 0; k < a.top; ++k) {
    const int at = lane * a.top + head;
    const bool there = lane < a.parts && head < a.top;
    const int mine = there ? s_token[at] : 0x7FFFFFFF;
    const float z = there ? s_z[at] : -INFINITY;
    uint32_t key = mine == 0x7FFFFFFF ? 0u : order_key(z);
    int id = mine;
    first_of_lanes(key, id, a.parts);
    if (mine == id && there) {       // one lane: tokens differ, and there are `top` of them at least
      a.top_logp[r * a.top + k] = log_prob(z, f);
      a.top_ids[r * a.top + k] = id;
      ++head;
    }
  }
}

struct GradArgs {
  const void* logits;
  const int64_t* targets;
  const float *stats, *entropy, *g_logp, *g_entropy;
  void* g_logits;
  int64_t vocab, first_row;
  int parts;
};
constexpr int kGradSpans = 4;   // spans of a workgroup

template <class T, bool ENTROPY, bool STREAM>
__global__ __launch_bounds__(kLanes) void logprob_grad_kernel(const GradArgs a) {
  const int64_t r = a.first_row + blockIdx.x / a.parts;
  const int64_t first = (int64_t)(blockIdx.x % a.parts) * (kGradSpans * kSpan) + threadIdx.x * 8;
  const T* const row = (const T*)a.logits + r * a.vocab;
  T* const out = (T*)a.g_logits + r * a.vocab;
  float v[kGradSpans][8];
  int n[kGradSpans];
#pragma unroll
  for (int u = 0; u < kGradSpans; ++u) {
    const int64_t at = first + u * kSpan;
    n[u] = (int)max(min((int64_t)8, a.vocab - at), (int64_t)0);
    load_values(row + at, n[u], v[u]);
  }
  const float2 st = *(const float2*)(a.stats + 2 * r);
  const int64_t target = a.targets ? a.targets[r] : -1;
  const float g_t = a.g_logp && target >= 0 && target < a.vocab ? a.g_logp[r] : 0.0f;
  const bool nothing = st.x == -INFINITY;    // a row of -inf alone
  const float g_h = ENTROPY ? a.g_entropy[r] : 0.0f, h = ENTROPY ? a.entropy[r] : 0.0f;
  const float base = ENTROPY ? fmaf(-g_h, h, -g_t) : -g_t;
#pragma unroll
  for (int u = 0; u < kGradSpans; ++u) {
    const int64_t at = first + u * kSpan;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = (v[u][i] - st.x) - st.y, e = exp_of(d);     // log p, p
      v[u][i] = e * (ENTROPY ? fmaf(-g_h, fmaxf(d, kFloor), base) : base);
    }
    if (rarely(target >= at && target < at + 8)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (target == at + i) v[u][i] += g_t;
    }
    if (rarely(nothing)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = 0.0f;
    }
    if (n[u] > 0) store8<STREAM>(out + at, v[u], n[u]);
  }
}

int spans_of_part(int64_t vocab, int parts) { return (int)ceil_div(ceil_div(vocab, parts), kSpan); }

template <class T>
hipError_t run_forward(LogProbArgs k, int64_t rows, hipStream_t s) {
  const int64_t run = (1ll << 23) / k.parts;   // 2^31 lanes a launch
  const bool entropy = k.entropy != nullptr;
  for (k.first_row = 0; k.first_row < rows; k.first_row += run) {
    const int64_t n = rows - k.first_row < run ? rows - k.first_row : run;
    if (entropy) logprob_kernel<T, true><<<(uint32_t)(n * k.parts), kLanes, 0, s>>>(k);
    else logprob_kernel<T, false><<<(uint32_t)(n * k.parts), kLanes, 0, s>>>(k);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (k.parts > 1) logprob_join_kernel<T><<<(uint32_t)n, 64, 0, s>>>(k);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T, bool STREAM>
hipError_t run_grad(GradArgs k, int64_t rows, hipStream_t s) {
  const int64_t run = (1ll << 23) / k.parts;
  for (k.first_row = 0; k.first_row < rows; k.first_row += run) {
    const int64_t n = rows - k.first_row < run ? rows - k.first_row : run;
    if (k.g_entropy) logprob_grad_kernel<T, true, STREAM><<<(uint32_t)(n * k.parts), kLanes, 0, s>>>(k);
    else logprob_grad_kernel<T, false, STREAM><<<(uint32_t)(n * k.parts), kLanes, 0, s>>>(k);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

// Few rows are cut into parts, so that there are workgroups for all compute units; a part is one span at least.
int logprob_parts(hot_type, int64_t rows, int64_t vocab) {
  const int64_t most = ceil_div(vocab, kSpan), wanted = ceil_div(2048, rows);
  int64_t parts = most < wanted ? most : wanted;
  if (parts > kMaxParts) parts = kMaxParts;
  return (int)ceil_div(vocab, (int64_t)spans_of_part(vocab, (int)parts) * kSpan);
}
size_t logprob_scratch_bytes(hot_type type, int64_t rows, int64_t vocab, int top) {
  const int parts = logprob_parts(type, rows, vocab);
  return parts == 1 ? 0 : (size_t)(rows * parts) * (16 + 8 * (size_t)top);
}

hipError_t launch_logprobs(const LogProbs& a, hipStream_t s) {
  LogProbArgs k{};
  k.logits = a.logits;
  k.targets = a.targets;
  k.logp = a.logp;
  k.entropy = a.entropy;
  k.stats = a.stats;
  k.top_logp = a.top_logp;
  k.top_ids = a.top_ids;
  k.vocab = a.vocab;
  k.top = a.top;
  k.parts = logprob_parts(a.type, a.rows, a.vocab);
  k.part = spans_of_part(a.vocab, k.parts) * kSpan;
  if (k.parts > 1) {
    k.part_sums = (float*)a.ws;
    k.part_top = k.part_sums + a.rows * k.parts * 4;
    k.part_ids = (int32_t*)(k.part_top + a.rows * k.parts * a.top);
  }
  return a.type == HOT_BF16 ? run_forward<bf16>(k, a.rows, s) : run_forward<float>(k, a.rows, s);
}

hipError_t launch_logprob_grad(const LogProbGrad& a, hipStream_t s) {
  GradArgs k{a.logits, a.targets, a.stats, a.entropy, a.g_logp, a.g_entropy, a.g_logits, a.vocab, 0,
             (int)ceil_div(a.vocab, kGradSpans * kSpan)};
  const bool stream = stream_output(a.rows, a.vocab * (a.type == HOT_BF16 ? 2 : 4));
  if (a.type == HOT_BF16) return stream ? run_grad<bf16, true>(k, a.rows, s) : run_grad<bf16, false>(k, a.rows, s);
  return stream ? run_grad<float, true>(k, a.rows, s) : run_grad<float, false>(k, a.rows, s);
}

}  // namespace hot
