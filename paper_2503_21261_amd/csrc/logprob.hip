// Log probabilities of given tokens, the entropy of each row's distribution, its likeliest tokens, and the gradient of the logits:
//   m = max z, S = sum exp(z - m), log p = z - m - log S, H = -sum p log p = log S - sum exp(z - m) (z - m) / S,
//   g_z = g_logp (1[target] - p) - g_H p (log p + H).
//
// Bound by memory: the forward call reads the logits once (running maximum and sums, rescaled every 32 elements of a lane), the
// gradient reads them and writes as much.  16384 x 32000 bfloat16 with entropy: 213 us (4.9 TB/s) and 378 us (5.6).
//
// A row is a workgroup's where there are rows for all compute units, so that nothing is joined; few rows are cut into parts, which a launch of
// one wave a row joins: 96 x 50257 fp32, 8 likeliest: 11.5 and 4.1 us; 1 x 32000, 20 likeliest: 7.3 and 5.0, latencies.
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

// 0 where the power is below 2^-126 (the instruction's way), which is 2^-126 |log p| of a gradient at most.
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

// Values in the order of the likeliest tokens, the first the largest number: a NaN first, then by value (-0 is 0), among equals the lower token.
__device__ __forceinline__ uint64_t order_of(float z, int token) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  const uint32_t key = z != z ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)key << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float value_of(uint64_t order) {
  const uint32_t key = (uint32_t)(order >> 32);
  return key == 0xFFFFFFFFu ? __uint_as_float(0x7FC00000u) : __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ int token_of(uint64_t order) { return (int)~(uint32_t)order; }

// A wave's values sorted, the largest in lane 0 (bitonic: 21 exchanges of neighbours at powers of two).
template <int RUN, int MASK>
__device__ __forceinline__ void sort_step(float& v) {
  const int lane = threadIdx.x & 63;
  const float o = lane_xor<MASK>(v);
  v = ((lane & MASK) == 0) == ((lane & RUN) == 0) ? fmaxf(v, o) : fminf(v, o);
  if constexpr (MASK > 1) sort_step<RUN, MASK / 2>(v);
}
__device__ __forceinline__ void sort_wave(float& v) {
  sort_step<2, 1>(v);
  sort_step<4, 2>(v);
  sort_step<8, 4>(v);
  sort_step<16, 8>(v);
  sort_step<32, 16>(v);
  sort_step<64, 32>(v);
}

// How many of the n orders at t come before `mine` (t is held to a multiple of eight, zeros behind the n, which come last).
__device__ __forceinline__ int rank_among(const uint64_t* t, int n, uint64_t mine) {
  int rank = 0;
#pragma unroll 1
  for (int i = 0; i < n; i += 8) {
    uint64_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = t[i + e];
#pragma unroll
    for (int e = 0; e < 8; ++e) rank += x[e] > mine;
  }
  return rank;
}
template <int MASK>
__device__ __forceinline__ uint64_t max_with(uint64_t v) {
  const uint64_t o = (uint64_t)lane_xor<MASK>((uint32_t)(v >> 32)) << 32 | lane_xor<MASK>((uint32_t)v);
  return o > v ? o : v;
}
// The largest of the first n lanes' (their number rounded up to a power of two, 16 at least), in all of them.
__device__ __forceinline__ uint64_t max_of_lanes(uint64_t v, int n) {
  v = max_with<1>(v);
  v = max_with<2>(v);
  v = max_with<4>(v);
  v = max_with<8>(v);
  if (n > 16) v = max_with<16>(v);
  if (n > 32) v = max_with<32>(v);
  return v;
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
  uint64_t* part_top;      // [rows][parts][top] orders
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

// The first `top` of a part in order, to out (LDS); zeros where a short part holds fewer.  v: the lane's values, those of 4 spans from `first` on (a part has
// no more, but for vocabularies that 64 parts of 4 spans do not hold: they are read again); tmax: the lane's largest of all but NaNs;
// nan: whether the part holds one.
template <class T>
__device__ void part_top(const T* row, int64_t first, int64_t end, int top, const float (&v)[4][8], float tmax, bool nan, uint64_t* out) {
  __shared__ float s_group[64];
  __shared__ uint64_t s_order[kCandidates];
  __shared__ int s_count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // The `top`-th largest of the maxima of 64 groups of lanes is at most the `top`-th largest value: a border that few values pass.
  float g = fmaxf(tmax, lane_xor<1>(tmax));
  g = fmaxf(g, lane_xor<2>(g));
  if ((lane & 3) == 0) s_group[wave * 16 + lane / 4] = g;
  s_order[tid] = 0;
  if (tid == 0) s_count = 0;
  __syncthreads();
  float sorted = s_group[lane];
  sort_wave(sorted);            // every wave for itself
  const float border = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_int(sorted), top - 1));
  if (!nan && border != -INFINITY) {
    if (tmax >= border) {
      const auto take = [&](const float (&x)[8], int64_t at) {
        int mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) mine += x[i] >= border;
        if (mine == 0) return;
        int k = atomicAdd(&s_count, mine);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (x[i] >= border && k < kCandidates) s_order[k] = order_of(x[i], (int)at + i);
          k += x[i] >= border;
        }
      };
#pragma unroll
      for (int u = 0; u < 4; ++u) take(v[u], first + u * kSpan + tid * 8);
      for (int64_t at = first + 4 * kSpan + tid * 8; at < end; at += kSpan) {
        float x[8];
        load_logits(row, at, end, x);
        take(x, at);
      }
    }
    __syncthreads();
    const int count = s_count;
    if (count <= kCandidates) {     // uniform; the order in which lanes came does not show in the ranks
      if (tid < count) {
        const uint64_t mine = s_order[tid];
        const int rank = rank_among(s_order, count, mine);
        if (rank < top) out[rank] = mine;
      }
      __syncthreads();
      return;
    }
  }
  // Many values at the border, rows with few finite values or NaNs: one after the other, each the first behind the last one.
  uint64_t last = ~0ull;
  for (int k = 0; k < top; ++k) {
    uint64_t best = 0;
    for (int64_t at = first + tid * 8; at < end; at += kSpan) {
      float v[8];
      load_logits(row, at, end, v);
      const int n = (int)min((int64_t)8, end - at);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint64_t c = order_of(v[i], (int)at + i);
        if (i < n && c < last && c > best) best = c;
      }
    }
    best = max_of_lanes(best, 64);
    __syncthreads();
    if (lane == 0) s_order[wave] = best;
    __syncthreads();
    for (int i = 0; i < kLanes / 64; ++i) best = s_order[i] > best ? s_order[i] : best;
    last = best;
    if (tid == 0) out[k] = best;
  }
  __syncthreads();
}

template <class T, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kLanes) void logprob_kernel(const LogProbArgs a) {
  __shared__ Sums s_sums[kLanes / 64];
  __shared__ uint64_t s_top[kMaxTop];
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
  const auto load = [&](int64_t at, float (&v)[4][8]) {
    if (at + 3 * kSpan + 8 <= end) {
      Raw8<T> raw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) raw[u] = load8(row + at + u * kSpan, 8);
#pragma unroll
      for (int u = 0; u < 4; ++u) widen(raw[u], v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) load_logits(row, at + u * kSpan, end, v[u]);
    }
  };
  int64_t at = first + tid * 8;
  float held[4][8];                // the first ones, for the likeliest tokens
  if constexpr (TOP) {
    load(at, held);
    add(held);
    at += 4 * kSpan;
  }
  for (; at < end; at += 4 * kSpan) {
    float v[4][8];
    load(at, v);
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
  if constexpr (TOP) part_top(row, first, end, a.top, held, tmax, q.s != q.s, s_top);
  if (a.parts > 1) {
    const int64_t at = r * a.parts + p;
    if (tid == 0) *(float4*)(a.part_sums + at * 4) = make_float4(q.m, q.s, q.w, 0.0f);
    if (tid < a.top) a.part_top[at * a.top + tid] = s_top[tid];
    return;
  }
  const RowResult f = finish(q);
  if (tid == 0) {
    if (a.logp) a.logp[r] = scored ? log_prob(z_target, f) : 0.0f;
    if (a.entropy) a.entropy[r] = f.entropy;
    if (a.stats) *(float2*)(a.stats + 2 * r) = make_float2(f.m, f.log_s);
  }
  if (tid < a.top) {
    a.top_logp[r * a.top + tid] = log_prob(value_of(s_top[tid]), f);
    a.top_ids[r * a.top + tid] = token_of(s_top[tid]);
  }
}

// Joins the parts of a row: one wave, a part a lane.  The parts' lists are in order, so the first of the row is the first of the
// lists' heads, `top` times.
template <class T>
__global__ __launch_bounds__(64) void logprob_join_kernel(const LogProbArgs a) {
  __shared__ uint64_t s_list[kMaxParts * kMaxTop];
  __shared__ uint64_t s_order[64];
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
#pragma unroll 8
  for (int i = lane; i < held; i += 64) s_list[i] = a.part_top[r * held + i];
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
  if (a.top == 0) return;
  __syncthreads();
  // Each list's `depth` first ones come no later than its entry at depth - 1, so that `top` or more come no later than the border below, and
  // mostly not many more.
  const int depth = min((2 * a.top + a.parts - 1) / a.parts, a.top), wanted = (a.top + depth - 1) / depth;
  const uint64_t mine = lane < a.parts ? s_list[lane * a.top + depth - 1] : 0ull;
  s_order[lane] = mine;
  __syncthreads();
  const bool chosen = mine != 0 && rank_among(s_order, a.parts, mine) == wanted - 1;
  const uint64_t vote = __builtin_amdgcn_ballot_w64(chosen);
  int count = 0;
  if (vote) {
    const int at = __ffsll((unsigned long long)vote) - 1;
    const uint64_t border = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), at) << 32 |
                            (uint32_t)__builtin_amdgcn_readlane((int)mine, at);
    __syncthreads();
    s_order[lane] = 0;
    __syncthreads();
    for (int j = 0; j < a.top; ++j) {
      const uint64_t x = lane < a.parts ? s_list[lane * a.top + j] : 0ull;
      const uint64_t passing = __builtin_amdgcn_ballot_w64(x >= border);
      if (passing == 0) break;
      const int place = count + __popcll(passing & ((1ull << lane) - 1));
      if (x >= border && place < 64) s_order[place] = x;
      count += __popcll(passing);
    }
    __syncthreads();
  }
  if (vote && count <= 64) {
    const uint64_t x = s_order[lane];
    const int rank = rank_among(s_order, count, x);
    if (lane < count && rank < a.top) {
      a.top_logp[r * a.top + rank] = log_prob(value_of(x), f);
      a.top_ids[r * a.top + rank] = token_of(x);
    }
    return;
  }
  int head = 0;
  for (int k = 0; k < a.top; ++k) {
    const uint64_t own = lane < a.parts && head < a.top ? s_list[lane * a.top + head] : 0ull;
    const uint64_t best = max_of_lanes(own, a.parts);
    if (own == best && own != 0) {       // one lane: there are `top` of them at least
      a.top_logp[r * a.top + k] = log_prob(value_of(own), f);
      a.top_ids[r * a.top + k] = token_of(own);
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
    const auto go = [&](auto kernel) { kernel<<<(uint32_t)(n * k.parts), kLanes, 0, s>>>(k); };
    if (k.top) entropy ? go(logprob_kernel<T, true, true>) : go(logprob_kernel<T, false, true>);
    else entropy ? go(logprob_kernel<T, true, false>) : go(logprob_kernel<T, false, false>);
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

// Few rows are cut into parts, so that there are workgroups for all compute units; a part is one span at least, and with likeliest tokens what a
// workgroup holds in registers at most.
static int logprob_parts(int64_t rows, int64_t vocab, int top) {
  const int64_t most = ceil_div(vocab, kSpan), wanted = ceil_div(2048, rows);
  int64_t parts = most < wanted ? most : wanted;
  if (top && parts < ceil_div(vocab, 4 * kSpan)) parts = ceil_div(vocab, 4 * kSpan);
  if (parts > kMaxParts) parts = kMaxParts;
  return (int)ceil_div(vocab, (int64_t)spans_of_part(vocab, (int)parts) * kSpan);
}
size_t logprob_scratch_bytes(int64_t rows, int64_t vocab, int top) {
  const int parts = logprob_parts(rows, vocab, top);
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
  k.parts = logprob_parts(a.rows, a.vocab, a.top);
  k.part = spans_of_part(a.vocab, k.parts) * kSpan;
  if (k.parts > 1) {
    k.part_sums = (float*)a.ws;
    k.part_top = (uint64_t*)(k.part_sums + a.rows * k.parts * 4);
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
