// One optimiser step (AdamW) over many tensors: m' = b1 m + (1 - b1) g, v' = b2 v + (1 - b2) g^2,
// p' = p - lr (decay p + (m' / c1) / (sqrt(v' / c2) + eps)), and the 8-bit form of the two moments.
//
// Bound by memory: an element is read and written once, 28 bytes with fp32 moments and parameters, 16.1 with 8-bit moments and
// fp32 parameters and gradients.  One launch takes forty tensors: a lane finds its tensor from its workgroup's number, so that
// small tensors (biases, norms) cost no launch of their own.  302 million fp32 elements: 1518 us, 5.6 TB/s; 361 million with 8-bit
// moments, bfloat16 gradients and copies: 1134 us, 5.1 TB/s; 18 million bfloat16 ones with 8-bit moments: 53 us, 3.5 TB/s, bound by the
// hundred vector instructions of an element (quotient and root rounded once, two codes), which come at the same rate in the larger one: 1.1 to 1.2
// of them in four cycles of a SIMD.  Both with moments
// rounded by their own low bits; by draws (below) 1114 us, for 1095 in the same process, and 57.
#include "block_device.h"
#include "tune_host.h"

namespace hot {

namespace {

// ---- the 8-bit moments ----------------------------------------------------------------------------
// m: the form of the 8-bit checkpoint, a signed code times a power-of-two step that 32 elements share.
// v, which spans the squares of what m does: a code of five exponent and three mantissa bits under the largest exponent e of 32
// elements: 0, or 1.fff x 2^(x - 31 + e - 127) with x the upper five bits.  All but the rounding is exact in both, and the
// roundings' inputs are single fp32 operations, so codes have one value whatever computes them.
// Rounding: with b2 = 0.999 a step moves v by 0.1 %, 1/60 to 1/120 of a code, so that rounding to the nearest would bring the same code back
// for ever; and so does rounding by the value's own low 11 bits, this library's way with what is quantised once, where a step does not change
// them: v decoded has none, and b2 v the same ones each time (gradients of zero: v stays; gradients that fall to a tenth: v is 14 times
// what it should be 3000 steps later).  So the bits that decide are drawn (HOT_ROUND_DRAWN), anew in each step, which leaves both moments right
// on average.  The other two are the definitions that a step's results can be compared by.
// A v that is not zero never becomes zero: the least code is held instead, so that 1 / sqrt(v) is not blown up.
constexpr uint32_t kVMinExp = 32;   // keeps the least code a normal number

// Draws of eight elements: h is uniform and new in each step, and eight multiples of the golden ratio (in the upper 16 bits and in the lower
// ones) spread the eight elements evenly behind it; the moments' own bits keep elements at the same place of other blocks from rounding
// alike.  What decides over v are the upper 20 bits, all that are rounded away; over m the lower 16.
__device__ __forceinline__ uint32_t mixed(uint32_t x) {      // a bijection: every bit of x changes every other with probability 0.496 to 0.504
  x = (x ^ x >> 16) * 0x6A09E667u;
  x = (x ^ x >> 15) * 0xBB67AE85u;
  return x ^ x >> 16;
}
__device__ __forceinline__ uint32_t seed_with(uint32_t seed, uint32_t x) { return mixed(seed ^ x ^ 0x9E3779B9u); }
__device__ __forceinline__ void draw8(uint32_t seed, int64_t at, const float (&m)[8], const float (&v)[8], uint32_t (&draw)[8]) {
  const uint32_t h = mixed(seed + ((uint32_t)at & (kStateBlock - 1)) / 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) draw[i] = h + __float_as_uint(m[i]) + __float_as_uint(v[i]) + (uint32_t)i * 0x9E379E37u;
}

template <hot_rounding ROUNDING>
__device__ __forceinline__ uint2 encode_m8(const float (&v)[8], float inverse, const uint32_t (&draw)[8]) {
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = v[i] * inverse;
    float q;
    if constexpr (ROUNDING == HOT_ROUND_NEAREST_EVEN) {
      q = rintf(t);
    } else if constexpr (ROUNDING == HOT_ROUND_DRAWN) {
      q = floorf(t + ((float)(draw[i] & 0xFFFFu) + 0.5f) * (1.0f / 65536.0f));
    } else {
      q = floorf(t);
      q += t - q > (float)(__float_as_uint(t) & 0x7FFu) * (1.0f / 2048.0f) ? 1.0f : 0.0f;
    }
    c[i] = (int)fminf(fmaxf(q, -127.0f), 127.0f);
  }
  return make_uint2(pack4_codes8(c[0], c[1], c[2], c[3]), pack4_codes8(c[4], c[5], c[6], c[7]));
}

// Upper bits of v after rounding: exponent and three bits of the mantissa.
template <hot_rounding ROUNDING>
__device__ __forceinline__ uint32_t rounded_v(float v, uint32_t draw) {
  const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;   // -0 is 0; below zero is marked as NaN
  if constexpr (ROUNDING == HOT_ROUND_NEAREST_EVEN) return (b + 0x7FFFFu + (b >> 20 & 1u)) >> 20;
  else if constexpr (ROUNDING == HOT_ROUND_DRAWN) return (b + (draw >> 12)) >> 20;
  else return (b >> 20) + ((b & 0xFFFFFu) > (b & 0x7FFu) << 9 ? 1u : 0u);
}

// Codes of eight elements of a group, by the four lanes of the group together; e: the group's exponent byte.
template <hot_rounding ROUNDING>
__device__ __forceinline__ uint2 store_v8(const float (&v)[8], const uint32_t (&draw)[8], uint32_t& e) {
  uint32_t k[8], top = 0;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    k[i] = rounded_v<ROUNDING>(v[i], draw[i]);
    top = max(top, k[i]);
    bad |= !(v[i] >= 0.0f && v[i] <= 0x1.fffffep+127f);
  }
  top = quad_max(bad ? 0xFFFu << 3 : top);
  e = min(max(top >> 3, kVMinExp), 254u);
  const int least = (int)(e - 31u) * 8;
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = v[i] == 0.0f ? 0 : min(max((int)k[i] - least, 1), 255);
  if (top >= 0xFFFu << 3) e = 255u;
  return make_uint2(pack4_codes8(c[0], c[1], c[2], c[3]), pack4_codes8(c[4], c[5], c[6], c[7]));
}
__device__ __forceinline__ void decode_v8(uint2 codes, uint32_t e, float (&v)[8]) {
  const uint32_t base = (e - 31u) * 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = (i < 4 ? codes.x >> (8 * i) : codes.y >> (8 * i - 32)) & 255u;
    v[i] = e == 255u ? __uint_as_float(0x7FC00000u) : c ? __uint_as_float((c + base) << 20) : 0.0f;
  }
}

__device__ __forceinline__ int64_t whole_blocks(int64_t n) { return (n + kStateBlock - 1) & -(int64_t)kStateBlock; }
__device__ __forceinline__ uint8_t* state_at(const void* s, int64_t i) {
  return (uint8_t*)s + (i / kStateBlock) * kStateBlockBytes + (i & (kStateBlock - 1));
}
__device__ __forceinline__ uint8_t* exp_at(const void* s, int64_t i) {
  return (uint8_t*)s + (i / kStateBlock) * kStateBlockBytes + kStateBlock + (i & (kStateBlock - 1)) / 32;
}

// ---- the step -------------------------------------------------------------------------------------
struct Scalars {
  float beta1, rest1, beta2, rest2, eps, step, root2, shrink, g_scale;
  uint32_t seed;
};

template <bool EIGHT, hot_rounding ROUNDING, class TP, class TG>
__device__ __forceinline__ void update8(const AdamWEntry& t, const Scalars& c, int64_t at) {
  const int n = (int)min((int64_t)8, t.n - at);
  if (EIGHT ? at >= whole_blocks(t.n) : n <= 0) return;   // 8 bits: all of the last block's codes are written
  float p[8], g[8], m[8], v[8];
  const Raw8<TP> rp = load8((const TP*)t.p + at, n);
  const Raw8<TG> rg = load8((const TG*)t.g + at, n);
  if constexpr (EIGHT) {
    const uint2 cm = *(const uint2*)state_at(t.m, at), cv = *(const uint2*)state_at(t.v, at);
    const uint32_t em = *exp_at(t.m, at), ev = *exp_at(t.v, at);
    decode8(cm, ckpt_step(em), m);
    decode_v8(cv, ev, v);
    if (rarely(n < 8)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= n) m[i] = v[i] = 0.0f;
    }
  } else {
    const Raw8<float> rm = load8((const float*)t.m + at, n), rv = load8((const float*)t.v + at, n);
    widen(rm, m);
    widen(rv, v);
  }
  widen(rp, p);
  widen(rg, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float gi = g[i] * c.g_scale;
    m[i] = m[i] * c.beta1 + gi * c.rest1;         // every operation rounded by itself: the codes of m' and v' rest on it
    v[i] = v[i] * c.beta2 + gi * c.rest2 * gi;
    const float move = m[i] / (sqrtf(v[i]) * c.root2 + c.eps);
    p[i] = p[i] - (p[i] * c.shrink + move * c.step);
  }
  if constexpr (EIGHT) {
    const uint32_t em = ckpt_exponent(quad_max(magnitude8(m)));
    uint32_t ev, draw[8]{};
    if constexpr (ROUNDING == HOT_ROUND_DRAWN) draw8(c.seed, at, m, v, draw);
    const uint2 cm = encode_m8<ROUNDING>(m, ckpt_inverse(em), draw), cv = store_v8<ROUNDING>(v, draw, ev);
    *(uint2*)state_at(t.m_out, at) = cm;
    *(uint2*)state_at(t.v_out, at) = cv;
    if ((at & 31) == 0) {
      *exp_at(t.m_out, at) = (uint8_t)em;
      *exp_at(t.v_out, at) = (uint8_t)ev;
    }
  } else {
    store8((float*)t.m_out + at, m, n);
    store8((float*)t.v_out + at, v, n);
  }
  store8((TP*)t.p_out + at, p, n);
  if (t.copy) store8((bf16*)t.copy + at, p, n);
}

template <bool EIGHT, hot_rounding ROUNDING>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamWArgs a) {
  uint32_t k = 0;
#pragma unroll
  for (int i = 1; i < kAdamWEntries; ++i) k += blockIdx.x >= a.block[i];
  const AdamWEntry& t = a.e[k];
  const int64_t at = (int64_t)(blockIdx.x - a.block[k]) * kAdamWChunk + (k == 0 ? a.first : 0) + threadIdx.x * 8;
  const float* const dyn = a.s.dyn;
  const float lr_all = dyn ? dyn[0] : a.s.lr, lr = lr_all * t.lr, corr1 = dyn ? dyn[1] : a.s.corr1, corr2 = dyn ? dyn[2] : a.s.corr2;
  Scalars c{a.s.beta1, a.s.rest1, a.s.beta2, a.s.rest2, a.s.eps, lr / corr1, 1.0f / sqrtf(corr2), t.decay * lr, dyn ? dyn[3] : 1.0f, 0};
  if constexpr (EIGHT && ROUNDING == HOT_ROUND_DRAWN) {
    c.seed = seed_with(seed_with(seed_with(0, __float_as_uint(lr_all)), __float_as_uint(corr1)), __float_as_uint(corr2));
    c.seed = seed_with(c.seed, !dyn ? a.s.word : a.s.words ? __float_as_uint(dyn[4]) : 0u);
  }
  if (t.types & 1u) {
    if (t.types & 2u) update8<EIGHT, ROUNDING, bf16, bf16>(t, c, at);
    else update8<EIGHT, ROUNDING, bf16, float>(t, c, at);
  } else {
    if (t.types & 2u) update8<EIGHT, ROUNDING, float, bf16>(t, c, at);
    else update8<EIGHT, ROUNDING, float, float>(t, c, at);
  }
}

// ---- moments as values -----------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(256) void state_read_kernel(const void* state, int second, int64_t first, int64_t n, T* out) {
  const int64_t at = first + ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= n) return;
  const uint2 c = *(const uint2*)state_at(state, at);
  const uint32_t e = *exp_at(state, at);
  float v[8];
  if (second) decode_v8(c, e, v);
  else decode8(c, ckpt_step(e), v);
  store8(out + at, v, (int)min((int64_t)8, n - at));
}

template <class T>
__global__ __launch_bounds__(256) void state_write_kernel(const T* x, int second, int64_t first, int64_t n, void* state) {
  const int64_t at = first + ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= whole_blocks(n)) return;
  float v[8];
  load_values(x + at, (int)min((int64_t)8, n - at), v);
  uint32_t e;
  uint2 c;
  const uint32_t draw[8]{};
  if (second) {
    c = store_v8<HOT_ROUND_NEAREST_EVEN>(v, draw, e);
  } else {
    e = ckpt_exponent(quad_max(magnitude8(v)));
    c = encode_m8<HOT_ROUND_NEAREST_EVEN>(v, ckpt_inverse(e), draw);
  }
  *(uint2*)state_at(state, at) = c;
  if ((at & 31) == 0) *exp_at(state, at) = (uint8_t)e;
}

}  // namespace

hipError_t launch_adamw(const AdamWArgs& a, uint32_t blocks, bool eight, hot_rounding rounding, hipStream_t s) {
  if (!eight) adamw_kernel<false, HOT_ROUND_NEAREST_EVEN><<<blocks, 256, 0, s>>>(a);
  else if (rounding == HOT_ROUND_NEAREST_EVEN) adamw_kernel<true, HOT_ROUND_NEAREST_EVEN><<<blocks, 256, 0, s>>>(a);
  else if (rounding == HOT_ROUND_DRAWN) adamw_kernel<true, HOT_ROUND_DRAWN><<<blocks, 256, 0, s>>>(a);
  else adamw_kernel<true, HOT_ROUND_PSEUDO_STOCHASTIC><<<blocks, 256, 0, s>>>(a);
  return hipGetLastError();
}

namespace {
constexpr int64_t kStateRun = 1ll << 33;   // elements of one launch: 2^30 lanes
}

hipError_t launch_state_read(const void* state, bool second, int64_t n, void* out, hot_type type, hipStream_t s) {
  for (int64_t first = 0; first < n; first += kStateRun) {
    const int64_t last = first + kStateRun < n ? first + kStateRun : n;
    const uint32_t blocks = (uint32_t)ceil_div(last - first, 2048);
    if (type == HOT_BF16) state_read_kernel<<<blocks, 256, 0, s>>>(state, second, first, last, (bf16*)out);
    else state_read_kernel<<<blocks, 256, 0, s>>>(state, second, first, last, (float*)out);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_state_write(const void* x, hot_type type, bool second, int64_t n, void* state, hipStream_t s) {
  for (int64_t first = 0; first < n; first += kStateRun) {
    const int64_t last = first + kStateRun < n ? first + kStateRun : n;
    const uint32_t blocks = (uint32_t)ceil_div(last - first, 2048);
    if (type == HOT_BF16) state_write_kernel<<<blocks, 256, 0, s>>>((const bf16*)x, second, first, last, state);
    else state_write_kernel<<<blocks, 256, 0, s>>>((const float*)x, second, first, last, state);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace hot
