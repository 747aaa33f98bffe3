// Device-side helpers of the operators around the linear backward (8-bit checkpoints, activations,
// layer norm, forward product): vectors of eight elements, the 8-bit form, activation functions,
// sums over the columns' lanes.  gfx950, wave64.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hot.h"
#include "hot_device.h"

namespace hot {

// ---- eight consecutive elements of a row per lane ------------------------------------------------
// Rows of a tensor are contiguous but need not begin at a multiple of 16 bytes (odd widths), so the
// vector types carry their element's alignment only: the hardware loads and stores them whole.
typedef __bf16 bf16;
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t h8_any __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ float bf16_to_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
// To nearest even (the hardware's conversion).
__device__ __forceinline__ uint16_t float_to_bf16(float v) { return __builtin_bit_cast(uint16_t, (bf16)v); }

// What a load brings, before it is widened: kept apart so that several loads can be on their way.
template <class T> struct Raw8;
template <> struct Raw8<float> { f4_any a, b; };
template <> struct Raw8<bf16> { h8_any a; };

// n: how many of the eight exist (a row's last chunk may be short); the others read as zero.
__device__ __forceinline__ Raw8<float> load8(const float* p, int n) {
  Raw8<float> r;
  if (n >= 8) {
    r.a = *(const f4_any*)p;
    r.b = *(const f4_any*)(p + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.a[i] = i < n ? p[i] : 0.0f;
      r.b[i] = i + 4 < n ? p[i + 4] : 0.0f;
    }
  }
  return r;
}
__device__ __forceinline__ Raw8<bf16> load8(const bf16* p, int n) {
  Raw8<bf16> r;
  const uint16_t* q = (const uint16_t*)p;
  if (n >= 8) {
    r.a = *(const h8_any*)q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.a[i] = i < n ? q[i] : (uint16_t)0;
  }
  return r;
}
__device__ __forceinline__ void widen(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = r.a[i];
    v[i + 4] = r.b[i];
  }
}
__device__ __forceinline__ void widen(const Raw8<bf16>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = bf16_to_float(r.a[i]);
}
// STREAM: with the hint that nothing reads the values soon.
template <bool STREAM = false>
__device__ __forceinline__ void store8(float* p, const float (&v)[8], int n) {
  if (n >= 8) {
    f4_any a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = v[i];
      b[i] = v[i + 4];
    }
    if constexpr (STREAM) {
      __builtin_nontemporal_store(a, (f4_any*)p);
      __builtin_nontemporal_store(b, (f4_any*)(p + 4));
      asm volatile("");   // else this store and the plain one of another branch become one plain store
    } else {
      *(f4_any*)p = a;
      *(f4_any*)(p + 4) = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}
template <bool STREAM = false>
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8], int n) {
  uint16_t* q = (uint16_t*)p;
  if (n >= 8) {
    h8_any a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = float_to_bf16(v[i]);
    if constexpr (STREAM) {
      __builtin_nontemporal_store(a, (h8_any*)q);
      asm volatile("");
    } else {
      *(h8_any*)q = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) q[i] = float_to_bf16(v[i]);
  }
}
template <class T>
__device__ __forceinline__ void load_values(const T* p, int n, float (&v)[8]) { widen(load8(p, n), v); }
// The value a store to T leaves.
__device__ __forceinline__ float rounded(float v, float) { return v; }
__device__ __forceinline__ float rounded(float v, bf16) { return bf16_to_float(float_to_bf16(v)); }

// ---- the 8-bit form -------------------------------------------------------------------------------
// 32 consecutive columns of a row share a step 2^(e - 133): the smallest power of two (from 2^-125 on)
// that leaves the group's largest magnitude within 127 steps after rounding.  A power of two makes
// every operation but the rounding to a whole number exact, so the codes have one value whatever
// computes them.  e is one byte; 255 marks a group that held an infinity or a NaN, and reads as NaN.
constexpr int kCkGroup = 32;
constexpr int kCkMinExp = 8;

// bits: the largest bit pattern of |t| in the group.  127.5 steps or more would round to 128:
// mantissas from 1.9921875 on carry into the exponent.
__device__ __forceinline__ uint32_t ckpt_exponent(uint32_t bits) {
  const uint32_t e = (bits + 0x10000u) >> 23;
  const uint32_t c = min(max(e, (uint32_t)kCkMinExp), 254u);
  return bits >= 0x7F800000u ? 255u : c;
}
__device__ __forceinline__ float ckpt_step(uint32_t e) { return e == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((e - 6u) << 23); }
__device__ __forceinline__ float ckpt_inverse(uint32_t e) { return e == 255u ? 0.0f : __uint_as_float((260u - e) << 23); }

// Whether any lane of the wave meets a condition that hardly ever holds: a branch around what it takes, which the compiler would
// otherwise compute always and select from.
__device__ __forceinline__ bool rarely(bool condition) {
  if (__builtin_amdgcn_ballot_w64(condition) == 0) return false;
  asm volatile("");    // not to be moved in front of the branch
  return true;
}

// Maximum over the four lanes of a group (lane ids 4 k .. 4 k + 3) of a bit pattern.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));   // quad_perm [1,0,3,2]
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));   // quad_perm [2,3,0,1]
  return v;
}
// Bit patterns order as magnitudes do, and put infinities and NaNs on top.
__device__ __forceinline__ uint32_t magnitude8(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return m;
}
// Eight codes under 1 / step: the product is exact, and the addition of 1.5 x 2^23 rounds it to a whole number, half to even, in the
// sum's low bits, whose lowest byte is the code.
__device__ __forceinline__ uint2 encode8(const float (&v)[8], float inverse) {
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = __float_as_int(fmaf(v[i], inverse, 12582912.0f));
  return make_uint2(pack4_codes8(c[0], c[1], c[2], c[3]), pack4_codes8(c[4], c[5], c[6], c[7]));
}
__device__ __forceinline__ void decode8(uint2 codes, float step, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (float)(int8_t)(codes.x >> (8 * i)) * step;
    v[i + 4] = (float)(int8_t)(codes.y >> (8 * i)) * step;
  }
}

// A checkpoint in memory: rows x pitch codes (pitch: whole groups), then one exponent per group.
struct CkptView {
  uint8_t* codes;
  uint8_t* exps;
  int64_t pitch;
};
// `at`: row * pitch + column, a multiple of 8; called by all four lanes of a group together.
template <bool STREAM = false>
__device__ __forceinline__ void ckpt_store8(const CkptView& k, int64_t at, const float (&v)[8]) {
  const uint32_t e = ckpt_exponent(quad_max(magnitude8(v)));
  const float inverse = ckpt_inverse(e);
  const uint2 c = encode8(v, inverse);
  if constexpr (STREAM) {
    __builtin_nontemporal_store((uint64_t)c.y << 32 | c.x, (uint64_t*)(k.codes + at));
    asm volatile("");
  } else {
    *(uint2*)(k.codes + at) = c;
  }
  if (rarely(e == 254u)) {   // at the type's end, where the next step is missing: 127.5 steps and more are held at 127
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = fminf(fmaxf(v[i], -0x1.fcp+127f), 0x1.fcp+127f);
    if (e == 254u) *(uint2*)(k.codes + at) = encode8(w, inverse);
  }
  if ((at & (kCkGroup - 1)) == 0) k.exps[at / kCkGroup] = (uint8_t)e;
}

// ---- activations ----------------------------------------------------------------------------------
// Phi(-a) = e^(-a^2 / 2) Q(a) for a >= 0; Q is fitted by a polynomial of t = 1 / (1 + 0.3 a) that
// minimises the largest relative error (1.5e-7, 4e-7 in fp32), so the tails of GELU keep their
// relative accuracy, which 1 + erf(x) loses.
__device__ __forceinline__ float normal_tail(float a, float gauss) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, a, 1.0f));
  float p = 0.03567494452f;
  p = fmaf(p, t, -0.157203719f);
  p = fmaf(p, t, 0.206354484f);
  p = fmaf(p, t, -0.05368447304f);
  p = fmaf(p, t, 0.1285620332f);
  p = fmaf(p, t, 0.09991338104f);
  p = fmaf(p, t, 0.1207539737f);
  p = fmaf(p, t, 0.1196293011f);
  return gauss * (p * t);
}
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float gauss_of(float x) { return __builtin_amdgcn_exp2f(x * x * -0.72134752044448170f); }
__device__ __forceinline__ float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_fast(-x)); }

__device__ __forceinline__ float clamp10(float x) { return x < -10.0f ? -10.0f : (x > 10.0f ? 10.0f : x); }   // a NaN stays one

// 2 sqrt(2 / pi) (x + 0.044715 x^3), the argument whose sigmoid the tanh form multiplies x by.
__device__ __forceinline__ float gelu_tanh_arg(float xc) { return xc * fmaf(xc * xc, 0.0713548162726f, 1.5957691216057f); }

template <int FN>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (FN == HOT_ACT_RELU) return x < 0.0f ? 0.0f : x;
  else if constexpr (FN == HOT_ACT_GELU) {
    // The tail of +inf is zero: times a number, so that x Phi(x) is infinite there.  Minimum and maximum of the bit patterns, one
    // instruction each: floats would be made quiet first.  A NaN stays one by its tail.
    const int bits = __float_as_int(x);
    const float held = __int_as_float(min(bits, 0x71800000)), positive = __int_as_float(max(bits, 0));
    return fmaf(-fabsf(held), normal_tail(fabsf(x), gauss_of(x)), positive);
  } else if constexpr (FN == HOT_ACT_GELU_TANH) {
    // the argument in powers of two; a NaN that the clamp loses is one by the last product
    const float xc = __builtin_amdgcn_fmed3f(x, -30.0f, 30.0f);
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(xc * fmaf(xc * xc, -0.1029432396f, -2.3022081985f)));
  } else if constexpr (FN == HOT_ACT_SILU) return x * sigmoid_of(x);
  else return x;
}
template <int FN>
__device__ __forceinline__ float act_slope(float x) {
  if constexpr (FN == HOT_ACT_RELU) return x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;   // a NaN (a group that held one, too) stays one
  else if constexpr (FN == HOT_ACT_GELU) {
    const float a = fabsf(x), g = gauss_of(x), tail = normal_tail(a, g);
    return fmaf(x * g, 0.39894228040143f, x < 0.0f ? tail : 1.0f - tail);
  } else if constexpr (FN == HOT_ACT_GELU_TANH) {
    // Beyond |x| = 10 the slope is 0 or 1 to 1e-36; within, e is finite.  1 - s is e s, which keeps what a difference loses near s = 1: the
    // slope is off by 1e-6 at x = 5 with that, 2e-7 so.
    const float xc = clamp10(x), e = exp_fast(-gelu_tanh_arg(xc)), s = __builtin_amdgcn_rcpf(1.0f + e);
    return fmaf(xc * s * (e * s), fmaf(xc * xc, 3.0f * 0.0713548162726f, 1.5957691216057f), s);
  } else if constexpr (FN == HOT_ACT_SILU) {
    const float s = sigmoid_of(x);
    return s * fmaf(x, 1.0f - s, 1.0f);
  } else return 1.0f;
}

// ---- sums -----------------------------------------------------------------------------------------
template <int MASK>
__device__ __forceinline__ double lane_xor(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __float_as_uint(lane_xor<MASK>(__uint_as_float((uint32_t)b)));
  const uint32_t hi = __float_as_uint(lane_xor<MASK>(__uint_as_float((uint32_t)(b >> 32))));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int MASK>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) { return __float_as_uint(lane_xor<MASK>(__uint_as_float(v))); }
// Sum over T consecutive lanes (T a power of two up to 64), in every one of them; float or double.
template <int T, class V>
__device__ __forceinline__ V lanes_sum(V v) {
  if constexpr (T >= 2) v += lane_xor<1>(v);
  if constexpr (T >= 4) v += lane_xor<2>(v);
  if constexpr (T >= 8) v += lane_xor<4>(v);
  if constexpr (T >= 16) v += lane_xor<8>(v);
  if constexpr (T >= 32) v += lane_xor<16>(v);
  if constexpr (T >= 64) v += lane_xor<32>(v);
  return v;
}

}  // namespace hot
