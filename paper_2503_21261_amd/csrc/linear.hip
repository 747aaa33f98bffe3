// Forward product of a linear layer, y = f(x.w^T + bias) + residual.
//
// linear_rows_kernel: few rows.  The weight is read once and is what bounds it (HBM): operands go from memory to the
// matrix instructions without LDS, every wave of a workgroup takes its part of K, and the waves' sums are added in
// LDS, in order.  A lane loads 16 consecutive bytes of a row; bfloat16 rows feed v_mfma_f32_16x16x32_bf16, fp32 rows
// four v_mfma_f32_16x16x4_f32, whose products and sums are plain fp32.  The weight is the first operand, so that a
// lane's accumulators are four consecutive outputs of a token.
#include "block_host.h"
#include "linear_device.h"

namespace hot {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// 16 bytes of a row: eight bfloat16 or four fp32.
template <class T> struct Frag;
template <> struct Frag<bf16> {
  static constexpr int kElems = 8;
  h8_any v;
};
template <> struct Frag<float> {
  static constexpr int kElems = 4;
  f4_any v;
};
// have: elements of the row from p on
__device__ __forceinline__ Frag<bf16> load_frag(const bf16* p, int64_t have) {
  Frag<bf16> f;
  if (have >= 8) {
    f.v = *(const h8_any*)p;
  } else {
    const uint16_t* q = (const uint16_t*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = i < have ? q[i] : (uint16_t)0;
  }
  return f;
}
__device__ __forceinline__ Frag<float> load_frag(const float* p, int64_t have) {
  Frag<float> f;
  if (have >= 4) {
    f.v = *(const f4_any*)p;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = i < have ? p[i] : 0.0f;
  }
  return f;
}
__device__ __forceinline__ v4f multiply(const Frag<bf16>& a, const Frag<bf16>& b, v4f acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a.v), __builtin_bit_cast(v8bf, b.v), acc, 0, 0, 0);
}
__device__ __forceinline__ v4f multiply(const Frag<float>& a, const Frag<float>& b, v4f acc) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], acc, 0, 0, 0);
  return acc;
}

constexpr int kWaves = 8;       // of a workgroup: parts of K
constexpr int kSteps = 4;       // loads of a row on their way together: 4 x 64 bytes

// NT x 16 outputs and MT x 16 tokens a workgroup.
template <class T, class TY, int NT, int MT>
__global__ __launch_bounds__(64 * kWaves) void linear_rows_kernel(const T* x, const T* w, int64_t I, int tiles_m, LinearOut out) {
  constexpr int E = Frag<T>::kElems;
  constexpr int STEP = 4 * E;               // elements of K in one matrix step (64 bytes of a row)
  constexpr int NC = NT * 16, MC = MT * 16;
  constexpr int PITCH = NC + 4;             // of a token's sums in LDS: rows apart by a multiple of 4 banks, not of 16
  __shared__ __align__(16) float s_sum[kWaves * MC * PITCH];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int tm = (int)blockIdx.x % tiles_m, tn = (int)blockIdx.x / tiles_m;
  const int64_t m0 = (int64_t)tm * MC;
  const int n0 = tn * NC;
  const T* wr[NT];
  const T* xr[MT];
  const int ke = (lane >> 4) * E;           // first element of the lane within a step
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int r = n0 + j * 16 + (lane & 15);
    wr[j] = w + (int64_t)(r < out.O ? r : out.O - 1) * I;   // rows past the last repeat it and are not stored
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t r = m0 + i * 16 + (lane & 15);
    xr[i] = x + (r < out.L ? r : out.L - 1) * I;
  }
  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0, 0, 0, 0};

  constexpr int SPAN = STEP * kSteps;       // of a wave at a time; the waves' spans follow each other
  for (int64_t k0 = (int64_t)wave * SPAN; k0 < I; k0 += (int64_t)kWaves * SPAN) {
    Frag<T> fw[kSteps][NT], fx[kSteps][MT];
    if (k0 + SPAN <= I) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
#pragma unroll
        for (int j = 0; j < NT; ++j) fw[s][j] = load_frag(wr[j] + k0 + s * STEP + ke, E);
#pragma unroll
        for (int i = 0; i < MT; ++i) fx[s][i] = load_frag(xr[i] + k0 + s * STEP + ke, E);
      }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int64_t k = k0 + s * STEP + ke;
#pragma unroll
        for (int j = 0; j < NT; ++j) fw[s][j] = load_frag(wr[j] + k, I - k);
#pragma unroll
        for (int i = 0; i < MT; ++i) fx[s][i] = load_frag(xr[i] + k, I - k);
      }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = multiply(fw[s][j], fx[s][i], acc[i][j]);
  }
  // accumulator register v of a tile: output 4 (lane / 16) + v, token lane % 16
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *(v4f*)&s_sum[(wave * MC + i * 16 + (lane & 15)) * PITCH + j * 16 + 4 * (lane >> 4)] = acc[i][j];
  __syncthreads();
  constexpr int CH = NC / 8;                // chunks of eight outputs of a token
  for (int q = (int)threadIdx.x; q < MC * CH; q += 64 * kWaves) {
    const int t = q / CH, c = q % CH * 8;
    if (m0 + t >= out.L) break;
    float v[8] = {};
#pragma unroll
    for (int z = 0; z < kWaves; ++z) {
      const v4f a = *(const v4f*)&s_sum[(z * MC + t) * PITCH + c], b = *(const v4f*)&s_sum[(z * MC + t) * PITCH + c + 4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] += a[e];
        v[e + 4] += b[e];
      }
    }
    linear_finish8<TY>(out, m0 + t, n0 + c, out.O - n0 - c, v);
  }
}

template <class T, class TY, int NT>
hipError_t rows_typed(const LinearForward& a, const LinearOut& o, hipStream_t s) {
  const int64_t tn = ceil_div(a.O, NT * 16);
  auto go = [&](auto mt) {
    constexpr int MT = decltype(mt)::value;
    const int64_t tm = ceil_div(a.L, MT * 16);
    linear_rows_kernel<T, TY, NT, MT><<<dim3((unsigned)(tm * tn)), dim3(64 * kWaves), 0, s>>>((const T*)a.x, (const T*)a.w, a.I,
                                                                                            (int)tm, o);
    return hipGetLastError();
  };
  if (a.L <= 16) return go(std::integral_constant<int, 1>{});
  if (a.L <= 32) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

template <class T, class TY>
hipError_t linear_typed(const LinearForward& a, hipStream_t s) {
  LinearOut o{a.bias, a.residual, a.y, CkptView{}, a.L, (int)a.O, a.fn};
  if (a.ckpt) {
    const CkptLayout l = ckpt_layout(a.L, a.O);
    o.k = CkptView{(uint8_t*)a.ckpt, (uint8_t*)a.ckpt + l.exps, l.pitch};
  }
  // 16 outputs a workgroup where that is what fills the card; a checkpoint's groups need 32
  stage_begin(kStLinear, s);
  const hipError_t e = a.ckpt || ceil_div(a.O, 32) * ceil_div(a.L, 64) >= 512 ? rows_typed<T, TY, 2>(a, o, s) : rows_typed<T, TY, 1>(a, o, s);
  stage_end(kStLinear, s);
  return e;
}

}  // namespace

size_t linear_scratch_bytes(hot_type, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_linear(const LinearForward& a, hipStream_t s) {
  if (a.type == HOT_F32) return linear_typed<float, float>(a, s);
  if (a.y_type == HOT_F32) return linear_typed<bf16, float>(a, s);
  return linear_typed<bf16, bf16>(a, s);
}

}  // namespace hot
