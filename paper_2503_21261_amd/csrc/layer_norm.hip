// Layer norm over the columns of [rows x cols], forward and backward, up to 16384 columns.
//
//   h = x (+ residual), y = (h - mean) rstd gamma + beta;   with n = (h - mean) rstd, t = g_y gamma:
//   g_h = rstd (t - mean(t) - n mean(t n)) (+ g_residual),  g_gamma = sum over rows of g_y n,  g_beta = of g_y.
//
// Both are bound by HBM.  A row stays in the registers of the T lanes that work on it (eight columns a
// lane, NV times), so it is read once: the mean first, then the squares of what is left, which keeps the
// variance of rows whose mean is large.  The mean is summed in 64 bits, so that it is the exact one rounded
// once, and y takes off what that rounding left.  The backward pass keeps a lane on its columns, so that the
// parameter gradients are sums in registers; a workgroup leaves one row of them, and column_sums adds those in order.
// 201728 x 1024 fp32 with residual and checkpoint: 660 us forward, 500 back, 5.3 TB/s.
#include <type_traits>

#include "block_device.h"
#include "block_host.h"

namespace hot {

namespace {

__device__ __forceinline__ void anew(Raw8<float>& r) { asm volatile("" : "+v"(r.a), "+v"(r.b)); }
__device__ __forceinline__ void anew(Raw8<bf16>& r) { asm volatile("" : "+v"(r.a)); }
__device__ __forceinline__ void anew(uint2& c) { asm volatile("" : "+v"(c.x), "+v"(c.y)); }

template <int T>
constexpr int kThreads = T > 256 ? T : 256;
template <int T>
constexpr int kSlots = kThreads<T> / T;   // rows a workgroup works on at a time

// Sums of two values over the T lanes of a row, in every lane.  T > 64: through LDS, whose halves
// alternate (`turn`), so that one barrier a call is enough.
template <int T>
__device__ __forceinline__ void row_sums(float& a, float& b, float (*s_red)[16][2], int turn) {
  constexpr int W = T < 64 ? T : 64;
  a = lanes_sum<W>(a);
  b = lanes_sum<W>(b);
  if constexpr (T > 64) {
    const int wave = (int)threadIdx.x >> 6;
    if (((int)threadIdx.x & 63) == 0) {
      s_red[turn][wave][0] = a;
      s_red[turn][wave][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) {
      a += s_red[turn][i][0];
      b += s_red[turn][i][1];
    }
  }
}

// Sum of one value over the T lanes of a row, in every lane; s_red: the caller's own for each call.
template <int T, class V>
__device__ __forceinline__ V row_sum(V a, V* s_red) {
  a = lanes_sum<(T < 64 ? T : 64)>(a);
  if constexpr (T > 64) {
    if (((int)threadIdx.x & 63) == 0) s_red[(int)threadIdx.x >> 6] = a;
    __syncthreads();
    a = V(0);
#pragma unroll
    for (int i = 0; i < T / 64; ++i) a += s_red[i];
  }
  return a;
}

// EVEN: cols is a multiple of eight, so that a lane's chunk is whole or absent.
template <int T, int NV, class TX, class TY, bool KEEP, bool EVEN>
__global__ __launch_bounds__(kThreads<T>) void layer_norm_kernel(const NormForward a, const CkptView k, int64_t first) {
  __shared__ double s_sum[16];
  __shared__ float s_sq[16];
  const int lane = (int)threadIdx.x % T, slot = (int)threadIdx.x / T;
  const int64_t row = first + (int64_t)blockIdx.x * kSlots<T> + slot;
  if (row >= a.rows) return;   // T > 64: one row a workgroup, all of it or none
  const int cols = (int)a.cols;
  auto have = [&](int c) { return EVEN ? 8 : cols - c; };
  const int64_t at = row * cols;
  Raw8<TX> xr[NV], rr[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + j * T) * 8;
    if (c < cols) {
      xr[j] = load8((const TX*)a.x + at + c, have(c));
      if (a.residual) rr[j] = load8((const TX*)a.residual + at + c, have(c));
    }
  }
  float v[NV][8];
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + j * T) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
    if (c < cols) {
      widen(xr[j], v[j]);
      if (a.residual) {
        float r[8];
        widen(rr[j], r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = rounded(v[j][i] + r[i], TX(0.0f));
        if (a.h) store8((TX*)a.h + at + c, v[j], have(c));
      }
    }
    if constexpr (KEEP) {
      if (c < (int)k.pitch) ckpt_store8(k, row * k.pitch + c, v[j]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += (double)v[j][i];
  }
  // What the mean loses by its rounding (large beside the variance where |mean| is) is taken off the squares and off y.  Sums in
  // 32 bits lose more, and the mean of the deviations does not bring it back: they are rounded too (rows of 768 about zero: 1.0e-7 of
  // the mean in 32 bits, 2.4e-7 with that, 2.6e-8 in 64; 201728 x 1024 takes as long either way).
  const double exact = row_sum<T>(sum, s_sum) / (double)cols;
  const float mean0 = (float)exact, off = (float)(exact - (double)mean0);
  float sq = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int n = cols - (lane + j * T) * 8;
    if constexpr (EVEN) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = n > 0 ? v[j][i] - mean0 : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = i < n ? v[j][i] - mean0 : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sq = fmaf(v[j][i], v[j][i], sq);
  }
  sq = row_sum<T>(sq, s_sq);
  float var = fmaf(-off, off, sq / (float)cols);
  var = var < 0.0f ? 0.0f : var;   // a constant row, by rounding
  const float rstd = 1.0f / sqrtf(var + a.eps);
  if (lane == 0) {
    a.mean[row] = mean0;
    a.rstd[row] = rstd;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + j * T) * 8;
    if (c < cols) {
      float g[8], b[8];
      if (a.gamma) load_values(a.gamma + c, have(c), g);
      if (a.beta) load_values(a.beta + c, have(c), b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float n = (v[j][i] - off) * rstd;
        if (a.gamma) n *= g[i];
        if (a.beta) n += b[i];
        v[j][i] = n;
      }
      store8((TY*)a.y + at + c, v[j], have(c));
    }
  }
}

template <int T, int NV, class TX, class TY, bool KEPT, bool EVEN, bool STREAM>
__global__ __launch_bounds__(kThreads<T>) void layer_norm_grad_kernel(const NormBackward a, const CkptView k) {
  constexpr int SPAN = T * NV * 8;    // columns the lanes of a row cover
  __shared__ float s_red[2][16][2];
  __shared__ float s_sum[T < 256 ? kSlots<T> * SPAN : 1];
  const int lane = (int)threadIdx.x % T, slot = (int)threadIdx.x / T;
  const int cols = (int)a.cols;
  auto have = [&](int c) { return EVEN ? 8 : cols - c; };
  float gamma[NV][8], sg[NV][8], sb[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (lane + j * T) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sg[j][i] = sb[j][i] = 0.0f;
      gamma[j][i] = a.gamma ? 0.0f : 1.0f;
    }
    if (a.gamma && c < cols) load_values(a.gamma + c, have(c), gamma[j]);
  }
  const float inv = 1.0f / (float)cols;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kSlots<T> + slot; row < a.rows; row += (int64_t)gridDim.x * kSlots<T>) {
    const int64_t at = row * cols;
    Raw8<TY> gr[NV];
    Raw8<TX> hr[NV], ar[NV];
    uint2 codes[NV];
    uint32_t e[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + j * T) * 8;
      if (c < cols) {
        gr[j] = load8((const TY*)a.g_y + at + c, have(c));
        if constexpr (KEPT) {
          const int64_t kat = row * k.pitch + c;
          codes[j] = *(const uint2*)(k.codes + kat);
          e[j] = k.exps[kat / kCkGroup];
        } else {
          hr[j] = load8((const TX*)a.h + at + c, have(c));
        }
        if (a.g_residual) ar[j] = load8((const TX*)a.g_residual + at + c, have(c));
      }
    }
    const float mean = a.mean[row], rstd = a.rstd[row];
    // n and g_y of a chunk
    auto values = [&](int j, float(&n)[8], float(&t)[8]) {
      widen(gr[j], t);
      if constexpr (KEPT) decode8(codes[j], ckpt_step(e[j]), n);
      else widen(hr[j], n);
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = (n[i] - mean) * rstd;
    };
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + j * T) * 8;
      if (c < cols) {
        float n[8], t[8];
        values(j, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sb[j][i] += t[i];
          sg[j][i] = fmaf(t[i], n[i], sg[j][i]);
          t[i] *= gamma[j][i];
          s1 += t[i];
          s2 = fmaf(t[i], n[i], s2);
        }
      }
    }
    row_sums<T>(s1, s2, s_red, turn);
    turn ^= 1;
    const float m1 = s1 * inv, m2 = s2 * inv;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + j * T) * 8;
      if (c < cols) {
        // Once more from what was loaded: to keep them takes 160 registers where 1024 lanes have 128 each (16384 x 11008 bfloat16 from
        // a checkpoint 252 us, 898 with what spilled), and leaves fewer rows on their way.  As new values to the compiler, which
        // would keep them all the same.
        anew(gr[j]);
        if constexpr (KEPT) anew(codes[j]);
        else anew(hr[j]);
        float n[8], t[8], r[8];
        values(j, n, t);
        if (a.g_residual) widen(ar[j], r);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = rstd * (t[i] * gamma[j][i] - m1 - n[i] * m2);
          t[i] = a.g_residual ? g + r[i] : g;
        }
        store8<STREAM>((TX*)a.g_x + at + c, t, have(c));
      }
    }
  }
  if (!a.sum_gamma) return;
  float* const to_gamma = a.sum_gamma + (int64_t)blockIdx.x * a.sum_pitch;
  float* const to_beta = a.sum_beta + (int64_t)blockIdx.x * a.sum_pitch;
  if constexpr (T >= 256) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (lane + j * T) * 8;
      if (c < cols) {
        store8(to_gamma + c, sg[j], have(c));
        store8(to_beta + c, sb[j], have(c));
      }
    }
  } else {
    auto add_slots = [&](const float(&s)[NV][8], float* dst) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s_sum[slot * SPAN + (lane + j * T) * 8 + i] = s[j][i];
      __syncthreads();
      for (int c = (int)threadIdx.x; c < SPAN && c < cols; c += 256) {
        float total = 0.0f;
#pragma unroll
        for (int y = 0; y < kSlots<T>; ++y) total += s_sum[y * SPAN + c];
        dst[c] = total;
      }
      __syncthreads();
    };
    add_slots(sg, to_gamma);
    add_slots(sb, to_beta);
  }
}

// Lanes to a row: the fewest that hold it with eight or sixteen columns each.  The gradient's registers, three fp32 values a column and
// what was loaded, leave no room for more.
template <class F>
hipError_t with_lanes(int64_t cols, F&& f) {
  using std::integral_constant;
  if (cols <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (cols <= 256) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (cols <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (cols <= 1024) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (cols <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (cols <= 4096) return f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (cols <= 8192) return f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
int slots_of(int64_t cols) { return cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 1024 ? 4 : 1; }

template <class F>
hipError_t with_types(hot_type x, hot_type y, bool even, F&& f) {
  auto go = [&](auto e) {
    if (x == HOT_BF16) return f(bf16(0.0f), bf16(0.0f), e);
    if (y == HOT_BF16) return f(0.0f, bf16(0.0f), e);
    return f(0.0f, 0.0f, e);
  };
  return even ? go(std::true_type{}) : go(std::false_type{});
}

CkptView view(const void* ckpt, int64_t rows, int64_t cols) {
  const CkptLayout l = ckpt_layout(rows, cols);
  return CkptView{(uint8_t*)ckpt, (uint8_t*)ckpt + l.exps, l.pitch};
}

}  // namespace

// Workgroups of the backward pass, one row of partial sums each: one, whose sums are the gradients themselves, while its turns
// take no longer than a second launch; two a compute unit while rows are few; once every workgroup has eight turns, as many as are
// resident together, so that none waits for another to end: four of 256 lanes a compute unit.  With sixteen columns a lane fp32 rows
// do better with three (50432 x 1024 with g_residual 161 us, 169 with four), bfloat16 ones with four (40000 x 1000 52, 54 with three).
int layer_norm_sum_rows(int64_t rows, int64_t cols, hot_type x_type) {
  const int64_t turns = ceil_div(rows, slots_of(cols));
  if (turns <= 2) return 1;
  const bool wide = (cols > 512 && cols <= 1024) || cols > 2048;
  const int64_t resident = cols > 8192 ? 256 : cols > 4096 ? 512 : wide && x_type == HOT_F32 ? 768 : 1024;
  const int64_t few = resident < 512 ? resident : 512;
  const int64_t g = turns < few ? turns : few, many = turns / 8 < resident ? turns / 8 : resident;
  return (int)(many > g ? many : g);
}

hipError_t launch_layer_norm(const NormForward& a, hipStream_t s) {
  return with_lanes(a.cols, [&](auto t, auto nv) {
    return with_types(a.x_type, a.y_type, a.cols % 8 == 0, [&](auto tx, auto ty, auto e) {
      constexpr int T = decltype(t)::value, NV = decltype(nv)::value;
      constexpr bool EVEN = decltype(e)::value;
      using TX = decltype(tx);
      using TY = decltype(ty);
      constexpr int64_t kRun = kMaxLaunch / T;     // rows of a launch
      for (int64_t first = 0; first < a.rows; first += kRun) {
        const int64_t rows = a.rows - first < kRun ? a.rows - first : kRun;
        const dim3 grid((unsigned)ceil_div(rows, kSlots<T>)), block(kThreads<T>);
        if (a.ckpt) layer_norm_kernel<T, NV, TX, TY, true, EVEN><<<grid, block, 0, s>>>(a, view(a.ckpt, a.rows, a.cols), first);
        else layer_norm_kernel<T, NV, TX, TY, false, EVEN><<<grid, block, 0, s>>>(a, CkptView{}, first);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      }
      return hipSuccess;
    });
  });
}

hipError_t launch_layer_norm_grad(const NormBackward& a, hipStream_t s) {
  return with_lanes(a.cols, [&](auto t, auto nv) {
    return with_types(a.x_type, a.y_type, a.cols % 8 == 0, [&](auto tx, auto ty, auto e) {
      constexpr int T = decltype(t)::value, NV = decltype(nv)::value;
      constexpr bool EVEN = decltype(e)::value;
      using TX = decltype(tx);
      using TY = decltype(ty);
      const dim3 grid((unsigned)layer_norm_sum_rows(a.rows, a.cols, a.x_type)), block(kThreads<T>);
      auto launch = [&](auto stream) {
        constexpr bool STREAM = decltype(stream)::value;
        if (a.ckpt) layer_norm_grad_kernel<T, NV, TX, TY, true, EVEN, STREAM><<<grid, block, 0, s>>>(a, view(a.ckpt, a.rows, a.cols));
        else layer_norm_grad_kernel<T, NV, TX, TY, false, EVEN, STREAM><<<grid, block, 0, s>>>(a, CkptView{});
        return hipGetLastError();
      };
      if constexpr (EVEN && sizeof(TX) == 2) {    // as for the activation's gradient: 8192 x 4096 bfloat16 42 -> 38 us
        if (stream_output(a.rows, a.cols * (int64_t)sizeof(TX))) return launch(std::true_type{});
      }
      return launch(std::false_type{});
    });
  });
}

}  // namespace hot
