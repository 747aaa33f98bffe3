// Point-wise operators over [rows x cols]: the 8-bit checkpoint and its reading, activations and their
// gradients (with the bias gradient, a sum over the rows), and the addition of partial column sums.
//
// All are bound by HBM: a pass reads and writes each element once.  A lane holds eight consecutive
// columns of a row (a 32-column group of the 8-bit form is four lanes, so its maximum is two DPP
// permutes), TX lanes a segment of a row, 256 / TX rows a workgroup at a time.  The walk is two-dimensional
// so that odd widths need no division per element and a lane keeps its columns for the column sums.
// SiLU, its gradient and the bias's of 16384 x 11008 bfloat16 334 us, 5.4 TB/s; a checkpoint of 12608 x 768 fp32 written and read 20 us.
#include <type_traits>

#include "block_device.h"
#include "block_host.h"

namespace hot {

namespace {

struct Walk {
  int64_t rows;
  int cols, chunks;    // chunks of eight columns, whole groups: 4 * ceil(cols / 32)
  int log_tx;          // lanes along a row: 1 << log_tx
  int col_tiles;
  int row_groups;      // of 256 / TX rows at a time; a group takes every row_groups-th batch
  int64_t batches;     // of 256 / TX * kRowsAtOnce rows
};

// The widest segment of a row that leaves at most an eighth of the lanes without columns; at most 16 lanes where the last
// segment is short and so takes the masked path (40251 x 946 bfloat16, GELU, gradient: 61 us with 16, 69 with 64).
int pick_log_tx(int64_t cols, int64_t chunks) {
  for (int l = cols % 32 ? 4 : 6; l > 2; --l)
    if (round_up(chunks, 1 << l) * 8 <= chunks * 9) return l;
  return 2;
}

constexpr int kRowsAtOnce = 4;   // rows of a lane whose loads are on their way together

Walk make_walk(int64_t rows, int64_t cols) {
  Walk w;
  w.rows = rows;
  w.cols = (int)cols;
  w.chunks = (int)(ceil_div(cols, 32) * 4);
  w.log_tx = pick_log_tx(cols, w.chunks);
  w.col_tiles = (int)ceil_div(w.chunks, 1 << w.log_tx);
  w.batches = ceil_div(rows, (int64_t)(256 >> w.log_tx) * kRowsAtOnce);
  w.row_groups = 0;
  return w;
}

// Row groups of a walk that keeps sums: at most a few workgroups per compute unit, and enough rows for
// each that the partial sums stay small beside the tensor.
int sum_groups(const Walk& w) {
  if (w.batches <= 2) return 1;     // no second launch for sums that one workgroup has
  const int64_t fill = ceil_div(4096, w.col_tiles);
  int64_t g = w.batches < fill ? w.batches : fill;
  return (int)(g > kMaxSumRows ? kMaxSumRows : g);
}

struct Position {
  int chunk, n;          // chunk of the row, elements of it that exist (may be negative)
  int64_t row;           // first row of the workgroup's first batch for this lane
};
__device__ __forceinline__ bool position(const Walk& w, Position& p, int& tx, int& ty, int& ct, int& rg) {
  const int b = (int)blockIdx.x;
  ct = b % w.col_tiles;
  rg = b / w.col_tiles;
  tx = (int)threadIdx.x & ((1 << w.log_tx) - 1);
  ty = (int)threadIdx.x >> w.log_tx;
  p.chunk = (ct << w.log_tx) + tx;
  p.n = w.cols - p.chunk * 8;
  return p.chunk < w.chunks;
}

__device__ __forceinline__ CkptView view_of(void* ckpt, int64_t rows, int chunks) {
  CkptView k;
  k.pitch = (int64_t)chunks * 8;
  k.codes = (uint8_t*)ckpt;
  k.exps = (uint8_t*)ckpt + (rows * k.pitch + 255) / 256 * 256;
  return k;
}

// Calls f with true_type where every row of a batch and every column of the workgroup's tile exist (the same in all its lanes, so
// that this path has no masks: a tenth of the time), else with false_type.
template <class F>
__device__ __forceinline__ void whole_or_not(const Walk& w, int ct, int64_t batch, int step, F&& f) {
  if ((ct + 1) << (w.log_tx + 3) <= w.cols && (batch + 1) * step * kRowsAtOnce <= w.rows) f(std::true_type{});
  else f(std::false_type{});
}

// y = f(x), the checkpoint of x, or both, from one read of x.
template <class T, int FN, bool VALUE, bool KEEP, bool STREAM>
__global__ __launch_bounds__(256) void activation_kernel(const T* x, Walk w, T* y, void* ckpt) {
  Position p;
  int tx, ty, ct, rg;
  if (!position(w, p, tx, ty, ct, rg)) return;
  const int step = 256 >> w.log_tx;
  const int64_t row0 = (int64_t)rg * step * kRowsAtOnce + ty;
  const int64_t col = (int64_t)p.chunk * 8;
  const CkptView k = view_of(ckpt, w.rows, w.chunks);
  whole_or_not(w, ct, rg, step, [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int n = WHOLE ? 8 : p.n;
    Raw8<T> raw[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const int64_t row = row0 + (int64_t)i * step;
      if (WHOLE || row < w.rows) raw[i] = load8(x + row * w.cols + col, n);
    }
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const int64_t row = row0 + (int64_t)i * step;
      if (WHOLE || row < w.rows) {
        float v[8];
        widen(raw[i], v);
        if constexpr (KEEP) ckpt_store8<STREAM>(k, row * k.pitch + col, v);
        if constexpr (VALUE) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = act_value<FN>(v[j]);
          store8<STREAM>(y + row * w.cols + col, v, n);
        }
      }
    }
  });
}

template <class T, bool STREAM>
__global__ __launch_bounds__(256) void checkpoint_read_kernel(const uint8_t* ckpt, Walk w, T* x) {
  Position p;
  int tx, ty, ct, rg;
  if (!position(w, p, tx, ty, ct, rg)) return;
  const int step = 256 >> w.log_tx;
  const int64_t row0 = (int64_t)rg * step * kRowsAtOnce + ty;
  const int64_t col = (int64_t)p.chunk * 8;
  const CkptView k = view_of(const_cast<uint8_t*>(ckpt), w.rows, w.chunks);
  whole_or_not(w, ct, rg, step, [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int n = WHOLE ? 8 : p.n;
    uint2 codes[kRowsAtOnce];
    uint32_t e[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const int64_t row = row0 + (int64_t)i * step;
      if (WHOLE || row < w.rows) {
        const int64_t at = row * k.pitch + col;
        codes[i] = *(const uint2*)(k.codes + at);
        e[i] = k.exps[at / kCkGroup];
      }
    }
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const int64_t row = row0 + (int64_t)i * step;
      if (WHOLE || row < w.rows) {
        float v[8];
        decode8(codes[i], ckpt_step(e[i]), v);
        store8<STREAM>(x + row * w.cols + col, v, n);
      }
    }
  });
}

// g_x = g_y f'(x); SUMS: a row of partial sums of g_x (in fp32, before it is rounded to T) per row group.
template <class T, int FN, bool KEPT, bool SUMS, bool STREAM>
__global__ __launch_bounds__(256) void activation_grad_kernel(const T* g_y, const T* x, const uint8_t* ckpt, Walk w, T* g_x,
                                                              float* partials, int64_t pitch) {
  __shared__ float s_sum[SUMS ? 256 * 8 : 1];
  Position p;
  int tx, ty, ct, rg;
  const bool active = position(w, p, tx, ty, ct, rg);
  const int step = 256 >> w.log_tx;
  const CkptView k = view_of(const_cast<uint8_t*>(ckpt), w.rows, w.chunks);
  const int64_t col = (int64_t)p.chunk * 8;
  float sum[8] = {};
  if (active) {
    for (int64_t batch = rg; batch < w.batches; batch += w.row_groups) {
      const int64_t row0 = batch * step * kRowsAtOnce + ty;
      whole_or_not(w, ct, batch, step, [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int n = WHOLE ? 8 : p.n;
        Raw8<T> gr[kRowsAtOnce], xr[kRowsAtOnce];
        uint2 codes[kRowsAtOnce];
        uint32_t e[kRowsAtOnce];
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
          const int64_t row = row0 + (int64_t)i * step;
          if (WHOLE || row < w.rows) {
            gr[i] = load8(g_y + row * w.cols + col, n);
            if constexpr (KEPT) {
              const int64_t at = row * k.pitch + col;
              codes[i] = *(const uint2*)(k.codes + at);
              e[i] = k.exps[at / kCkGroup];
            } else {
              xr[i] = load8(x + row * w.cols + col, n);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
          const int64_t row = row0 + (int64_t)i * step;
          if (WHOLE || row < w.rows) {
            float v[8], g[8];
            if constexpr (KEPT) decode8(codes[i], ckpt_step(e[i]), v);
            else widen(xr[i], v);
            widen(gr[i], g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              g[j] *= act_slope<FN>(v[j]);
              if constexpr (SUMS) sum[j] += g[j];
            }
            store8<STREAM>(g_x + row * w.cols + col, g, n);
          }
        }
      });
    }
  }
  if constexpr (SUMS) {
    // the workgroup's 256 / TX sums of a column, in row order
#pragma unroll
    for (int j = 0; j < 8; ++j) s_sum[threadIdx.x * 8 + j] = sum[j];
    __syncthreads();
    const int width = 8 << w.log_tx;
    for (int c = (int)threadIdx.x; c < width; c += 256) {
      const int at = ct * width + c;
      if (at >= w.cols) break;
      float total = 0.0f;
      for (int y = 0; y < step; ++y) total += s_sum[y * width + c];
      partials[(int64_t)rg * pitch + at] = total;
    }
  }
}

// 32 columns a workgroup, 32 rows of partial sums at a time: one or two memory round trips.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* partials, int rows, int64_t width, int cols, float* out,
                                                           float* out2) {
  __shared__ float s[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const bool second = blockIdx.y != 0;
  float* const dst = second ? out2 : out;
  if (!dst) return;
  const int c = (int)blockIdx.x * 32 + tx;
  const float* src = partials + (second ? width / 2 : 0) + c;
  float a = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int r = ty; r < rows; r += 32) a += src[(int64_t)r * width];
  }
  s[ty][tx] = a;
  __syncthreads();
  // lane = partial row, so that the wave adds 32 of them by permutes: columns ty, in both halves
  float v = s[tx][ty];
  v = lanes_sum<32>(v);
  const int oc = (int)blockIdx.x * 32 + ty;
  if (tx == 0 && oc < cols) dst[oc] = v;
}

// f(true_type) for outputs that are stored with the streaming hint.  Cold tensors of 16384 x 11008 bfloat16: SiLU with checkpoint 168 -> 160
// us, its gradient 165 -> 159, checkpoint read 94 -> 89; with rows that end inside a line (100000 x 1000) the read takes 102 instead of 64.
// Not for fp32, whose eight columns a lane are two stores that each leave half a line to the other: 201728 x 1024 350 us, 450 with it.
template <class T, class F>
hipError_t with_stream(int64_t rows, int64_t cols, F&& f) {
  if constexpr (sizeof(T) == 2) {
    if (stream_output(rows, cols * (int64_t)sizeof(T))) return f(std::true_type{});
  }
  return f(std::false_type{});
}

template <class T, int FN>
hipError_t activation_typed(const T* x, int64_t rows, int64_t cols, T* y, void* ckpt, hipStream_t s) {
  const Walk w = make_walk(rows, cols);
  const dim3 grid((unsigned)(w.col_tiles * w.batches)), block(256);
  return with_stream<T>(rows, cols, [&](auto stream) {
    constexpr bool STREAM = decltype(stream)::value;
    if (y && ckpt) activation_kernel<T, FN, true, true, STREAM><<<grid, block, 0, s>>>(x, w, y, ckpt);
    else if (y) activation_kernel<T, FN, true, false, STREAM><<<grid, block, 0, s>>>(x, w, y, nullptr);
    else activation_kernel<T, HOT_ACT_NONE, false, true, STREAM><<<grid, block, 0, s>>>(x, w, nullptr, ckpt);
    return hipGetLastError();
  });
}

template <class T, int FN>
hipError_t grad_typed(const T* g_y, const T* x, const void* ckpt, int64_t rows, int64_t cols, T* g_x, float* partials,
                      int64_t pitch, hipStream_t s) {
  Walk w = make_walk(rows, cols);
  const uint8_t* k = (const uint8_t*)ckpt;
  auto go = [&](auto sums, dim3 grid) {
    constexpr bool SUMS = decltype(sums)::value;
    return with_stream<T>(rows, cols, [&](auto stream) {
      constexpr bool STREAM = decltype(stream)::value;
      if (k) activation_grad_kernel<T, FN, true, SUMS, STREAM><<<grid, dim3(256), 0, s>>>(g_y, x, k, w, g_x, partials, pitch);
      else activation_grad_kernel<T, FN, false, SUMS, STREAM><<<grid, dim3(256), 0, s>>>(g_y, x, k, w, g_x, partials, pitch);
      return hipGetLastError();
    });
  };
  if (partials) {
    w.row_groups = sum_groups(w);
    const dim3 grid((unsigned)(w.col_tiles * w.row_groups));
    return go(std::true_type{}, grid);
  }
  w.row_groups = (int)w.batches;
  return go(std::false_type{}, dim3((unsigned)(w.col_tiles * w.batches)));
}

template <class F>
hipError_t with_fn(int fn, F&& f) {
  switch (fn) {
    case HOT_ACT_RELU: return f(std::integral_constant<int, HOT_ACT_RELU>{});
    case HOT_ACT_GELU: return f(std::integral_constant<int, HOT_ACT_GELU>{});
    case HOT_ACT_GELU_TANH: return f(std::integral_constant<int, HOT_ACT_GELU_TANH>{});
    case HOT_ACT_SILU: return f(std::integral_constant<int, HOT_ACT_SILU>{});
  }
  return f(std::integral_constant<int, HOT_ACT_NONE>{});
}

}  // namespace

int activation_sum_rows(int64_t rows, int64_t cols) { return sum_groups(make_walk(rows, cols)); }

hipError_t launch_activation(int fn, const void* x, hot_type type, int64_t rows, int64_t cols, void* y, void* ckpt,
                             hipStream_t s) {
  return with_fn(fn, [&](auto f) {
    if (type == HOT_BF16) return activation_typed<bf16, decltype(f)::value>((const bf16*)x, rows, cols, (bf16*)y, ckpt, s);
    return activation_typed<float, decltype(f)::value>((const float*)x, rows, cols, (float*)y, ckpt, s);
  });
}

hipError_t launch_checkpoint_read(const void* ckpt, int64_t rows, int64_t cols, void* x, hot_type type, hipStream_t s) {
  const Walk w = make_walk(rows, cols);
  const dim3 grid((unsigned)(w.col_tiles * w.batches)), block(256);
  if (type == HOT_BF16)
    return with_stream<bf16>(rows, cols, [&](auto stream) {
      checkpoint_read_kernel<bf16, decltype(stream)::value><<<grid, block, 0, s>>>((const uint8_t*)ckpt, w, (bf16*)x);
      return hipGetLastError();
    });
  checkpoint_read_kernel<float, false><<<grid, block, 0, s>>>((const uint8_t*)ckpt, w, (float*)x);
  return hipGetLastError();
}

hipError_t launch_activation_grad(int fn, const void* g_y, hot_type type, const void* x, const void* ckpt, int64_t rows,
                                  int64_t cols, void* g_x, float* partials, int64_t pitch, hipStream_t s) {
  return with_fn(fn, [&](auto f) {
    if (type == HOT_BF16)
      return grad_typed<bf16, decltype(f)::value>((const bf16*)g_y, (const bf16*)x, ckpt, rows, cols, (bf16*)g_x, partials, pitch, s);
    return grad_typed<float, decltype(f)::value>((const float*)g_y, (const float*)x, ckpt, rows, cols, (float*)g_x, partials, pitch, s);
  });
}

hipError_t launch_column_sums(const float* partials, int rows, int64_t width, int64_t cols, float* out, float* out2,
                              hipStream_t s) {
  column_sums_kernel<<<dim3((unsigned)ceil_div(cols, 32), out2 ? 2 : 1), dim3(1024), 0, s>>>(partials, rows, width, (int)cols, out,
                                                                                          out2);
  return hipGetLastError();
}

}  // namespace hot
