// Low-rank adapters beside a shared projection, each row with the adapter k of its request:
//   u = x A_k^T,  y = base + s_k u B_k^T;   g_u = s_k g_y B_k,  g_x = g_base + g_u A_k,
//   g_A_k = sum of g_u^T x,  g_B_k = s_k sum of g_y^T u  over the adapter's rows.
//
// Bound by memory: with a rank of some tens, x, g_y and the outputs are read or written for two operations a rank and element.  Three
// kernels, all on the matrix cores, none with a library call:
//   shrink  [rows x K] . [rank x K]^T -> [rows x rank]: a wave holds 32 rows (or one) and all ranks, K in slices where rows are few;
//   expand  [rows x rank] . [N x rank]^T -> [rows x N]: the ranks' factors of the rows stay in registers, columns go by;
//   outer   [rows x rank]^T . [rows x N] -> [rank x N]: rows as they lie are transposed in registers, 8 x 8 values a lane.
// u and g_u are fp32.  Where they meet bfloat16 operands they are split into bfloat16 parts, cut off and not rounded, so that three
// parts are the number itself: three for fp32 results (g_A, g_B), two (2^-16) for bfloat16 ones.
#include "adapter_host.h"
#include "block_device.h"
#include "block_host.h"

namespace hot {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements of the reduced dimension: lane (i, q) = (id % 16, id / 16) of a matrix instruction holds those from 8 q on
// of row i.  Both operands number the reduced elements alike, which is all that counts.
template <class T> struct Frag;
template <> struct Frag<bf16> { u4 v; };
template <> struct Frag<float> { float v[8]; };

__device__ __forceinline__ f4 mma(const Frag<bf16>& a, const Frag<bf16>& b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a.v), __builtin_bit_cast(b8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f4 mma(const Frag<float>& a, const Frag<float>& b, f4 c) {
#pragma unroll
  for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[t], b.v[t], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ Frag<bf16> frag(const Raw8<bf16>& r) { return Frag<bf16>{__builtin_bit_cast(u4, r.a)}; }
__device__ __forceinline__ Frag<float> frag(const Raw8<float>& r) {
  Frag<float> f;
  widen(r, f.v);
  return f;
}

// Parts of eight fp32 numbers as bfloat16: the upper 16 bits, then those of what is left.  An infinity or a NaN is whole in the first.
template <int PARTS>
__device__ __forceinline__ void split8(const float (&v)[8], Frag<bf16> (&out)[PARTS]) {
  float left[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) left[i] = v[i];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    uint32_t bits[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(left[i]);
      if (p == 0) {
        const bool finite = (b & 0x7F800000u) != 0x7F800000u;
        bits[i] = (b & 0x7FFFFFFFu) > 0x7F800000u ? b | 0x400000u : b;      // a NaN that the cut leaves one
        left[i] = finite ? left[i] - __uint_as_float(b & 0xFFFF0000u) : 0.0f;
      } else {
        bits[i] = b;
        left[i] = left[i] - __uint_as_float(b & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out[p].v[i] = __builtin_amdgcn_perm(bits[2 * i + 1], bits[2 * i], 0x07060302u);
  }
}

// How many of the n ascending numbers at t are at most x, by the wave together: each trip narrows the range to a 64th.
__device__ __forceinline__ int count_up_to(const int32_t* t, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 64) {
    const int step = (n + 63) / 64, at = lane * step;
    const int below = __popcll(__builtin_amdgcn_ballot_w64(at < n && t[lo + min(at, n - 1)] <= x));
    if (below == 0) return lo;
    lo += (below - 1) * step;
    n = min(step, n - (below - 1) * step);
  }
  return lo + __popcll(__builtin_amdgcn_ballot_w64(lane < n && t[lo + min(lane, n - 1)] <= x));
}

// The rows from `row` on that share an adapter, at most up to `limit`: their adapter (-1: none; -2: rows of no request) and their end.
// Offsets that do not ascend name other rows, but none outside the batch.
struct Run {
  int adapter;
  int64_t end;
};
__device__ __forceinline__ Run run_at(const AdapterBatch& b, int64_t row, int64_t limit) {
  if (!b.offsets) return Run{0, limit};
  const int c = __builtin_amdgcn_readfirstlane(count_up_to(b.offsets, b.segments + 1, (int)row));
  if (c == 0 || c > b.segments) {
    const int64_t end = c == 0 ? (int64_t)b.offsets[0] : limit;
    return Run{-2, end > row && end < limit ? end : limit};
  }
  const int64_t end = b.offsets[c];
  const int k = b.index[c - 1];
  return Run{k >= 0 && k < b.adapters ? k : -1, end > row && end < limit ? end : (end > row ? limit : row + 1)};
}

// ---- shrink ---------------------------------------------------------------------------------------
// RT tiles of 16 ranks, R tiles of 16 rows; ROWS: rows that a wave takes (1, or 16 R).  A step is 128 bytes of each row.
template <class T, int RT, int R, int ROWS>
__global__ __launch_bounds__(256) void shrink_kernel(const AdapterShrink a) {
  constexpr int kStep = 128 / sizeof(T), kPer = kStep / 4, kFrags = kPer / 8;   // a lane's elements of a step, in fragments of 8
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  const int64_t tiles = (a.b.L + ROWS - 1) / ROWS;
  const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int slice = __builtin_amdgcn_readfirstlane((int)(task / tiles));
  if (slice >= a.slices) return;
  const int64_t row0 = (task - slice * tiles) * ROWS;
  const int64_t row1 = min(row0 + ROWS, a.b.L);
  const int64_t k0 = slice * a.slice, k1 = min(k0 + a.slice, a.K);
  float* const out = a.out + (int64_t)slice * a.b.L * a.pitch;

  for (int64_t row = row0; row < row1;) {
    const Run run = run_at(a.b, row, row1);
    if (run.adapter >= 0) {
      const T* const w = (const T*)a.w + run.adapter * a.w_stride;
      const T* x[R];
      const T* wr[RT];
      bool part_of_run[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t l = min(max(row0 + r * 16 + i, row), run.end - 1);
        x[r] = (const T*)a.q + l * a.K + q * kPer;
        part_of_run[r] = row0 + r * 16 < run.end && row0 + r * 16 + 16 > row;
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) wr[t] = w + min(t * 16 + i, a.rank - 1) * a.w_pitch + q * kPer;
      f4 acc[RT][R];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[t][r] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      int64_t k = k0;
      for (; k + kStep <= k1; k += kStep) {
        Raw8<T> fx[R][kFrags], fw[RT][kFrags];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (R == 1 || part_of_run[r]) fx[r][f] = load8(x[r] + k + f * 8, 8);
#pragma unroll
          for (int t = 0; t < RT; ++t) fw[t][f] = load8(wr[t] + k + f * 8, 8);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (R == 1 || part_of_run[r]) {
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
#pragma unroll
              for (int t = 0; t < RT; ++t) acc[t][r] = mma(frag(fw[t][f]), frag(fx[r][f]), acc[t][r]);
          }
      }
      if (k < k1) {     // the row's last elements: zeros behind them, on both sides
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
          const int n = (int)max(min((int64_t)8, k1 - k - q * kPer - f * 8), (int64_t)0);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const Frag<T> fx = frag(load8(x[r] + k + f * 8, n));
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t][r] = mma(frag(load8(wr[t] + k + f * 8, n)), fx, acc[t][r]);
          }
        }
      }
      // Lane (i, q) has ranks 16 t + 4 q .. + 3 of row i.
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t l = row0 + r * 16 + i;
        if (l >= row && l < run.end) {
#pragma unroll
          for (int t = 0; t < RT; ++t)
            if (t * 16 + q * 4 < a.pitch) *(f4*)(out + l * a.pitch + t * 16 + q * 4) = acc[t][r];
        }
      }
    }
    row = run.end;
  }
}

// ---- expand ---------------------------------------------------------------------------------------
// RC chunks of 32 ranks (0: at most 16 ranks; the chunk's second half is the second part of the same ranks).
// A wave's step is 64 columns: tile t of the four has columns 16 (m / 4) + 4 t + m % 4 in its row m, so that a lane ends with 16
// columns in a row of its row.
template <class T, int RC, int R, int ROWS>
__global__ __launch_bounds__(256) void expand_kernel(const AdapterExpand a, int64_t span) {
  constexpr bool kSingle = sizeof(T) == 4, kPack = RC == 0 && !kSingle;
  constexpr int kChunks = RC == 0 ? 1 : RC, kParts = kSingle || kPack ? 1 : 2;
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  const int64_t tiles = (a.b.L + ROWS - 1) / ROWS;
  const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t cut = task / tiles;
  const int64_t n0 = cut * span, n1 = min(n0 + span, a.N);
  if (n0 >= a.N) return;
  const int64_t row0 = (task - cut * tiles) * ROWS;
  const int64_t row1 = min(row0 + ROWS, a.b.L);
  const int j0 = kPack ? (q & 1) * 8 : q * 8;      // this lane's ranks within a chunk

  for (int64_t row = row0; row < row1;) {
    const Run run = run_at(a.b, row, row1);
    if (run.adapter == -2) {
      row = run.end;
      continue;
    }
    const bool none = run.adapter < 0;
    const float scale = none ? 0.0f : a.scale ? a.scale[run.adapter] : 1.0f;
    Frag<T> p[R][kChunks][kParts];
    bool mine[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t l = min(row0 + r * 16 + i, a.b.L - 1);
      mine[r] = row0 + r * 16 + i >= row && row0 + r * 16 + i < run.end;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int j = c * 32 + j0;
        float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (!none && mine[r]) {
          for (int s = 0; s < a.slices; ++s) {
            const float* const from = a.p + ((int64_t)s * a.b.L + l) * a.pitch + j;
            float w[8];
            load_values(from, min(max(a.rank - j, 0), 8), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
          }
        }
        if (a.u && n0 == 0 && mine[r] && !(kPack && q >= 2)) store8(a.u + l * a.rank + j, v, min(a.rank - j, 8));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        if constexpr (kSingle) {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[r][c][0].v[e] = v[e];
        } else if constexpr (kPack) {
          Frag<bf16> two[2];
          split8<2>(v, two);
          p[r][c][0] = q < 2 ? two[0] : two[1];
        } else {
          split8<2>(v, p[r][c]);
        }
      }
    }
    const T* const w = (const T*)a.w + (none ? 0 : run.adapter * a.w_stride);
    for (int64_t n = n0; n < n1; n += 64) {
      f4 acc[4][R];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[t][r] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      const int64_t col = n + q * 16;
      const int have[2] = {(int)max(min((int64_t)8, a.N - col), (int64_t)0), (int)max(min((int64_t)8, a.N - col - 8), (int64_t)0)};
      Raw8<T> base[R][2];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t l = row0 + r * 16 + i;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          base[r][h] = load8((const T*)a.base + l * a.N + col + h * 8, a.base && mine[r] ? have[h] : 0);
      }
      if (!none) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const int j = c * 32 + j0, nj = min(max(a.rank - j, 0), 8);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int64_t wn = min(n + (i >> 2) * 16 + t * 4 + (i & 3), a.N - 1);
            const Frag<T> fw = frag(load8(w + wn * a.w_pitch + j, nj));
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int part = 0; part < kParts; ++part) acc[t][r] = mma(fw, p[r][c][part], acc[t][r]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t l = row0 + r * 16 + i;
        if (!mine[r]) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[8];
          widen(base[r][h], v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += acc[h * 2 + e / 4][r][e & 3];
          if (have[h] > 0) store8((T*)a.y + l * a.N + col + h * 8, v, have[h]);
        }
      }
    }
    row = run.end;
  }
}

// ---- what a backward call needs first -------------------------------------------------------------
// Workgroups of the first `adapters` blocks: the segments of adapter k, in the order they have, behind those of the lower ones.  The others:
// 64 x 64 tiles of the two transposes.
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* s_sum) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  __syncthreads();
  if (lane == 0) s_sum[threadIdx.x >> 6] = v;
  __syncthreads();
  return s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

__device__ void sort_segments(const AdapterPrepare& a, int k) {
  __shared__ int64_t s_sum[4];
  __shared__ int s_len[4], s_cnt[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int L = (int)a.b.L;
  const auto length = [&](int s) {
    const int b = min(max(a.b.offsets[s], 0), L);
    return min(max(a.b.offsets[s + 1], b), L) - b;
  };
  int64_t before = 0;                       // rows, and (upper half) segments, of lower adapters
  for (int s = tid; s < a.b.segments; s += 256) {
    const int x = a.b.index[s];
    if (x >= 0 && x < k) before += (int64_t)1 << 32 | (int64_t)length(s);
  }
  before = block_sum(before, s_sum);
  int rows = (int)(before & 0x7FFFFFFF), count = (int)(before >> 32 & 0x7FFFFFFF);
  if (tid == 0) a.first[k] = rows;
  for (int s0 = 0; s0 < a.b.segments; s0 += 256) {
    const int s = s0 + tid;
    const bool mine = s < a.b.segments && a.b.index[s] == k;
    int len = mine ? length(s) : 0;
    const int own = len;
    const uint64_t votes = __builtin_amdgcn_ballot_w64(mine);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int other = __shfl_up(len, m);
      if (lane >= m) len += other;
    }
    __syncthreads();
    if (lane == 63) s_len[wave] = len;
    if (lane == 0) s_cnt[wave] = __popcll(votes);
    __syncthreads();
    int at = rows + len - own, place = count + __popcll(votes & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) {
      at += s_len[w];
      place += s_cnt[w];
    }
    if (mine && place < a.b.segments) {      // always, but for offsets that do not ascend
      a.order[place] = s;
      a.start[place] = at;
    }
    for (int w = 0; w < 4; ++w) {
      rows += s_len[w];
      count += s_cnt[w];
    }
  }
  if (k == a.b.adapters - 1) {              // behind the last one: all that no adapter has, past every row
    if (tid == 0) a.first[k + 1] = rows;
    for (int s = count + tid; s <= a.b.segments; s += 256) {
      a.start[s] = rows;
      if (s < a.b.segments) a.order[s] = 0;
    }
  }
}

template <class T>
__device__ void transpose_tile(const T* from, int64_t rows, int64_t cols, T* to, int64_t to_pitch, int64_t r0, int64_t c0) {
  __shared__ T s_tile[64][65];
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  for (int r = y; r < 64; r += 4)
    s_tile[r][x] = r0 + r < rows && c0 + x < cols ? from[(r0 + r) * cols + c0 + x] : (T)0.0f;
  __syncthreads();
  for (int c = y; c < 64; c += 4)
    if (c0 + c < cols && r0 + x < to_pitch) to[(c0 + c) * to_pitch + r0 + x] = s_tile[x][c];   // the pitch past the rows: zeros
}

template <class T>
__global__ __launch_bounds__(256) void prepare_kernel(const AdapterPrepare a, int sorts, int tiles_a, int tiles_w, int rank_tiles) {
  int b = blockIdx.x;
  if (b < sorts) {
    sort_segments(a, b);
    return;
  }
  b -= sorts;
  const int per = tiles_a + tiles_w, k = b / per, t = b % per;
  if (t < tiles_a)
    transpose_tile((const T*)a.a + (int64_t)k * a.rank * a.I, a.rank, a.I, (T*)a.at + (int64_t)k * a.I * a.rank_pitch, a.rank_pitch,
                   (int64_t)(t % rank_tiles) * 64, (int64_t)(t / rank_tiles) * 64);
  else
    transpose_tile((const T*)a.w + (int64_t)k * a.O * a.rank, a.O, a.rank, (T*)a.wt + (int64_t)k * a.rank * a.O, a.O,
                   (int64_t)((t - tiles_a) / rank_tiles) * 64, (int64_t)((t - tiles_a) % rank_tiles) * 64);
}

// ---- outer ----------------------------------------------------------------------------------------
// Eight rows of eight columns a lane.  bfloat16: column c's eight rows come together in 32 byte permutes; fp32: they are registers.
__device__ __forceinline__ void columns_of(const Raw8<bf16> (&rows)[8], Frag<bf16> (&out)[8]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const u4 lo = __builtin_bit_cast(u4, rows[2 * r].a), hi = __builtin_bit_cast(u4, rows[2 * r + 1].a);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      out[2 * c].v[r] = __builtin_amdgcn_perm(hi[c], lo[c], 0x05040100u);
      out[2 * c + 1].v[r] = __builtin_amdgcn_perm(hi[c], lo[c], 0x07060302u);
    }
  }
}
__device__ __forceinline__ void columns_of(const Raw8<float> (&rows)[8], Frag<float> (&out)[8]) {
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    float v[8];
    widen(rows[r], v);
#pragma unroll
    for (int c = 0; c < 8; ++c) out[c].v[r] = v[c];
  }
}

constexpr int kOuterCols = 128;

// A workgroup: 128 columns, up to 64 ranks, one part of the rows that have adapters, in the order of their adapters.  Its four waves take
// steps of 32 rows in turn and join their sums through LDS, once for each adapter of the part.
template <class T, int RT>
__global__ __launch_bounds__(256) void outer_kernel(const AdapterOuter a, int tiles_first, int tiles, int rank_blocks) {
  constexpr int kParts = sizeof(T) == 4 ? 1 : 3;
  __shared__ float s_acc[2][RT * 16 * kOuterCols];
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int part = blockIdx.x / (tiles * rank_blocks), in = blockIdx.x % (tiles * rank_blocks);
  const int tile = in % tiles, rank0 = in / tiles * 64;
  const bool second = tile >= tiles_first;
  const AdapterOuterOperand& o = second ? a.a[1] : a.a[0];
  const int64_t col0 = (int64_t)(second ? tile - tiles_first : tile) * kOuterCols, col = col0 + i * 8;
  const int have = (int)max(min((int64_t)8, o.N - col), (int64_t)0);
  const int64_t total = a.first ? max(min((int64_t)a.first[a.b.adapters], a.b.L), (int64_t)0) : a.b.L;
  const int64_t lo = total * part / a.parts, hi = total * (part + 1) / a.parts;

  for (int64_t pos = lo; pos < hi;) {
    int k = 0;
    int64_t k_end = hi;
    if (a.first) {
      k = __builtin_amdgcn_readfirstlane(count_up_to(a.first, a.b.adapters + 1, (int)pos)) - 1;
      k = min(max(k, 0), a.b.adapters - 1);
      k_end = min((int64_t)a.first[k + 1], hi);
      if (k_end <= pos) break;
    }
    f4 acc[RT][8];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[t][c] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    int turn = 0;
    while (pos < k_end) {
      int64_t row = pos, end = k_end;       // rows row .. row + end - pos - 1
      if (a.first) {
        const int s = min(max(__builtin_amdgcn_readfirstlane(count_up_to(a.start, a.b.segments + 1, (int)pos)) - 1, 0), a.b.segments - 1);
        row = max((int64_t)a.b.offsets[a.order[s]] + pos - a.start[s], (int64_t)0);
        end = min(k_end, max((int64_t)a.start[s + 1], pos + 1));
      }
      const int64_t last = min(row + (end - pos), a.b.L) - 1;
      for (; row <= last; row += 32) {
        if ((turn++ & 3) != wave) continue;
        Raw8<T> x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int64_t l = min(row + q * 8 + e, last);      // rows past the run's end: the last one, times zero
          x[e] = load8((const T*)o.q + l * o.N + col, have);
        }
        Frag<T> p[RT][kParts];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const int j = rank0 + t * 16 + i;
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int64_t l = row + q * 8 + e;
            v[e] = 0.0f;
            if (l <= last && j < a.rank) {
              for (int s = 0; s < o.slices; ++s) v[e] += o.p[((int64_t)s * a.b.L + l) * o.p_pitch + j];
            }
          }
          if constexpr (kParts == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[t][0].v[e] = v[e];
          } else {
            split8<3>(v, p[t]);
          }
        }
        Frag<T> f[8];
        columns_of(x, f);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int s = 0; s < kParts; ++s)
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[t][c] = mma(p[t][s], f[c], acc[t][c]);
      }
      pos = end;
    }
    // Waves 2 and 3 hand their sums to 0 and 1, then 1 to 0.  Lane (i, q) has ranks 16 t + 4 q + e of columns 8 i + c.
#pragma unroll
    for (int half = 2; half >= 1; half /= 2) {
      __syncthreads();
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float* const to = &s_acc[wave - half][(t * 16 + q * 4 + e) * kOuterCols + i * 8];
            *(f4*)to = f4{acc[t][0][e], acc[t][1][e], acc[t][2][e], acc[t][3][e]};
            *(f4*)(to + 4) = f4{acc[t][4][e], acc[t][5][e], acc[t][6][e], acc[t][7][e]};
          }
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float* const from = &s_acc[wave][(t * 16 + q * 4 + e) * kOuterCols + i * 8];
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[t][c][e] += from[c];
          }
      }
    }
    if (wave == 0) {
      const float scale = o.scaled && a.scale ? a.scale[k] : 1.0f;
      float* const to = o.part + (int64_t)(part + k) * a.rank * o.N;
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = rank0 + t * 16 + q * 4 + e;
          float v[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) v[c] = acc[t][c][e] * scale;
          if (j < a.rank && have > 0) store8(to + (int64_t)j * o.N + col, v, have);
        }
    }
  }
}

// Sums of the parts of each adapter, in order.  Block: (adapter, 256 columns of [I | O]); part p of adapter k is slot p + k.
__global__ __launch_bounds__(256) void reduce_kernel(const AdapterReduce a, int tiles_a, int tiles) {
  const int k = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const bool second = tile >= tiles_a;
  const int64_t N = second ? a.O : a.I, n = (int64_t)(second ? tile - tiles_a : tile) * 256 + threadIdx.x;
  if (n >= N) return;
  const float* const part = second ? a.part_b : a.part_a;
  const int64_t total = a.first ? max(min((int64_t)a.first[a.adapters], a.L), (int64_t)0) : a.L;
  const int64_t lo = a.first ? a.first[k] : (k == 0 ? 0 : total), hi = a.first ? a.first[k + 1] : (k == 0 ? total : total);
  for (int j = 0; j < a.rank; ++j) {
    float v = 0.0f;
    for (int p = 0; p < a.parts; ++p) {
      const int64_t b = total * p / a.parts, e = total * (p + 1) / a.parts;
      if (max(b, lo) < min(e, hi)) v += part[((int64_t)(p + k) * a.rank + j) * N + n];
    }
    if (second) a.g_b[((int64_t)k * a.O + n) * a.rank + j] = v;
    else a.g_a[((int64_t)k * a.rank + j) * a.I + n] = v;
  }
}

template <class T, int RT>
hipError_t run_shrink(const AdapterShrink& a, bool rows, hipStream_t s) {
  if (rows) {
    const int64_t tasks = a.b.L * a.slices;
    shrink_kernel<T, RT, 1, 1><<<(uint32_t)ceil_div(tasks, 4), 256, 0, s>>>(a);
  } else {
    const int64_t tasks = ceil_div(a.b.L, 32) * a.slices;
    shrink_kernel<T, RT, 2, 32><<<(uint32_t)ceil_div(tasks, 4), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}
template <class T>
hipError_t shrink_of(const AdapterShrink& a, bool rows, hipStream_t s) {
  if (a.rank <= 16) return run_shrink<T, 1>(a, rows, s);
  if (a.rank <= 32) return run_shrink<T, 2>(a, rows, s);
  if (a.rank <= 64) return run_shrink<T, 4>(a, rows, s);
  return run_shrink<T, 8>(a, rows, s);
}

// Waves that an expansion is cut into where its rows alone are fewer.
constexpr int64_t kExpandWaves = 4096;

template <class T, int RC>
hipError_t run_expand(const AdapterExpand& a, bool rows, hipStream_t s) {
  const int64_t tiles = rows ? a.b.L : ceil_div(a.b.L, 32), steps = ceil_div(a.N, 64);
  int64_t cuts = ceil_div(kExpandWaves, tiles);
  if (cuts > steps) cuts = steps;
  const int64_t span = ceil_div(steps, cuts) * 64;
  const int64_t tasks = tiles * ceil_div(a.N, span);
  if (rows) expand_kernel<T, RC, 1, 1><<<(uint32_t)ceil_div(tasks, 4), 256, 0, s>>>(a, span);
  else expand_kernel<T, RC, 2, 32><<<(uint32_t)ceil_div(tasks, 4), 256, 0, s>>>(a, span);
  return hipGetLastError();
}
template <class T>
hipError_t expand_of(const AdapterExpand& a, bool rows, hipStream_t s) {
  if (a.rank <= 16) return run_expand<T, 0>(a, rows, s);
  if (a.rank <= 32) return run_expand<T, 1>(a, rows, s);
  if (a.rank <= 64) return run_expand<T, 2>(a, rows, s);
  return run_expand<T, 4>(a, rows, s);
}

template <class T>
hipError_t outer_of(const AdapterOuter& a, hipStream_t s) {
  const int tiles_first = (int)ceil_div(a.a[0].N, kOuterCols), tiles = tiles_first + (int)ceil_div(a.a[1].N, kOuterCols);
  const int blocks = (int)ceil_div(a.rank, 64);
  const uint32_t grid = (uint32_t)((int64_t)tiles * blocks * a.parts);
  if (a.rank <= 16) outer_kernel<T, 1><<<grid, 256, 0, s>>>(a, tiles_first, tiles, blocks);
  else if (a.rank <= 32) outer_kernel<T, 2><<<grid, 256, 0, s>>>(a, tiles_first, tiles, blocks);
  else outer_kernel<T, 4><<<grid, 256, 0, s>>>(a, tiles_first, tiles, blocks);
  return hipGetLastError();
}

}  // namespace

AdapterPlan adapter_plan(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters, int64_t segments) {
  AdapterPlan p{};
  const int64_t size = type == HOT_BF16 ? 2 : 4, step = 128 / size;
  p.rows = L <= 4 * (segments > 0 ? segments : 1) && L <= 1 << 20;
  p.pitch = (int)round_up(rank, 4);
  p.rank_pitch = (int)round_up(rank, 8);
  const auto slices = [&](int64_t K, int& count, int64_t& slice) {
    const int64_t tiles = p.rows ? L : ceil_div(L, 32);
    int64_t n = 2048 / tiles;
    const int64_t most = ceil_div(K, 4 * step);
    if (n > most) n = most;
    if (n > kMaxSlices) n = kMaxSlices;
    if (n < 1) n = 1;
    slice = round_up(ceil_div(K, n), step);
    count = (int)ceil_div(K, slice);
  };
  slices(I, p.slices_forward, p.slice_forward);
  slices(O, p.slices_backward, p.slice_backward);
  const int64_t tiles = (ceil_div(I, kOuterCols) + ceil_div(O, kOuterCols)) * ceil_div(rank, 64);
  int64_t parts = ceil_div(768, tiles);
  const int64_t most = ceil_div(L, 128);
  p.parts = (int)(parts < most ? parts : most);

  const int64_t row_bytes = L * p.pitch * 4;
  p.forward = (size_t)round_up(row_bytes * p.slices_forward, 256);
  size_t at = (size_t)round_up(row_bytes * p.slices_backward, 256);
  const auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)round_up(bytes, 256);
    return here;
  };
  p.at = take(adapters * I * p.rank_pitch * size);
  p.wt = take(adapters * rank * O * size);
  p.sorted = take((2 * segments + 1 + adapters + 1) * 4);
  p.part_a = take((p.parts + adapters) * rank * I * 4);
  p.part_b = take((p.parts + adapters) * rank * O * 4);
  p.backward = at;
  return p;
}

hipError_t launch_adapter_shrink(const AdapterShrink& a, bool rows, hot_type type, hipStream_t s) {
  return type == HOT_BF16 ? shrink_of<bf16>(a, rows, s) : shrink_of<float>(a, rows, s);
}
hipError_t launch_adapter_expand(const AdapterExpand& a, bool rows, hot_type type, hipStream_t s) {
  return type == HOT_BF16 ? expand_of<bf16>(a, rows, s) : expand_of<float>(a, rows, s);
}
hipError_t launch_adapter_prepare(const AdapterPrepare& a, hot_type type, hipStream_t s) {
  const int sorts = a.b.offsets ? a.b.adapters : 0;
  const int rank_tiles = (int)ceil_div(a.rank_pitch, 64);
  const int tiles_a = a.at ? (int)ceil_div(a.I, 64) * rank_tiles : 0, tiles_w = a.wt ? (int)ceil_div(a.O, 64) * rank_tiles : 0;
  const int64_t grid = sorts + (int64_t)a.b.adapters * (tiles_a + tiles_w);
  if (grid == 0) return hipSuccess;
  if (type == HOT_BF16) prepare_kernel<bf16><<<(uint32_t)grid, 256, 0, s>>>(a, sorts, tiles_a, tiles_w, rank_tiles);
  else prepare_kernel<float><<<(uint32_t)grid, 256, 0, s>>>(a, sorts, tiles_a, tiles_w, rank_tiles);
  return hipGetLastError();
}
hipError_t launch_adapter_outer(const AdapterOuter& a, hot_type type, hipStream_t s) {
  return type == HOT_BF16 ? outer_of<bf16>(a, s) : outer_of<float>(a, s);
}
hipError_t launch_adapter_reduce(const AdapterReduce& a, hipStream_t s) {
  const int tiles_a = (int)ceil_div(a.I, 256), tiles = tiles_a + (int)ceil_div(a.O, 256);
  reduce_kernel<<<(uint32_t)((int64_t)a.adapters * tiles), 256, 0, s>>>(a, tiles_a, tiles);
  return hipGetLastError();
}

}  // namespace hot
