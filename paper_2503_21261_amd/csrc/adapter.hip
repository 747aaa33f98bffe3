// Low-rank adapters beside a shared projection, each row with the adapter k of its request:
//   u = x A_k^T,  y = base + s_k u B_k^T;   g_u = s_k g_y B_k,  g_x = g_base + g_u A_k,
//   g_A_k = sum of g_u^T x,  g_B_k = s_k sum of g_y^T u  over the adapter's rows.
//
// Bound by memory: with a rank of some tens, x, g_y and the outputs are read or written for two operations a rank and element.  Three
// kernels, all on the matrix cores, none with a library call:
//   shrink  [rows x K] . [rank x K]^T -> [rows x rank]: a workgroup has 16 to 64 rows (or one) and all ranks, K in slices where rows are few;
//   expand  [rows x rank] . [N x rank]^T -> [rows x N]: a wave holds the factors of its columns in registers, rows go by;
//   outer   [rows x rank]^T . [rows x N] -> [rank x N]: rows as they lie are transposed in registers, 8 x 8 values a lane, the factors
//           before, by a launch of its own.
// u and g_u are fp32.  Where they meet bfloat16 operands they are split into bfloat16 parts, cut off and not rounded, so that three
// parts are the number itself: three for fp32 results (g_A, g_B), two for bfloat16 ones, the second of which is rounded: 16 bits, within 2^-16
// of the number (cut off as well it would be within 2^-15).
#include <type_traits>

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

// Eight elements for a lane, of 32 that four lanes share: bfloat16 those from 8 q on; fp32 in two loads of four, those from 4 q and from 16 + 4 q
// on (the order of the reduced elements is free), which are APART elements apart in memory.
template <class T> struct Piece;
template <> struct Piece<bf16> { h8_any v; };
template <> struct Piece<float> { f4_any v[2]; };
template <int APART>
__device__ __forceinline__ Piece<bf16> load_piece(const bf16* p) { return Piece<bf16>{*(const h8_any*)p}; }
template <int APART>
__device__ __forceinline__ Piece<float> load_piece(const float* p) { return Piece<float>{{*(const f4_any*)p, *(const f4_any*)(p + APART)}}; }
// Of the 32 elements from p on, of which `left` exist; zeros for the others.
__device__ __forceinline__ Piece<bf16> load_piece_of(const bf16* p, int q, int left) {
  return Piece<bf16>{load8(p + q * 8, min(max(left - q * 8, 0), 8)).a};
}
__device__ __forceinline__ Piece<float> load_piece_of(const float* p, int q, int left) {
  Piece<float> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int at = e / 4 * 16 + q * 4 + e % 4;
    r.v[e / 4][e % 4] = at < left ? p[at] : 0.0f;
  }
  return r;
}
// The same where the elements from p on are a row's last `left`, of `row` in all: a row of eight (four) or more is loaded as its last ones, and
// they are moved down.
__device__ __forceinline__ Piece<bf16> load_piece_end(const bf16* p, int q, int left, int row) {
  const int n = min(max(left - q * 8, 0), 8);
  if (row < 8) return load_piece_of(p, q, left);
  const int by = n > 0 ? 8 - n : 0;
  u4 v = __builtin_bit_cast(u4, *(const h8_any*)(p + (n > 0 ? q * 8 - by : left - 8)));
  uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
  if (by & 4) {
    lo = hi;
    hi = 0;
  }
  const int bits = (by & 3) * 16;
  if (bits) lo = lo >> bits | hi << (64 - bits);
  hi >>= bits;
  if (n == 0) lo = hi = 0;
  v = u4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  return Piece<bf16>{__builtin_bit_cast(h8_any, v)};
}
__device__ __forceinline__ Piece<float> load_piece_end(const float* p, int q, int left, int row) {
  if (row < 4) return load_piece_of(p, q, left);
  Piece<float> r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * 16 + q * 4, n = min(max(left - at, 0), 4), by = n > 0 ? 4 - n : 0;
    const f4_any v = *(const f4_any*)(p + (n > 0 ? at - by : left - 4));
    const float a = v[0], b = v[1], c = v[2], d = v[3];
    r.v[h][0] = n == 0 ? 0.0f : by == 0 ? a : by == 1 ? b : by == 2 ? c : d;
    r.v[h][1] = n <= 1 ? 0.0f : by == 0 ? b : by == 1 ? c : d;
    r.v[h][2] = n <= 2 ? 0.0f : by == 0 ? c : d;
    r.v[h][3] = n <= 3 ? 0.0f : d;
  }
  return r;
}
// fp32 numbers in the places that a piece of T has them.
template <class T>
__device__ __forceinline__ Piece<float> load_piece_as(const float* p, int q, int left) {
  if constexpr (sizeof(T) == 4) {
    return load_piece_of(p, q, left);
  } else {
    const Raw8<float> r = load8(p + q * 8, min(max(left - q * 8, 0), 8));
    return Piece<float>{{r.a, r.b}};
  }
}
// Elements that a wave's 64 lanes have of 16 rows and 32 reduced elements: a packed tile.
constexpr int kTile = 512;
__device__ __forceinline__ Frag<bf16> frag(const Piece<bf16>& r) { return Frag<bf16>{__builtin_bit_cast(u4, r.v)}; }
__device__ __forceinline__ Frag<float> frag(const Piece<float>& r) {
  Frag<float> f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f.v[e] = r.v[0][e];
    f.v[4 + e] = r.v[1][e];
  }
  return f;
}

__device__ __forceinline__ f4 mma(const Frag<bf16>& a, const Frag<bf16>& b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a.v), __builtin_bit_cast(b8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f4 mma(const Frag<float>& a, const Frag<float>& b, f4 c) {
#pragma unroll
  for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[t], b.v[t], c, 0, 0, 0);
  return c;
}

// Parts of eight fp32 numbers as bfloat16: the upper 16 bits, then those of what is left, rounded to nearest in the second of two.  An infinity
// or a NaN is whole in the first.
__device__ __forceinline__ uint32_t rounded_pair(uint32_t a, uint32_t b) {
  return (uint32_t)float_to_bf16(__uint_as_float(b)) << 16 | float_to_bf16(__uint_as_float(a));
}
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
    for (int i = 0; i < 4; ++i)
      out[p].v[i] = PARTS == 2 && p == 1 ? rounded_pair(bits[2 * i], bits[2 * i + 1]) : __builtin_amdgcn_perm(bits[2 * i + 1], bits[2 * i], 0x07060302u);
  }
}

// Factors of the expansion in the order of its lanes: for 16 rows and 32 ranks a tile (bfloat16: two, the two parts), [rows / 16][chunks].  Up to 16
// ranks in bfloat16 are one tile: the second half of its 32 elements is the second part of the first.  Ranks j .. j + 3 of row l.
__device__ __forceinline__ void store_factors(float* p, int64_t l, int j, int chunks, f4 v) {
  const int in = j & 31, q = (in & 15) / 4;
  *(f4*)(p + ((l >> 4) * chunks + (j >> 5)) * kTile + in / 16 * 256 + (q * 16 + (l & 15)) * 4) = v;
}
__device__ __forceinline__ void store_factors(bf16* p, int64_t l, int j, int chunks, f4 v) {
  uint32_t part[2][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t b = __float_as_uint(v[e]);
    const bool finite = (b & 0x7F800000u) != 0x7F800000u;
    part[0][e] = (b & 0x7FFFFFFFu) > 0x7F800000u ? b | 0x400000u : b;      // as split8()
    part[1][e] = finite ? __float_as_uint(v[e] - __uint_as_float(b & 0xFFFF0000u)) : 0u;
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const auto pair = [&](uint32_t a, uint32_t b) { return s == 0 ? __builtin_amdgcn_perm(b, a, 0x07060302u) : rounded_pair(a, b); };
    const uint2 x = make_uint2(pair(part[s][0], part[s][1]), pair(part[s][2], part[s][3]));
    const int in = j & 31;
    bf16* const at = chunks == 0 ? p + (l >> 4) * kTile + ((s * 2 + in / 8) * 16 + (l & 15)) * 8
                                 : p + (((l >> 4) * chunks + (j >> 5)) * 2 + s) * kTile + (in / 8 * 16 + (l & 15)) * 8;
    *(uint2*)(at + (j & 4)) = x;
  }
}

// A row's 128 bytes of a step as fragments, from a lane's pieces of the first and the second half.
__device__ __forceinline__ void frags_of(u4 lo, u4 hi, Frag<bf16> (&f)[2]) {
  f[0].v = lo;
  f[1].v = hi;
}
__device__ __forceinline__ void frags_of(u4 lo, u4 hi, Frag<float> (&f)[1]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[0].v[e] = __uint_as_float(lo[e]);
    f[0].v[4 + e] = __uint_as_float(hi[e]);
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
  int c, k;
  int64_t end;
  if (b.segments < 64) {        // all in one load of the wave
    const int lane = threadIdx.x & 63;
    const int at = b.offsets[min(lane, b.segments)], own = b.index[min(lane, b.segments - 1)];
    c = __popcll(__builtin_amdgcn_ballot_w64(lane <= b.segments && at <= row));
    end = __builtin_amdgcn_readlane(at, c <= b.segments ? c : 0);
    k = __builtin_amdgcn_readlane(own, c > 0 && c <= b.segments ? c - 1 : 0);
  } else {
    c = __builtin_amdgcn_readfirstlane(count_up_to(b.offsets, b.segments + 1, (int)row));
    end = c <= b.segments ? b.offsets[c] : 0;
    k = c > 0 && c <= b.segments ? b.index[c - 1] : -1;
  }
  if (c == 0 || c > b.segments) return Run{-2, c == 0 && end > row && end < limit ? end : limit};
  return Run{k >= 0 && k < b.adapters ? k : -1, end > row ? (end < limit ? end : limit) : row + 1};
}

// The consecutive columns of a row that a lane has: 16 bytes.
template <class T> struct Cols;
template <> struct Cols<bf16> { typedef h8_any V; V v; };
template <> struct Cols<float> { typedef f4_any V; V v; };
template <class T>
constexpr int kCols = 16 / sizeof(T);
template <class T>
__device__ __forceinline__ Cols<T> load_cols(const T* p) { return Cols<T>{*(const typename Cols<T>::V*)p}; }

// ---- shrink ---------------------------------------------------------------------------------------
// The memory pipe takes the 64 bytes of four neighbouring lanes at a time, where they lie together; lanes of a matrix instruction's operand are
// rows, so that a load of 16 rows takes four times as long as one of 1024 bytes in a row.  So rows are loaded eight lanes a row and change
// lanes through LDS (12608 x 768 and x 2304 fp32, rank 16: 14.0 -> 11.3 us and 29.3 -> 26.2; 3330 x 771 bfloat16: 14.7 -> 11.1); weights are packed
// in the order of the lanes first, where that pays or they have to be transposed anyway; and the sums are left in that order for the expansion.
//
// RT tiles of 16 ranks, R tiles of 16 rows; ROWS: rows that a workgroup takes (1, or 16 R).  A step is 128 bytes of each row; the four waves
// take steps in turn, DEPTH of them on their way, and join their sums through LDS.  Weights come from the L2 once a workgroup, which bounds large
// ranks: 16384 x 11008 and x 4096 bfloat16, rank 64: 105 and 39 us (3.4 TB/s of the rows) with 64 rows a workgroup, 113 and 45 with 32.  Rank 16,
// 12608 x 768 and x 2304 fp32: 11.8 and 25.5 us, 3.3 and 4.6 TB/s.
template <class T, int RT, int R, int ROWS, int DEPTH, bool PACKED>
__global__ __launch_bounds__(256, RT <= 4 && R <= 2 ? 2 : 1) void shrink_kernel(const AdapterShrink a) {
  constexpr int kStep = 128 / sizeof(T), kFrags = kStep / 32, kPer = 16 / sizeof(T);
  constexpr bool kTurned = ROWS > 1;         // rows through LDS
  constexpr int kLoads = kTurned ? 2 * R : 0;
  __shared__ f4 s_acc[3][RT * R][64];
  __shared__ u4 s_x[4][kTurned ? R * 16 : 1][8];
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t tiles = (a.b.L + ROWS - 1) / ROWS;
  const int slice = (int)(blockIdx.x / tiles);
  const int64_t row0 = (blockIdx.x - slice * tiles) * ROWS;
  const int64_t row1 = min(row0 + ROWS, a.b.L);
  const int64_t k0 = slice * a.slice, k1 = min(k0 + a.slice, a.K);
  float* const out = a.out + (int64_t)slice * a.b.L * a.pitch;
  const int64_t first = k0 + wave * kStep, whole = k0 + (k1 - k0) / kStep * kStep;      // this wave's first step, the end of the whole ones
  const int rank_tiles = (a.rank + 15) / 16;

  for (int64_t row = row0; row < row1;) {
    const Run run = run_at(a.b, row, row1);
    if (run.adapter >= 0) {
      const T* const w = (const T*)a.w + run.adapter * a.w_stride;
      const auto row_at = [&](int r) { return (const T*)a.q + min(max(row0 + r, row), run.end - 1) * a.K; };
      const T* x[kTurned ? kLoads : 1];
      const T* wr[RT];
      // Row 8 g + lane / 8, of its eight pieces of 16 bytes the one that lies in place lane % 8: they are dealt so that reads of 16 rows meet
      // all banks.
      if constexpr (kTurned) {
#pragma unroll
        for (int g = 0; g < kLoads; ++g) x[g] = row_at(g * 8 + lane / 8) + ((lane & 7) ^ (lane / 8)) * kPer;
      } else {
        x[0] = row_at(0) + q * kPer;
      }
#pragma unroll
      for (int t = 0; t < RT; ++t)      // ranks past the last: the last one's, whose sums are not kept
        wr[t] = PACKED ? w + min(t, rank_tiles - 1) * kTile + lane * kPer : w + min(t * 16 + i, a.rank - 1) * a.K;
      f4 acc[RT][R];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[t][r] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      struct Step {
        Cols<T> rows[kTurned ? kLoads : 1];
        Piece<T> x[kTurned ? 1 : kFrags], w[RT][kFrags];
      };
      const auto load = [&](int64_t at, Step& d) {
        if constexpr (kTurned) {
#pragma unroll
          for (int g = 0; g < kLoads; ++g) d.rows[g] = load_cols(x[g] + at);
        } else {
#pragma unroll
          for (int f = 0; f < kFrags; ++f) d.x[f] = load_piece<16>(x[0] + at + f * 32);
        }
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            if constexpr (PACKED) d.w[t][f] = load_piece<256>(wr[t] + (at / 32 + f) * rank_tiles * kTile);
            else d.w[t][f] = load_piece<16>(wr[t] + at + f * 32 + q * kPer);
          }
        }
      };
      const auto multiply = [&](const Step& d) {
        Frag<T> fx[R][kFrags];
        if constexpr (kTurned) {      // in order within the wave: no barrier
          u4(&place)[R * 16][8] = s_x[wave];
#pragma unroll
          for (int g = 0; g < kLoads; ++g) place[g * 8 + lane / 8][lane & 7] = __builtin_bit_cast(u4, d.rows[g].v);
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const u4 lo = place[r * 16 + i][q ^ (i & 7)], hi = place[r * 16 + i][(4 + q) ^ (i & 7)];
            frags_of(lo, hi, fx[r]);
          }
          __builtin_amdgcn_wave_barrier();
        } else {
#pragma unroll
          for (int f = 0; f < kFrags; ++f) fx[0][f] = frag(d.x[f]);
        }
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t][r] = mma(frag(d.w[t][f]), fx[r][f], acc[t][r]);
      };
      if (first < whole) {
        // Each workgroup begins its walk elsewhere: side by side they would all ask for the same columns of the weights.
        constexpr int kTurn = 4 * kStep;
        const int n = (int)((whole - 1 - first) / kTurn) + 1, from = (int)(blockIdx.x % (uint32_t)n);
        // The last step's loads are made once more instead of a branch around them, which would make the waits wait for all.
        const auto step_at = [&](int s) {
          const int k = min(s, n - 1) + from;
          return first + (int64_t)(k < n ? k : k - n) * kTurn;
        };
        Step d[DEPTH];
#pragma unroll
        for (int s = 0; s < DEPTH - 1; ++s) load(step_at(s), d[s]);
        // Rounds of DEPTH steps without a way out of their middle, which would have the buffers copied at each round's end; what is left is
        // loaded already.
        int at = 0;
        for (; at + DEPTH <= n; at += DEPTH) {
#pragma unroll
          for (int s = 0; s < DEPTH; ++s) {
            load(step_at(at + s + DEPTH - 1), d[(s + DEPTH - 1) % DEPTH]);
            __builtin_amdgcn_sched_barrier(0);      // else the loads sink to where they are used
            multiply(d[s]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
#pragma unroll
        for (int s = 0; s < DEPTH - 1; ++s)
          if (at + s < n) multiply(d[s]);
      }
      if (whole < k1 && wave == 3) {              // the row's last elements: zeros behind them, on both sides
        for (int64_t at = whole; at < k1; at += 32) {
          const int left = (int)min(k1 - at, (int64_t)32);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const Frag<T> fx = frag(load_piece_of(row_at(r * 16 + i) + at, q, left));
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              if constexpr (PACKED) acc[t][r] = mma(frag(load_piece<256>(wr[t] + at / 32 * rank_tiles * kTile)), fx, acc[t][r]);
              else acc[t][r] = mma(frag(load_piece_of(wr[t] + at, q, left)), fx, acc[t][r]);
            }
          }
        }
      }
      if (wave > 0) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int r = 0; r < R; ++r) s_acc[wave - 1][t * R + r][lane] = acc[t][r];
      }
      __syncthreads();
      // Lane (i, q) has ranks 16 t + 4 q .. + 3 of row i.
      if (wave == 0) {
        const float scale = a.scale ? a.scale[run.adapter] : 1.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int64_t l = row0 + r * 16 + i;
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const int j = t * 16 + q * 4;
            f4 v = acc[t][r];
#pragma unroll
            for (int o = 0; o < 3; ++o) {
              const f4 other = s_acc[o][t * R + r][lane];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] += other[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = j + e < a.rank ? v[e] : 0.0f;
            if (l < row || l >= run.end) continue;
            if (j < a.pitch) *(f4*)(out + l * a.pitch + j) = v;
            if (a.u) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (j + e < a.rank) a.u[l * a.rank + j + e] = v[e];
            }
            if (a.packed) store_factors((T*)a.packed, l, j, a.chunks, v * scale);
          }
          if (a.packed && RT == 1 && sizeof(T) == 4 && l >= row && l < run.end)    // the other half of a chunk of 32 ranks
            store_factors((T*)a.packed, l, 16 + q * 4, a.chunks, f4{0.0f, 0.0f, 0.0f, 0.0f});
        }
      }
      __syncthreads();
    } else if (run.adapter == -1 && a.u) {
      for (int64_t at = row * a.rank + threadIdx.x; at < run.end * a.rank; at += 256) a.u[at] = 0.0f;
    }
    row = run.end;
  }
}

__device__ __forceinline__ int64_t ceil_of(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- expand ---------------------------------------------------------------------------------------
__device__ __forceinline__ Cols<bf16> sum_cols(const Cols<bf16>& b, const f4 (&x)[8], int e) {
  Cols<bf16> r;
#pragma unroll
  for (int t = 0; t < 8; ++t) r.v[t] = float_to_bf16(bf16_to_float(b.v[t]) + x[t][e]);
  return r;
}
__device__ __forceinline__ Cols<float> sum_cols(const Cols<float>& b, const f4 (&x)[4], int e) {
  Cols<float> r;
#pragma unroll
  for (int t = 0; t < 4; ++t) r.v[t] = b.v[t] + x[t][e];
  return r;
}

// The rows of [row, end) and 16 lanes' columns, NT from col on each: the rows' factors as they were packed, DEPTH tiles of 16 rows on their way.  Rows are
// the product's rows here: tile t of NT has column t of each lane, so that lane (i, q) ends with its columns of rows 4 q .. + 3, 16 lanes a row.
// Nothing here branches but the loop, so that a wait is for one tile and not for all: where the rows do not fill their tiles (WHOLE says that they
// do), the nearest one of them stands for those beside them, from its factors to its output, which is written more than once (by one
// instruction, or by the same wave: the same bits).  Reading and writing 16384 x 11008 bfloat16, rank 64: 136 us, 5.3 TB/s; with the streaming
// hint on y 8 % more.
template <class T, int NT, int PIECES, int CHUNKS, int PARTS, int DEPTH, bool BASE, bool WHOLE>
__device__ __forceinline__ void expand_tiles(const AdapterExpand& a, int64_t row, int64_t end, int64_t col, const Frag<T> (&fw)[NT][CHUNKS]) {
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  struct Tile {
    std::conditional_t<NT == 1, T, Cols<T>> base[4];
    Piece<T> p[PIECES];
  };
  const int64_t first = row & -16ll;
  const int count = (int)((((end - 1) & -16ll) - first) / 16) + 1, m = (int)(row - first), rows = (int)(end - 1 - first);
  const int64_t from = (WHOLE ? (first + q * 4) * a.N : first * a.N) + col;
  const T* const factors = (const T*)a.packed + (first >> 4) * PIECES * kTile + (WHOLE ? lane : q * 16) * (16 / (int)sizeof(T));
  const auto row_of = [&](int t, int e) -> int64_t { return (WHOLE ? t * 16 + e : min(max(t * 16 + q * 4 + e, m), rows)) * a.N; };
  const auto load = [&](int tile, Tile& d) {
    const int t = min(tile, count - 1);
    if constexpr (BASE) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const T* const at = (const T*)a.base + from + row_of(t, e);
        if constexpr (NT == 1) d.base[e] = *at;
        else d.base[e] = load_cols(at);
      }
    }
#pragma unroll
    for (int c = 0; c < PIECES; ++c)
      d.p[c] = load_piece<256>(factors + ((int64_t)t * PIECES + c) * kTile + (WHOLE ? 0 : (min(max(t * 16 + i, m), rows) & 15) * (16 / (int)sizeof(T))));
  };
  const auto finish = [&](int tile, const Tile& d) {
    f4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = mma(frag(d.p[c * PARTS + part]), fw[t][c], acc[t]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      T* const to = (T*)a.y + from + row_of(tile, e);
      if constexpr (NT == 1) *to = (T)(acc[0][e] + (BASE ? (float)d.base[e] : 0.0f));
      else *(typename Cols<T>::V*)to = sum_cols(BASE ? d.base[e] : Cols<T>{}, acc, e).v;
    }
  };
  Tile d[DEPTH];
#pragma unroll
  for (int s = 0; s < DEPTH - 1; ++s) load(s, d[s]);
  int at = 0;
  for (; at + DEPTH <= count; at += DEPTH) {
#pragma unroll
    for (int s = 0; s < DEPTH; ++s) {
      load(at + s + DEPTH - 1, d[(s + DEPTH - 1) % DEPTH]);
      __builtin_amdgcn_sched_barrier(0);
      finish(at + s, d[s]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int s = 0; s < DEPTH - 1; ++s)
    if (at + s < count) finish(at + s, d[s]);
}

// y = base in the rows of [row, end), NT columns a lane from col on; 32 rows are loaded together, the last one more than once.
template <class T, int NT>
__device__ __forceinline__ void copy_rows(const AdapterExpand& a, int64_t row, int64_t end, int64_t col) {
  const int q = (threadIdx.x & 63) >> 4;
  for (; row < end; row += 32) {
    typedef std::conditional_t<NT == 1, T, typename Cols<T>::V> V;
    V v[8]{};
    if (a.base) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = *(const V*)((const T*)a.base + min(row + e * 4 + q, end - 1) * a.N + col);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) *(V*)((T*)a.y + min(row + e * 4 + q, end - 1) * a.N + col) = v[e];
  }
}

// A lane's ranks of a row of weights: bfloat16 8 q .. + 7 of each chunk (of its half, where that is all), fp32 4 q .. + 3 and 16 + 4 q .. + 3.
template <class T, int CHUNKS, bool PACK>
__device__ __forceinline__ void load_ranks(const T* w, int rank, Frag<T> (&out)[CHUNKS]) {
  const int q = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) out[c] = frag(load_piece_end(w + c * 32, PACK ? q & 1 : q, rank - c * 32, rank));
}

// RC chunks of 32 ranks (0: at most 16 ranks; in bfloat16 the chunk's second half is the second part of the same ranks).  A wave holds the
// factors of 128 columns (fp32: 64) and goes over the rows; the four waves of a workgroup are side by side.
template <class T, int RC, int DEPTH>
__global__ __launch_bounds__(256, RC <= 2 ? 2 : 1) void expand_kernel(const AdapterExpand a, int col_groups, int64_t chunk) {
  constexpr bool kSingle = sizeof(T) == 4, kPack = RC == 0 && !kSingle;
  constexpr int kChunks = RC == 0 ? 1 : RC, kParts = kSingle || kPack ? 1 : 2, NT = kCols<T>;
  const int lane = threadIdx.x & 63, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n = ((int64_t)(blockIdx.x % col_groups) * 4 + wave) * (16 * NT);
  if (n >= a.N) return;
  const bool few = n + NT > a.N;             // the last columns, too few for a load of NT: one a lane
  const int64_t row0 = (int64_t)(blockIdx.x / col_groups) * chunk, row1 = min(row0 + chunk, a.b.L);

  for (int64_t row = row0; row < row1;) {
    const Run run = run_at(a.b, row, row1);
    const T* const w = (const T*)a.w + run.adapter * a.w_stride;
    if (run.adapter < 0) {
      if (run.adapter == -1 && a.base != a.y) {
        if (few) copy_rows<T, 1>(a, row, run.end, min(n + i, a.N - 1));
        else copy_rows<T, NT>(a, row, run.end, min(n + i * NT, a.N - NT));
      }
    } else if (few) {
      const int64_t col = min(n + i, a.N - 1);          // the last one more than once
      Frag<T> fw[1][kChunks];
      load_ranks<T, kChunks, kPack>(w + col * a.w_pitch, a.rank, fw[0]);
      if (a.base) expand_tiles<T, 1, kChunks * kParts, kChunks, kParts, DEPTH, true, false>(a, row, run.end, col, fw);
      else expand_tiles<T, 1, kChunks * kParts, kChunks, kParts, DEPTH, false, false>(a, row, run.end, col, fw);
    } else {
      const int64_t col = min(n + i * NT, a.N - NT);    // past the last column: the last NT once more
      Frag<T> fw[NT][kChunks];
#pragma unroll
      for (int t = 0; t < NT; ++t) load_ranks<T, kChunks, kPack>(w + (col + t) * a.w_pitch, a.rank, fw[t]);
      const auto tiles = [&](auto base, auto full) {
        expand_tiles<T, NT, kChunks * kParts, kChunks, kParts, DEPTH, decltype(base)::value, decltype(full)::value>(a, row, run.end, col, fw);
      };
      const std::true_type yes{};
      const std::false_type no{};
      if (((row | run.end) & 15) == 0) a.base ? tiles(yes, yes) : tiles(no, yes);
      else a.base ? tiles(yes, no) : tiles(no, no);
    }
    row = run.end;
  }
}

// The same with factors in slices that are summed here, so that they cannot be asked for so far ahead: for few rows.  Columns are the
// product's rows: lane (i, q) ends with columns NT (4 q + e) + t of row i.
template <class T, int RC>
__global__ __launch_bounds__(256, RC <= 2 ? 2 : 1) void expand_slices_kernel(const AdapterExpand a, int col_groups, int64_t chunk) {
  constexpr bool kSingle = sizeof(T) == 4, kPack = RC == 0 && !kSingle;
  constexpr int kChunks = RC == 0 ? 1 : RC, kParts = kSingle || kPack ? 1 : 2, NT = kCols<T>;
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = (int)(blockIdx.x % col_groups);
  const int64_t n = ((int64_t)group * 4 + wave) * (16 * NT);
  if (n >= a.N) return;
  const bool whole = n + 16 * NT <= a.N;
  const int64_t row0 = (int64_t)(blockIdx.x / col_groups) * chunk, row1 = min(row0 + chunk, a.b.L);
  const bool writes_u = a.u && group == 0 && wave == 0;

  for (int64_t row = row0; row < row1;) {
    const Run run = run_at(a.b, row, row1);
    if (run.adapter == -2) {
      row = run.end;
      continue;
    }
    const bool none = run.adapter < 0;
    const float scale = none ? 0.0f : a.scale ? a.scale[run.adapter] : 1.0f;
    Frag<T> fw[NT][kChunks];
    if (!none) {
      const T* const w = (const T*)a.w + run.adapter * a.w_stride;
#pragma unroll
      for (int t = 0; t < NT; ++t) load_ranks<T, kChunks, kPack>(w + min(n + i * NT + t, a.N - 1) * a.w_pitch, a.rank, fw[t]);
    }
    for (int64_t at = row; at < run.end; at += 16) {
      const int64_t l = min(at + i, run.end - 1);
      const bool mine = at + i < run.end;
      f4 acc[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      if (!none) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const int jq = kPack ? q & 1 : q, left = a.rank - c * 32;
          Piece<float> p = load_piece_as<T>(a.p + l * a.pitch + c * 32, jq, left);
#pragma unroll 4
          for (int s = 1; s < a.slices; ++s) {
            const Piece<float> more = load_piece_as<T>(a.p + ((int64_t)s * a.b.L + l) * a.pitch + c * 32, jq, left);
            p.v[0] += more.v[0];
            p.v[1] += more.v[1];
          }
          if (writes_u && mine && !(kPack && q >= 2)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int j = kSingle ? e / 4 * 16 + q * 4 + e % 4 : q * 8 + e;
              if (j < left) a.u[l * a.rank + c * 32 + j] = p.v[e / 4][e % 4];
            }
          }
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = p.v[e / 4][e % 4] * scale;
          Frag<T> f[kParts];
          if constexpr (kSingle) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[0].v[e] = v[e];
          } else if constexpr (kPack) {
            Frag<bf16> two[2];
            split8<2>(v, two);
            f[0] = q < 2 ? two[0] : two[1];
          } else {
            split8<2>(v, f);
          }
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mma(fw[t][c], f[part], acc[t]);
        }
      } else if (writes_u && mine) {
        for (int j = q; j < a.rank; j += 4) a.u[l * a.rank + j] = 0.0f;
      }
      const int64_t to = l * a.N + n + q * (4 * NT);
      if (mine && whole) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Cols<T> base = a.base ? load_cols((const T*)a.base + to + e * NT) : Cols<T>{};
          *(typename Cols<T>::V*)((T*)a.y + to + e * NT) = sum_cols(base, acc, e).v;
        }
      } else if (mine) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (n + q * (4 * NT) + e * NT + t < a.N)
              ((T*)a.y)[to + e * NT + t] = (T)(acc[t][e] + (a.base ? (float)((const T*)a.base)[to + e * NT + t] : 0.0f));
      }
    }
    row = run.end;
  }
}

// One row a workgroup and `span` columns of it: a row of weights is dealt to its rank / 8 lanes (a power of two, from 1 to 16), so that a wave
// reads 1024 bytes in a row.  For rows that have an adapter each there is nothing that a matrix instruction could share (64 requests, 11008 columns,
// rank 16: 8.4 us, 21.5 in tiles of 16 rows).
template <class T>
__global__ __launch_bounds__(256) void expand_row_kernel(const AdapterExpand a, int cuts, int64_t span) {
  __shared__ float s_p[kMaxRank];
  const int tid = threadIdx.x, per = a.rank / 8;                // lanes of a column
  const int64_t row = blockIdx.x / cuts, n0 = (int64_t)(blockIdx.x % cuts) * span, n1 = min(n0 + span, a.N);
  if (n0 >= a.N) return;
  const Run run = run_at(a.b, row, row + 1);
  if (run.adapter == -2) return;
  const int step = 256 / per, j0 = tid % per * 8;
  if (run.adapter < 0) {
    for (int64_t n = n0 + tid; n < n1; n += 256)
      ((T*)a.y)[row * a.N + n] = a.base ? ((const T*)a.base)[row * a.N + n] : (T)0.0f;
    if (a.u && n0 == 0 && tid < a.rank) a.u[row * a.rank + tid] = 0.0f;
    return;
  }
  constexpr int kAhead = 4;
  const T* const w = (const T*)a.w + run.adapter * a.w_stride + j0;
  const int64_t first = n0 + tid / per;
  Raw8<T> next[kAhead];
#pragma unroll
  for (int s = 0; s < kAhead; ++s) next[s] = load8(w + min(first + s * step, a.N - 1) * a.w_pitch, 8);
  if (tid < a.rank) {
    float v = 0.0f;
#pragma unroll 8
    for (int s = 0; s < a.slices; ++s) v += a.p[((int64_t)s * a.b.L + row) * a.pitch + tid];
    if (a.u && n0 == 0) a.u[row * a.rank + tid] = v;
    s_p[tid] = v * (a.scale ? a.scale[run.adapter] : 1.0f);
  }
  __syncthreads();
  float p[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = s_p[j0 + e];
  for (int64_t n = first, left = ceil_of(n1 - n0, kAhead * step); left > 0; --left, n += kAhead * step) {
    Raw8<T> now[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) now[s] = next[s];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) next[s] = load8(w + min(n + (kAhead + s) * step, a.N - 1) * a.w_pitch, 8);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      float x[8], sum = 0.0f;
      widen(now[s], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(x[e], p[e], sum);
      if (per >= 2) sum += lane_xor<1>(sum);
      if (per >= 4) sum += lane_xor<2>(sum);
      if (per >= 8) sum += lane_xor<4>(sum);
      if (per >= 16) sum += lane_xor<8>(sum);
      const int64_t c = n + s * step;
      if (tid % per == 0 && c < n1) {
        const int64_t at = row * a.N + c;
        ((T*)a.y)[at] = (T)(sum + (a.base ? (float)((const T*)a.base)[at] : 0.0f));
      }
    }
  }
}

// ---- what a backward call needs first -------------------------------------------------------------
// Workgroups of the first blocks: the segments of a range of adapters each, in the order they have, behind those of the lower ones.  The others:
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

// A workgroup reads every segment twice, so there are at most kSorts of them, whatever the adapters are: 65536 adapters are ranges of 256
// (262144 segments: 0.67 ms, with a workgroup for each adapter 32.4).  2^20 segments of 16 adapters: 6.5 ms, all in the order of the waves.
constexpr int kSorts = 256, kSortRange = 256;
__device__ void sort_segments(const AdapterPrepare& a, int k0, int k1) {
  __shared__ int64_t s_sum[4];
  __shared__ uint32_t s_rows[kSortRange], s_count[kSortRange];      // of each adapter's segments; then where its next one goes
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int L = (int)a.b.L, range = k1 - k0;
  // Four segments' adapters (-1 past the last one) and lengths, 64 apart, in loads that wait together.
  struct Four {
    int x[4];
    uint32_t len[4];
  };
  const auto load = [&](int s, Four& f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = min(s + e * 64, a.b.segments - 1);
      const int b = min(max(a.b.offsets[at], 0), L);
      f.len[e] = (uint32_t)(min(max(a.b.offsets[at + 1], b), L) - b);
      f.x[e] = s + e * 64 < a.b.segments ? a.b.index[at] : -1;
    }
  };
  s_rows[tid] = s_count[tid] = 0;
  __syncthreads();
  int64_t before = 0;                       // rows, and (upper half) segments, of lower adapters
  for (int s0 = wave * 256 + lane; s0 < a.b.segments; s0 += 1024) {
    Four f;
    load(s0, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (f.x[e] >= 0 && f.x[e] < k0) before += (int64_t)1 << 32 | (int64_t)f.len[e];
      if (range > 1 && f.x[e] >= k0 && f.x[e] < k1) {
        atomicAdd(&s_rows[f.x[e] - k0], f.len[e]);
        atomicAdd(&s_count[f.x[e] - k0], 1u);
      }
    }
  }
  before = block_sum(before, s_sum);
  uint32_t rows = (uint32_t)before & 0x7FFFFFFFu, count = (uint32_t)(before >> 32) & 0x7FFFFFFFu;
  if (range > 1) {                          // those of the range's lower ones too
    const uint32_t own_rows = s_rows[tid], own_count = s_count[tid];
    uint32_t r = own_rows, c = own_count;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const uint32_t r_other = __shfl_up(r, m), c_other = __shfl_up(c, m);
      if (lane >= m) {
        r += r_other;
        c += c_other;
      }
    }
    __syncthreads();
    if (lane == 63) s_sum[wave] = (int64_t)c << 32 | r;
    __syncthreads();
    rows += r - own_rows;
    count += c - own_count;
    for (int w = 0; w < wave; ++w) {
      rows += (uint32_t)s_sum[w];
      count += (uint32_t)(s_sum[w] >> 32);
    }
  }
  s_rows[tid] = rows;
  s_count[tid] = count;
  if (tid < range) a.first[k0 + tid] = (int)rows;
  __syncthreads();
  Four next;
  load(wave * 256 + lane, next);
  for (int s0 = 0; s0 < a.b.segments; s0 += 1024) {
    const int first = s0 + wave * 256 + lane;
    const Four f = next;
    load(min(first, a.b.segments) + 1024, next);      // on their way meanwhile
    for (int w = 0; w < 4; ++w) {           // the waves in turn, in each one adapter after the other
      if (wave == w) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int s = first + e * 64, x = f.x[e];
          const bool mine = x >= k0 && x < k1;
          for (uint64_t left = __builtin_amdgcn_ballot_w64(mine); left;) {
            const int k = __builtin_amdgcn_readlane(x, __ffsll((unsigned long long)left) - 1);
            const uint64_t same = __builtin_amdgcn_ballot_w64(mine && x == k);
            const bool here = same >> lane & 1;
            const uint32_t own = here ? f.len[e] : 0;
            uint32_t len = own;
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
              const uint32_t other = __shfl_up(len, m);
              if (lane >= m) len += other;
            }
            const uint32_t at = s_rows[k - k0], place = s_count[k - k0] + __popcll(same & ((1ull << lane) - 1));
            if (here && place < (uint32_t)a.b.segments) {      // always, but for offsets that do not ascend
              a.order[place] = s;
              a.start[place] = (int)(at + len - own);
            }
            if (lane == 63) {
              s_rows[k - k0] = at + len;
              s_count[k - k0] = place + (here ? 1 : 0);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // the next of these may be read in the next trip
            left &= ~same;
          }
        }
      }
      __syncthreads();
    }
  }
  if (k1 == a.b.adapters) {                 // behind the last one: all that no adapter has, past every row
    const int end = (int)s_rows[range - 1], done = (int)s_count[range - 1];
    if (tid == 0) a.first[k1] = end;
    for (int s = done + tid; s <= a.b.segments; s += 256) {
      a.start[s] = end;
      if (s < a.b.segments) a.order[s] = 0;
    }
  }
}

// Rows `j` and reduced elements `k` of weights, at j * by_j + k * by_k, in the order of the lanes: [K / 32][tiles of 16 rows] packed tiles, zeros past
// the last ones.  A lane: eight of them.
template <class T>
__device__ void pack_weights(const T* w, int64_t by_j, int64_t by_k, int rows, int64_t K, T* out, int64_t block) {
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4, tiles = (rows + 15) / 16;
  const int64_t tile = block * 4 + (threadIdx.x >> 6), k0 = tile / tiles * 32;
  if (k0 >= ((K + 63) & -64ll)) return;
  const int j = (int)(tile % tiles) * 16 + i;
  T v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t k = k0 + (sizeof(T) == 4 ? e / 4 * 16 + q * 4 + e % 4 : q * 8 + e);
    v[e] = j < rows && k < K ? w[j * by_j + k * by_k] : (T)0.0f;
  }
  T* const to = out + tile * kTile;
#pragma unroll
  for (int e = 0; e < 8; ++e) to[sizeof(T) == 4 ? e / 4 * 256 + lane * 4 + e % 4 : lane * 8 + e] = v[e];
}

// at[n][j] of a [rank x I].
template <class T>
__device__ void transpose_tile(const T* from, int64_t rows, int64_t cols, T* to, int64_t r0, int64_t c0) {
  __shared__ T s_tile[64][65];
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  for (int r = y; r < 64; r += 4)
    if (r0 + r < rows && c0 + x < cols) s_tile[r][x] = from[(r0 + r) * cols + c0 + x];
  __syncthreads();
  for (int c = y; c < 64; c += 4)
    if (c0 + c < cols && r0 + x < rows) to[(c0 + c) * rows + r0 + x] = s_tile[x][c];
}

template <class T>
__global__ __launch_bounds__(256) void prepare_kernel(const AdapterPrepare a, int sorts, int range, int tiles_a, int tiles_w, int rank_tiles) {
  int b = blockIdx.x;
  if (b < sorts) {
    sort_segments(a, b * range, min((b + 1) * range, a.b.adapters));
    return;
  }
  b -= sorts;
  const int per = tiles_a + tiles_w, k = b / per, t = b % per;
  if (t < tiles_a)
    transpose_tile((const T*)a.a + (int64_t)k * a.rank * a.I, a.rank, a.I, (T*)a.at + (int64_t)k * a.I * a.rank, (int64_t)(t % rank_tiles) * 64,
                   (int64_t)(t / rank_tiles) * 64);
  else
    pack_weights((const T*)a.w + (int64_t)k * a.rank * a.K, a.by_j, a.by_k, a.rank, a.K, (T*)a.wt + k * a.wt_stride, t - tiles_a);
}

// ---- outer ----------------------------------------------------------------------------------------
// Rows of a part of the sums over `total` rows.
__device__ __forceinline__ int64_t rows_of_part(int64_t total, int parts) { return ((total + parts - 1) / parts + 31) & -32ll; }

// Row e of lane quarter q in a step of 32 rows, in the order that pieces have.
template <class T>
__device__ __forceinline__ int row_in_step(int q, int e) { return sizeof(T) == 4 ? e / 4 * 16 + q * 4 + e % 4 : q * 8 + e; }
// Rows m .. n - 1 of a step, zeros beside them.
__device__ __forceinline__ void keep_rows(Piece<bf16>& p, int q, int m, int n) {
#pragma unroll
  for (int e = 0; e < 8; ++e) p.v[e] = row_in_step<bf16>(q, e) >= m && row_in_step<bf16>(q, e) < n ? p.v[e] : (uint16_t)0;
}
__device__ __forceinline__ void keep_rows(Piece<float>& p, int q, int m, int n) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    p.v[e / 4][e % 4] = row_in_step<float>(q, e) >= m && row_in_step<float>(q, e) < n ? p.v[e / 4][e % 4] : 0.0f;
}

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

// u and g_u for the sums over rows: rows in the order of their adapters, a rank's factors of 32 rows one after the other, so that a lane's eight
// rows are one load; bfloat16 in its three parts.  packed tiles of 16 ranks and 32 rows, [steps of 32 rows][parts][tiles]: what a wave loads lies
// together, in the order of its lanes.  A workgroup: 64 positions of one operand.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const AdapterPack a) {
  constexpr int kParts = sizeof(T) == 4 ? 1 : 3;
  __shared__ float s_p[kMaxRank * 65];
  __shared__ int s_row[64];
  const int tid = threadIdx.x;
  const bool second = blockIdx.y != 0;
  const int64_t pos0 = (int64_t)blockIdx.x * 64;
  const int64_t total = a.first ? max(min((int64_t)a.first[a.b.adapters], a.b.L), (int64_t)0) : a.b.L;
  if (pos0 >= total) return;
  if (tid < 64) {
    const int pos = (int)min(pos0 + tid, total - 1);
    int64_t row = pos;
    if (a.first) {
      int lo = 0, n = a.b.segments + 1;          // the last segment that starts at or before it
      while (n > 1) {
        const int half = n / 2;
        if (a.start[lo + half] <= pos) {
          lo += half;
          n -= half;
        } else {
          n = half;
        }
      }
      lo = min(lo, a.b.segments - 1);
      row = min(max((int64_t)a.b.offsets[min(max(a.order[lo], 0), a.b.segments - 1)] + pos - a.start[lo], (int64_t)0), a.b.L - 1);
    }
    if (!second) a.rows[pos0 + tid] = (int)row;
    s_row[tid] = (int)row;
  }
  __syncthreads();
  const float* const p = second ? a.u : a.g_u;
  const int pitch = second ? a.rank : a.g_pitch, slices = second ? 1 : a.slices, ranks = (a.rank + 15) & -16;
  for (int at = tid; at < 64 * ranks; at += 256) {
    const int j = at % ranks, x = at / ranks;
    float v = 0.0f;
    if (j < a.rank) {
      for (int s = 0; s < slices; ++s) v += p[((int64_t)s * a.b.L + s_row[x]) * pitch + j];
    }
    s_p[j * 65 + x] = v;
  }
  __syncthreads();
  T* const out = (T*)(second ? a.u_out : a.g_out);
  for (int at = tid; at < 8 * ranks; at += 256) {
    const int j = at / 8, x = at % 8 * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s_p[j * 65 + x + e];
    T* const to = out + ((pos0 + x) / 32 * kParts * (ranks / 16) + j / 16) * kTile;
    const int q = x % 32 / 8;
    if constexpr (kParts == 1) {
#pragma unroll
      for (int e = 0; e < 2; ++e)       // rows 8 q + 4 e .. + 3 of 32: piece x % 32 / 16, of lane (j, x / 4 % 4)
        *(f4_any*)((float*)to + (x % 32 / 16) * 256 + (((x / 4 + e) & 3) * 16 + j % 16) * 4) = f4_any{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
    } else {
      Frag<bf16> f[kParts];
      split8<kParts>(v, f);
#pragma unroll
      for (int part = 0; part < kParts; ++part) *(u4*)(to + part * (ranks / 16) * kTile + (q * 16 + j % 16) * 8) = f[part].v;
    }
  }
}

constexpr int kOuterCols = 128, kOuterWaves = 4;    // columns of a wave, waves of a workgroup side by side

// A wave: 128 columns, up to 64 ranks, one part of the rows that have adapters, in steps of 32, DEPTH of them on their way.  The four waves
// of a workgroup are side by side and share the rows' factors through LDS: each loads a quarter, with its rows, so that both are as far
// ahead (a wait for factors loaded later than rows is one for the rows).  Sums over rows leave as one partial sum a part and adapter.
// 16384 x (4096 + 11008) bfloat16, rank 64: 130 to 145 us for 495 MB of rows (each wave loading all factors: 175), 4.1 TB/s with the factors; matrix and
// vector pipes are busy for 31 and 30 % of it, and the one wave a SIMD that 64 ranks leave room for waits with the others at every step's
// barrier.  12608 x (768 + 2304) fp32, rank 16: 32.7 us for 155 MB, 4.7 TB/s.
// MODE: 0 all rows as they lie, 1 in the order of a.rows, 2 too, with fewer than eight columns in one of the products.
template <class T, int RT, int MODE, int DEPTH>
__global__ __launch_bounds__(64 * kOuterWaves) void outer_kernel(const AdapterOuter a, int tiles_first, int tiles, int rank_blocks) {
  constexpr int kParts = sizeof(T) == 4 ? 1 : 3, kHeld = 16;       // steps whose rows' numbers are held
  constexpr int kFactors = kParts * RT, kOwn = (kFactors + kOuterWaves - 1) / kOuterWaves;   // packed tiles of a step, of a wave
  __shared__ int s_rows[kOuterWaves][MODE ? kHeld * 32 : 1];
  __shared__ Piece<T> s_p[2][kFactors][64];
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = blockIdx.x / (tiles * rank_blocks), in = blockIdx.x % (tiles * rank_blocks);
  const int tile = in % tiles, rank0 = in / tiles * 64, ranks = (a.rank + 15) & -16;
  const bool second = tile >= tiles_first;
  const AdapterOuterOperand o = second ? a.a[1] : a.a[0];
  const int64_t col0 = ((int64_t)(second ? tile - tiles_first : tile) * kOuterWaves + wave) * kOuterCols;
  // Columns past the last one: the last eight once more, which come out the same.
  const bool narrow = MODE == 2 && o.N < 8;
  const int64_t col = narrow ? col0 + i * 8 : min(col0 + i * 8, o.N - 8);
  const int have = narrow ? (int)max(min((int64_t)8, o.N - col), (int64_t)0) : 8;
  const int64_t total = a.first ? max(min((int64_t)a.first[a.b.adapters], a.b.L), (int64_t)0) : a.b.L;
  const int64_t per = rows_of_part(total, a.parts);
  const int64_t hi = min(per * (part + 1), total);

  for (int64_t pos = per * part; pos < hi;) {
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
    const T* const p_at = (const T*)o.p + rank0 * 32 + lane * (16 / (int)sizeof(T));
    const int64_t begin = pos & -32ll, last = (k_end - 1) & -32ll;          // the first and the last step
    const int steps = (int)((last - begin) / 32) + 1;
    struct Step {
      Raw8<T> x[8];
      Piece<T> p[kOwn];
    };
    const auto load = [&](int step, Step& d) {
      const int64_t at = begin + min(step, steps - 1) * 32;
      if (MODE && step < steps && step % kHeld == 0) {          // the rows' numbers, for many steps at once: a wait for them is one for all
        const int64_t l = at + lane * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) s_rows[wave][lane * 8 + e] = a.rows[max(min(l + e, k_end - 1), pos)];
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {     // beside the adapter's rows: its nearest one, times zero
        const int64_t r = MODE ? s_rows[wave][min(step, steps - 1) % kHeld * 32 + row_in_step<T>(q, e)] : max(min(at + row_in_step<T>(q, e), k_end - 1), pos);
        const T* const from = (const T*)o.q + r * o.N + col;
        if (narrow) d.x[e] = load8(from, have);
        else d.x[e] = load8(from, 8);
      }
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {  // ranks past the last tile: the last tile's, whose sums are not stored
        const int tile = min(wave + k * kOuterWaves, kFactors - 1), t = min(tile % RT, (ranks - rank0) / 16 - 1);
        d.p[k] = load_piece<256>(p_at + at * kParts * ranks + (tile / RT * (ranks / 16) + t) * kTile);
      }
    };
    const auto multiply = [&](int step, Step& d) {
      const int64_t at = begin + step * 32;
      const int n = (int)min(k_end - at, (int64_t)32), m = (int)max(pos - at, (int64_t)0);
      Piece<T>(&slot)[kFactors][64] = s_p[step & 1];
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        keep_rows(d.p[k], q, m, n);
        slot[min(wave + k * kOuterWaves, kFactors - 1)][lane] = d.p[k];
      }
      // The waves are done with this slot's last content: they have passed the barrier of the step between.
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      Frag<T> f[8];
      columns_of(d.x, f);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int s = 0; s < kParts; ++s) {
          const Frag<T> p = frag(slot[s * RT + t][lane]);
#pragma unroll
          for (int c = 0; c < 8; ++c) acc[t][c] = mma(p, f[c], acc[t][c]);
        }
    };
    // DEPTH steps on their way, as in the first product; every wave takes every step, for the barriers.
    Step d[DEPTH];
#pragma unroll
    for (int s = 0; s < DEPTH - 1; ++s) load(s, d[s]);
    int at = 0;
    for (; at + DEPTH <= steps; at += DEPTH) {
#pragma unroll
      for (int s = 0; s < DEPTH; ++s) {
        load(at + s + DEPTH - 1, d[(s + DEPTH - 1) % DEPTH]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(at + s, d[s]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int s = 0; s < DEPTH - 1; ++s)
      if (at + s < steps) multiply(at + s, d[s]);
    __syncthreads();          // the next adapter begins with the first slot again
    pos = k_end;
    // Lane (i, q) has ranks 16 t + 4 q + e of its eight columns.
    const float scale = a.scale ? a.scale[k] : 1.0f;
    float* const to = o.part + (int64_t)(part + k) * a.rank * o.N;
    if (col0 + i * 8 < o.N) {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = rank0 + t * 16 + q * 4 + e;
          float v[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) v[c] = acc[t][c][e] * scale;
          if (j < a.rank) store8(to + (int64_t)j * o.N + col, v, have);
        }
    }
  }
}

// Sums of the parts of each adapter, in order; part p of adapter k is slot p + k.  A workgroup: 64 columns of 4 / G ranks, the parts of
// each in G runs of lanes that are joined through LDS.
template <int G>
__global__ __launch_bounds__(256) void reduce_kernel(const AdapterReduce a, int64_t block, int tiles_a, int tiles, int ranks) {
  block += blockIdx.x;
  constexpr int kRanks = 4 / G;
  __shared__ float s_sum[4][64];
  const int tid = threadIdx.x, x = tid & 63, y = tid >> 6;
  const int k = (int)(block / ((int64_t)tiles * ranks)), in = (int)(block % ((int64_t)tiles * ranks)), tile = in / ranks;
  const int j0 = in % ranks * kRanks, j = j0 + y / G;
  const int64_t total = a.first ? max(min((int64_t)a.first[a.adapters], a.L), (int64_t)0) : a.L;
  const int64_t lo = a.first ? max(a.first[k], 0) : (k == 0 ? 0 : total), hi = a.first ? min((int64_t)a.first[k + 1], total) : total;
  const int64_t per = rows_of_part(total, a.parts);         // the parts that hold rows of this adapter
  const int p0 = lo < hi ? (int)(lo / per) : 0, p1 = lo < hi ? (int)min((hi + per - 1) / per, (int64_t)a.parts) : 0;
  const int run = (p1 - p0 + G - 1) / G, b = p0 + y % G * run, e = min(b + run, p1);
  const bool second = tile >= tiles_a;
  const int64_t N = second ? a.O : a.I, n0 = (int64_t)(second ? tile - tiles_a : tile) * 64, n = n0 + x;
  float v = 0.0f;
  if (n < N && j < a.rank) {
    const float* from = (second ? a.part_b : a.part_a) + ((int64_t)(b + k) * a.rank + j) * N + n;
#pragma unroll 8
    for (int p = b; p < e; ++p, from += a.rank * N) v += *from;
  }
  s_sum[y][x] = v;
  __syncthreads();
  if (second) {             // [n][rank]: a column's ranks side by side
    const int c = tid / kRanks, r = tid % kRanks;
    if (tid < 64 * kRanks && n0 + c < N && j0 + r < a.rank) {
      float t = 0.0f;
#pragma unroll
      for (int g = 0; g < G; ++g) t += s_sum[r * G + g][c];
      a.g_b[((int64_t)k * N + n0 + c) * a.rank + j0 + r] = t;
    }
  } else if (y < kRanks && n < N && j0 + y < a.rank) {
    float t = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) t += s_sum[y * G + g][x];
    a.g_a[((int64_t)k * a.rank + j0 + y) * N + n] = t;
  }
}

template <class T, int RT>
hipError_t run_shrink(const AdapterShrink& a, int tile, hipStream_t s) {
  constexpr int kDepth = RT <= 2 ? 4 : RT == 4 ? 3 : 2;     // as the registers of two waves allow
  const uint32_t grid = (uint32_t)(ceil_div(a.b.L, tile) * a.slices);
  const auto run = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(a); };
  if (tile == 1) a.w_packed ? run(shrink_kernel<T, RT, 1, 1, kDepth, true>) : run(shrink_kernel<T, RT, 1, 1, kDepth, false>);
  else if (tile == 16) a.w_packed ? run(shrink_kernel<T, RT, 1, 16, kDepth, true>) : run(shrink_kernel<T, RT, 1, 16, kDepth, false>);
  else if constexpr (RT <= 4) {
    if (tile == 32) a.w_packed ? run(shrink_kernel<T, RT, 2, 32, kDepth, true>) : run(shrink_kernel<T, RT, 2, 32, kDepth, false>);
    else if constexpr (RT >= 2) run(shrink_kernel<T, RT, 4, 64, 3, true>);
  }
  return hipGetLastError();
}
template <class T>
hipError_t shrink_of(const AdapterShrink& a, int tile, hipStream_t s) {
  if (a.rank <= 16) return run_shrink<T, 1>(a, tile, s);
  if (a.rank <= 32) return run_shrink<T, 2>(a, tile, s);
  if (a.rank <= 64) return run_shrink<T, 4>(a, tile, s);
  return run_shrink<T, 8>(a, tile, s);
}

template <class T, int RC>
hipError_t run_expand(const AdapterExpand& a, bool rows, hipStream_t s) {
  constexpr int kDepth = RC <= 2 ? 3 : 2;
  const int64_t groups = ceil_div(a.N, 64 * kCols<T>);
  // Packed factors are asked for ahead, so that workgroups need only be as many as are resident; slices are waited for, and more waves hide
  // that (packed, 12608 x 768 fp32: 21.7 us, with 1024 of them 26.4; four slices, 3330 x 2307 bfloat16: 26 us, with 512 of them 32.5).
  const int64_t wanted = a.packed ? 512 : 1024;
  const int64_t chunk = rows ? ceil_div(a.b.L * groups, 1 << 22) : round_up(ceil_div(a.b.L, groups < wanted ? wanted / groups : 1), 16);
  const uint32_t grid = (uint32_t)(groups * ceil_div(a.b.L, chunk));
  if (a.packed) expand_kernel<T, RC, kDepth><<<grid, 256, 0, s>>>(a, (int)groups, chunk);
  else expand_slices_kernel<T, RC><<<grid, 256, 0, s>>>(a, (int)groups, chunk);
  return hipGetLastError();
}
template <class T>
hipError_t expand_of(const AdapterExpand& a, bool rows, hipStream_t s) {
  const int per = a.rank / 8;
  if (rows && a.rank % 8 == 0 && (per & (per - 1)) == 0) {
    const int64_t step = 256 / per, steps = ceil_div(a.N, step);
    int64_t cuts = ceil_div(1024, a.b.L);
    if (a.b.L > 1 && cuts < 8 && steps >= 64) cuts = 8;
    if (cuts > steps) cuts = steps;
    const int64_t span = ceil_div(steps, cuts) * step;
    cuts = ceil_div(a.N, span);
    // The eight XCDs take workgroups in turn: with eight cuts or a multiple of them an adapter's cut is read by one of them, for all of its rows
    // (24 adapters, 11008 columns, rank 16: 64 rows 8.4 us, with 15 cuts 9.8; 1000 rows 46.5, with two cuts 50.7).  Cuts of few steps wait more than
    // they read (1000 x 2304: 14.8 us in two, 23 in eight).
    if (cuts > 4 && a.b.L > 1) cuts = round_up(cuts, 8);
    expand_row_kernel<T><<<(uint32_t)(a.b.L * cuts), 256, 0, s>>>(a, (int)cuts, span);
    return hipGetLastError();
  }
  if (a.rank <= 16) return run_expand<T, 0>(a, rows, s);
  if (a.rank <= 32) return run_expand<T, 1>(a, rows, s);
  if (a.rank <= 64) return run_expand<T, 2>(a, rows, s);
  return run_expand<T, 4>(a, rows, s);
}

template <class T>
hipError_t outer_of(const AdapterOuter& a, hipStream_t s) {
  constexpr int kCols = kOuterCols * kOuterWaves;
  const int tiles_first = (int)ceil_div(a.a[0].N, kCols), tiles = tiles_first + (int)ceil_div(a.a[1].N, kCols);
  const int blocks = (int)ceil_div(a.rank, 64);
  const uint32_t grid = (uint32_t)((int64_t)tiles * blocks * a.parts);
  const auto run = [&](auto kernel) { kernel<<<grid, 64 * kOuterWaves, 0, s>>>(a, tiles_first, tiles, blocks); };
  constexpr int kMost = sizeof(T) == 4 ? 2 : 4;      // steps on their way that the registers hold with 64 ranks
  if (a.a[0].N < 8 || a.a[1].N < 8) run(outer_kernel<T, 4, 2, 2>);
  else if (a.first) a.rank <= 16 ? run(outer_kernel<T, 1, 1, 3>) : a.rank <= 32 ? run(outer_kernel<T, 2, 1, 3>) : run(outer_kernel<T, 4, 1, kMost>);
  else a.rank <= 16 ? run(outer_kernel<T, 1, 0, 3>) : a.rank <= 32 ? run(outer_kernel<T, 2, 0, 3>) : run(outer_kernel<T, 4, 0, kMost>);
  return hipGetLastError();
}

}  // namespace

AdapterPlan adapter_plan(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters, int64_t segments) {
  AdapterPlan p{};
  const int64_t size = type == HOT_BF16 ? 2 : 4, step = 128 / size;
  p.rows = L <= 4 * (segments > 0 ? segments : 1) && L <= 1 << 20;
  p.pitch = (int)round_up(rank, 8);      // zeros behind the ranks
  // Rows of a workgroup: 16 to 64.  First product and expansion of a bfloat16 pass 4096 -> 11008, in us with 16 and with 32 rows: rank 16, 1024 rows 30 and
  // 36, 2048 54 and 57, 5000 66 and 100; rank 64 67 and 99, 71 and 92, 82 and 132; fp32, rank 64: 213 and 378, 239 and 401, 187 and 433.  The first
  // product itself is the faster with 32 (5000 rows, fp32, rank 64: 41 for 60), but in slices up to 8192 rows, with 16 up to 4096, which the expansion
  // adds.  So 32 rows pay from where they need no slices; the border here is lower than that.
  p.tile = p.rows ? 1 : L >= 64 * 224 && rank > 16 && rank <= 64 ? 64 : L >= 64 * 32 && rank <= 64 ? 32 : 16;
  // With no slices the expansion finds its factors packed: not where each wave has four steps at most, which are all on their way at once, and
  // the workgroups are not too few (3330 x 771 bfloat16, rank 12: 10.8 us in four slices or in none, and the expansion to 2307 then 26 us or 13.9).
  const auto slices = [&](int64_t K, int& count, int64_t& slice) {
    int64_t n = (p.tile == 64 ? 256 : 512) / ceil_div(L, p.tile);      // workgroups that are resident
    const int64_t most = ceil_div(K, 4 * step);      // a step for each wave
    if (n > most) n = most;
    if (n > kMaxSlices) n = kMaxSlices;
    if (n < 1 || (K <= 16 * step && ceil_div(L, p.tile) >= 64)) n = 1;
    slice = round_up(ceil_div(K, n), 4 * step);
    count = (int)ceil_div(K, slice);
  };
  slices(I, p.slices_forward, p.slice_forward);
  slices(O, p.slices_backward, p.slice_backward);
  // Parts of the sums over rows: workgroups for all compute units (one each with the registers of 64 ranks, two below), and no more, since each part's
  // sums are written and added (8192 rows 4096 -> 11008, rank 64: 67 us and 11 for the parts, with twice as many 81 and 35).  That leaves compute units
  // idle where tiles are just more than half of them (136 tiles, 4096 rows, rank 128: 219 us and 28, in four parts 183 and 38).
  const int64_t tiles = (ceil_div(I, kOuterCols * kOuterWaves) + ceil_div(O, kOuterCols * kOuterWaves)) * ceil_div(rank, 64);
  const int64_t wanted = 256 / tiles, most = ceil_div(L, 64);
  p.parts = (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
  p.positions = round_up(L, 64);

  // Packed weights of the forward call: 2 to 4 us for a launch, against 48 cycles of a compute unit's memory pipe for each kilobyte of
  // weights and 32 rows (16384 x 4096, rank 64: 53 us without).
  p.pack_forward = p.tile == 64 || (!p.rows && ceil_div(L, 32) * (rank * I * size / 1024) > 60000);
  p.chunks = rank <= 16 && type == HOT_BF16 ? 0 : rank <= 32 ? 1 : rank <= 64 ? 2 : 4;    // as the expansion's kernels have them
  p.wt_stride = round_up(rank, 16) * round_up(I > O ? I : O, 64);
  const int64_t row_bytes = L * p.pitch * 4;
  const int64_t factors = ceil_div(L, 16) * kTile * size * (type == HOT_BF16 ? (p.chunks ? 2 * p.chunks : 1) : p.chunks);
  size_t at = 0;
  const auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)round_up(bytes, 256);
    return here;
  };
  const int slices_most = p.slices_forward > p.slices_backward ? p.slices_forward : p.slices_backward;
  take(row_bytes * slices_most);
  p.factors = take(factors);
  p.wt = take(p.pack_forward ? adapters * p.wt_stride * size : 0);
  p.forward = at;
  at = p.wt;
  take(adapters * p.wt_stride * size);
  p.at = take(adapters * I * rank * size);
  p.sorted = take((2 * segments + 1 + adapters + 1 + p.positions) * 4);
  p.packed = take(2 * (type == HOT_BF16 ? 3 : 1) * size * round_up(rank, 16) * p.positions);
  p.part_a = take((p.parts + adapters) * rank * I * 4);
  p.part_b = take((p.parts + adapters) * rank * O * 4);
  p.backward = at;
  return p;
}

hipError_t launch_adapter_shrink(const AdapterShrink& a, int tile, hot_type type, hipStream_t s) {
  return type == HOT_BF16 ? shrink_of<bf16>(a, tile, s) : shrink_of<float>(a, tile, s);
}
hipError_t launch_adapter_expand(const AdapterExpand& a, bool rows, hot_type type, hipStream_t s) {
  return type == HOT_BF16 ? expand_of<bf16>(a, rows, s) : expand_of<float>(a, rows, s);
}
hipError_t launch_adapter_prepare(const AdapterPrepare& a, hot_type type, hipStream_t s) {
  const int range = (int)ceil_div(a.b.adapters, kSorts), sorts = a.order ? (int)ceil_div(a.b.adapters, range) : 0;      // 256 of 256 at most
  const int rank_tiles = (int)ceil_div(a.rank, 64);
  const int tiles_a = a.at ? (int)ceil_div(a.I, 64) * rank_tiles : 0, tiles_w = (int)ceil_div(round_up(a.K, 64) / 32 * ceil_div(a.rank, 16), 4);
  const uint32_t grid = (uint32_t)(sorts + (int64_t)a.b.adapters * (tiles_a + tiles_w));
  if (type == HOT_BF16) prepare_kernel<bf16><<<grid, 256, 0, s>>>(a, sorts, range, tiles_a, tiles_w, rank_tiles);
  else prepare_kernel<float><<<grid, 256, 0, s>>>(a, sorts, range, tiles_a, tiles_w, rank_tiles);
  return hipGetLastError();
}
hipError_t launch_adapter_pack(const AdapterPack& a, hot_type type, hipStream_t s) {
  const dim3 grid((uint32_t)ceil_div(a.b.L, 64), 2);
  if (type == HOT_BF16) pack_kernel<bf16><<<grid, 256, 0, s>>>(a);
  else pack_kernel<float><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_adapter_outer(const AdapterOuter& a, hot_type type, hipStream_t s) {
  return type == HOT_BF16 ? outer_of<bf16>(a, s) : outer_of<float>(a, s);
}
hipError_t launch_adapter_reduce(const AdapterReduce& a, hipStream_t s) {
  const bool runs = a.parts >= 16;
  const int tiles_a = (int)ceil_div(a.I, 64), tiles = tiles_a + (int)ceil_div(a.O, 64), ranks = (int)ceil_div(a.rank, runs ? 1 : 4);
  const int64_t all = (int64_t)a.adapters * tiles * ranks, most = 1 << 23;   // 2^31 lanes a launch
  for (int64_t block = 0; block < all; block += most) {
    const uint32_t grid = (uint32_t)(all - block < most ? all - block : most);
    if (runs) reduce_kernel<4><<<grid, 256, 0, s>>>(a, block, tiles_a, tiles, ranks);
    else reduce_kernel<1><<<grid, 256, 0, s>>>(a, block, tiles_a, tiles, ranks);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace hot
