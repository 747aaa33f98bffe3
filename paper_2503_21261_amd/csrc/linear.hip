// Forward product of a linear layer, y = f(x.w^T + bias) + residual.
//
// Three kernels multiply, and make_plan chooses between them by the time that each is expected to take:
//   linear_rows_kernel            few rows: operands from memory to the matrix instructions, the weight's way from HBM is the time;
//   linear_tile_kernel, direct    small tiles of the operands as they are: products over before operands could be packed;
//   linear_tile_kernel, packed    large tiles, for products that the matrix cores bound; fp32 operands as two fp16 parts.
// Each splits K where its workgroups would leave compute units idle, and a second launch adds the slices' sums in order.
// All sums are fp32.  Sizes are given as L x O x I, times as those of a replayed graph.
#include <math.h>

#include <atomic>
#include <utility>

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

// Floats of a row of a slice's sums.
__host__ __device__ constexpr int64_t sums_pitch(int64_t O) { return (O + 7) / 8 * 8; }

constexpr int kWaves = 8;       // of a workgroup: parts of K
constexpr int kSteps = 4;       // loads of a row on their way together: 4 x 64 bytes

// linear_rows_kernel: NT x 16 outputs and MT x 16 tokens a workgroup, every wave on its part of K; the waves' sums are added in LDS, in
// order.  A lane loads 16 consecutive bytes of a row; bfloat16 rows feed v_mfma_f32_16x16x32_bf16, fp32 rows four
// v_mfma_f32_16x16x4_f32, whose products and sums are plain fp32.  The weight is the first operand, so that a lane's accumulators
// are four consecutive outputs of a token.  Operands do not meet in LDS: a weight row serves MT tokens from registers, and with few
// tokens nothing else would read it.  1 x 4096 x 11008 bfloat16 16.8 us, 5.4 TB/s of weight.  Both sizes are the plan's:
// 62 x 418 x 896 fp32 8.8 us with 16 outputs and 16 tokens, 18.8 with 32 and 64, whose workgroups are too few;
// 191 x 7833 x 8640 bfloat16 341 us against 145, as every operand byte is loaded less often.  K in slices: 18 x 216 x 8281
// bfloat16 45 -> 14 us; 5 x 3118 x 2048 8.0 us whole, 10.6 in slices.
template <class T, class TY, int NT, int MT>
__global__ __launch_bounds__(64 * kWaves) void linear_rows_kernel(const T* x, const T* w, int64_t I, int tiles_m, int slices, float* sums, LinearOut out) {
  constexpr int E = Frag<T>::kElems;
  constexpr int STEP = 4 * E;               // elements of K in one matrix step (64 bytes of a row)
  constexpr int NC = NT * 16, MC = MT * 16;
  constexpr int PITCH = NC + 4;             // of a token's sums in LDS: rows apart by a multiple of 4 banks, not of 16
  __shared__ __align__(16) float s_sum[kWaves * MC * PITCH];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  // slices of K fastest, then tokens: workgroups that share weight rows run side by side
  const int z = (int)blockIdx.x % slices, tile = (int)blockIdx.x / slices;
  const int tm = tile % tiles_m, tn = tile / tiles_m;
  const int64_t k_first = I * z / slices / 16 * 16, k_end = z + 1 < slices ? I * (z + 1) / slices / 16 * 16 : I;
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

  // The waves' spans of K follow each other; all loads of a span are on their way together.
  constexpr int SPAN = STEP * kSteps;
  for (int64_t k0 = k_first + (int64_t)wave * SPAN; k0 < k_end; k0 += (int64_t)kWaves * SPAN) {
    Frag<T> fw[kSteps][NT], fx[kSteps][MT];
    if (k0 + SPAN <= k_end) {
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
        for (int j = 0; j < NT; ++j) fw[s][j] = load_frag(wr[j] + k, k_end - k);
#pragma unroll
        for (int i = 0; i < MT; ++i) fx[s][i] = load_frag(xr[i] + k, k_end - k);
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
    const int n = out.O - n0 - c;
    if (sums) {      // a slice's: added by linear_rows_combine_kernel
      if (n > 0) store8(sums + ((int64_t)z * out.L + m0 + t) * sums_pitch(out.O) + n0 + c, v, 8);
      continue;
    }
    float b[8];
    load_bias8(out, n0 + c, n, b);
    linear_finish8<TY>(out, m0 + t, n0 + c, n, b, v);
  }
}

// The slices' sums, in order, and the epilogue: eight outputs of a token a thread.  Bound by its launch and one way to the caches.
template <class TY>
__global__ __launch_bounds__(256) void linear_rows_combine_kernel(const float* sums, int slices, int chunks, LinearOut out) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = q / chunks;
  const int c = (int)(q % chunks) * 8, n = out.O - c;
  if (row >= out.L) return;
  float v[8] = {};
  if (n > 0) {
#pragma unroll 4
    for (int z = 0; z < slices; ++z) {
      float p[8];
      load_values(sums + ((int64_t)z * out.L + row) * sums_pitch(out.O) + c, 8, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += p[e];
    }
  }
  float b[8];
  load_bias8(out, c, n, b);
  linear_finish8<TY>(out, row, c, n, b, v);
}

// ---- many rows -------------------------------------------------------------------------------------
// linear_tile_kernel: BM tokens x BN outputs a workgroup, both operands through LDS.  Operand rows are K-contiguous; a stage is
// 128 bytes of every row of the tile:
//   bfloat16: 64 elements, of x and w as they are where I is even, else of a padded copy;
//   fp32: 32 elements as two fp16 parts, twice [16 high | 16 low], of the row scaled by a power of two so that its largest
//   value lies in [2^14, 2^15): x = high + low to 22 bits (values down to 2^-17 of the row's largest keep them, smaller
//   ones keep 2^-39 of it), and x.w = high.high + high.low + low.high with 2^-22 left out: a
//   third of the fp16 rate, five times that of the fp32 instructions.  Tiles with rows of so wide a range that this is worse than
//   an fp32 product take those instructions (wide_tile).
// Pieces go from memory to LDS without registers (buffer_load ... lds), two stages deep: one arrives while one is worked on.  LDS
// holds a row's eight 16-byte chunks at chunk ^ (row % 8): eight rows that read the same chunk hit different banks.  As a load
// writes 64 consecutive chunks, it is the lanes' sources that are permuted.
// A wave reads the fragments of a stage's second half under the first half's matrix instructions, then meets the others at a
// barrier, behind which the next stage is complete and this stage's buffer free, and reads the next stage's first half and issues
// the loads of the one behind under the second's.  16 x 16 x 32 instructions: those of 32 x 32 x 16 move a quarter more through the
// registers for each product, and as the chip's power holds such products down, that is time (8192^3 bfloat16 1417 TFLOP/s, 1323
// with them; stages of 64 bytes, four deep: a tenth less).  The weight is the first operand, so that accumulators are runs of four
// outputs of a token; they leave through LDS, a wave's 32 tokens at a time, as runs of eight outputs a lane.
// Measured, in a graph by itself: 16384 x 11008 x 4096 bfloat16 1060 us, 1390 TFLOP/s; with a checkpoint 1080, with GELU 1105 (vector
// instructions of the epilogue, under which no matrix instruction runs), with both 1150, and 1210 to 1260 where its gradient runs between
// its calls; 12608 x 2304 x 768 fp32 126 to 147 us from run to run, 128 at best in each, 1060 to 910 TFLOP/s of fp16 products, and 18 us
// for its operands.
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));

// Compile-time loop: f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>).
template <int... Is, class F>
__device__ __forceinline__ void static_for_impl(std::integer_sequence<int, Is...>, F&& f) {
  (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(std::make_integer_sequence<int, N>{}, static_cast<F&&>(f));
}

// 16 bytes a lane, at byte offset `lane_off` + `off` of the descriptor, to 1024 consecutive bytes of LDS (`to`: the same in
// all lanes).  Counted by vmcnt; the caller waits.  The source may begin at any byte (the memory pipe runs in its unaligned mode):
// at a multiple of four it costs a tenth at most, at an odd multiple of two as much again.
using rsrc_t = decltype(__builtin_amdgcn_make_buffer_rsrc((void*)nullptr, 0, 0, 0));
__device__ __forceinline__ void load_to_lds(rsrc_t from, uint8_t* to, int lane_off, int off) {
#if defined(__HIP_DEVICE_COMPILE__)   // the host's pass does not know gfx950's 16-byte form
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, lane_off, off, 0, 0);
#endif
}

struct TileArgs {
  const uint8_t *x, *w;       // operand rows
  int64_t pitch;              // bytes of one, a multiple of 128 in the first two modes
  const uint8_t *x_plain, *w_plain;   // fp32 in two parts: the rows as they are, for tiles whose rows the parts do not hold (wide_tile)
  int64_t plain_pitch;
  const uint32_t *ex, *ew;    // and a word for each row: its scale and range
  int tiles_m, tiles_n;
  int whole;                  // tiles with a workgroup each; every other one has `slices`, which leave their sums in
  int slices;                 // images[tile - whole][slice], added by linear_combine_kernel
  float* images;
  LinearOut out;
};

constexpr int kStages = 2, kPiece = 128;

template <int BM, int BN, int WM, int WN>
constexpr int kTileLds = kStages * (BM + BN) * kPiece > (BM / WM) * (BN / WN) * 32 * (WN + 4) * 4
                             ? kStages * (BM + BN) * kPiece : (BM / WM) * (BN / WN) * 32 * (WN + 4) * 4;

// What a tile's operand rows are.
enum TileMode {
  kBf16Rows = 0,      // bfloat16, a whole number of pieces
  kSplitRows = 1,     // fp32 in two fp16 parts, a whole number of pieces
  // The others are x and w as they are, of any width from 16 bytes on.  The chunk that reaches past a row's end is loaded as the row's
  // last 16 bytes, so that nothing outside the row is read, and the bytes that belong to the chunk before it are masked.
  kBf16Ragged = 2,    // large tiles, rows of a multiple of four bytes: no copy as kBf16Rows would need
  // Small tiles, several workgroups a compute unit, which hide each other's waits; fp32 on v_mfma_f32_16x16x4_f32.
  // 15774 x 64 x 128 fp32 in 64 x 64 9.2 us, packed 128 x 128 21.9; for 7383 x 1664 x 1152 259 us against 98, where the matrix
  // instructions count.  1872 x 624 x 640 bfloat16 9.7 us, 128 x 128 12.6; 3308 x 2079 x 2808 95 against 61.
  kBf16Direct = 3,
  kF32Direct = 4,
  // Large tiles of fp32 rows that two parts do not hold (wide_tile): the plain fp32 instructions, 12608 x 2304 x 768 429 us if all
  // tiles are such, 146 in parts.
  kF32Wide = 5,
};

// A row's word: the exponent of what its parts are multiplied by, and its range (linear_split_kernel) in units of 1 / 1024.
__device__ __forceinline__ int word_exponent(uint32_t word) { return (int)(word << 22) >> 22; }
__device__ __forceinline__ uint32_t row_word(int exponent, uint32_t large, uint32_t lossy) {
  return ((uint32_t)exponent & 1023u) | large << 10 | lossy << 21;
}

__device__ __forceinline__ uint32_t widest_of(uint32_t a, uint32_t b) {    // of both halves
  typedef uint16_t u2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u2, a), __builtin_bit_cast(u2, b)));
}
// Words of ROWS rows, each lane's, of which `rows` exist (the last one repeats).
template <int ROWS>
struct RowRanges {
  uint32_t words[ROWS / 64];
  __device__ __forceinline__ RowRanges(const uint32_t* from, int rows) {
    static_assert(ROWS % 64 == 0, "rows");
#pragma unroll
    for (int i = 0; i < ROWS / 64; ++i) {
      const int r = (int)(threadIdx.x & 63) + 64 * i;
      words[i] = from[r < rows ? r : rows - 1];
    }
  }
  // The lane's widest: the largest 1024 - large above the largest lossy.
  __device__ __forceinline__ uint32_t widest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < ROWS / 64; ++i) m = widest_of(m, (1024u - (words[i] >> 10 & 2047u)) << 16 | words[i] >> 21);
    return m;
  }
};
// Whether the two fp16 parts of a tile's rows do not give its products as near the exact ones as fp32 does.  In scaled values: a lossy
// element is off by 2^-25 at most and meets less than 2^15, so that of the I columns those of x and w that are lossy (shares n) put
// 2^-10 n I into a sum.  Columns that are large in both rows, a share of large_x + large_w - 1 at least, make |x|.|w| at
// least 2^(5 + 7) I times that share: while n is no more than it, the sum is off by 2^-22 |x|.|w| at most.  All other elements are held
// to 2^-22 each.  Every wave looks at all rows, so that none waits for another.
// The words are asked for in front of the first stages and used behind them (12608 x 2304 x 768 143.6 -> 144.6 us with this; words
// waited for first, their rows one after another, 146).
template <int BM, int BN>
__device__ __forceinline__ bool wide_tile(const RowRanges<BM>& of_x, const RowRanges<BN>& of_w) {
  __builtin_amdgcn_sched_barrier(0);     // the words are waited for here, behind the first stages' loads
  // x's in the lower half of the wave, w's in the upper one
  const bool upper = (threadIdx.x & 32) != 0;
  const uint32_t x = of_x.widest(), w = of_w.widest();
  uint32_t m = widest_of(upper ? w : x, lane_xor<32>(upper ? x : w));
  m = widest_of(m, lane_xor<1>(m));
  m = widest_of(m, lane_xor<2>(m));
  m = widest_of(m, lane_xor<4>(m));
  m = widest_of(m, lane_xor<8>(m));
  m = widest_of(m, lane_xor<16>(m));
  const uint32_t mx = (uint32_t)__builtin_amdgcn_readlane((int)m, 0), mw = (uint32_t)__builtin_amdgcn_readlane((int)m, 32);
  const int shared = 1024 - (int)(mx >> 16) - (int)(mw >> 16), lossy = (int)(mx & 0xFFFFu) + (int)(mw & 0xFFFFu);
  return lossy > (shared > 0 ? shared : 0);
}

// acc = the products of nk stages from k_first on, of the tile at row m0 of x and n0 of w; all LDS reads and loads are over when it
// returns.  pitch: of x and w, `rows_x` and `rows_w` of whose rows the tile has.  go(): asked while the first loads are on their way, the
// same in all lanes; where it says no there are no products, and false is returned.
template <int BM, int BN, int WM, int WN, int MODE, class Go>
__device__ __forceinline__ bool tile_products(const uint8_t* x, const uint8_t* w, const int64_t pitch, const int64_t m0, const int n0,
                                              const int64_t rows_x, const int64_t rows_w, const int k_first, const int nk,
                                              uint8_t* const smem, v4f (&acc)[WM / 16][WN / 16], Go&& go) {
  constexpr bool SPLIT = MODE == kSplitRows, DIRECT = MODE == kBf16Direct || MODE == kF32Direct, AS_IS = MODE >= kBf16Ragged;
  constexpr int WAVES_M = BM / WM, WAVES = WAVES_M * (BN / WN);
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int XL = BM / 8 / WAVES, WL = BN / 8 / WAVES;   // loads of a wave and stage: 8 rows each
  static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "loads");
  constexpr int STAGE = (BM + BN) * kPiece;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // Sources of the wave's loads: row lane / 8 of 8, the chunk that belongs where the lane writes.
  const auto rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(x) + m0 * pitch, 0, (int)(rows_x * pitch), 0x00027000);
  const auto rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(w) + (int64_t)n0 * pitch, 0, (int)(rows_w * pitch), 0x00027000);
  int off_x[XL], off_w[WL];
  auto source = [&](int row, int64_t rows) {
    const int chunk = (lane & 7) ^ (row & 7);           // row & 7 is lane / 8
    const int r = row < rows ? row : (int)rows - 1;     // rows past the last repeat it and are not stored
    return r * (int)pitch + (AS_IS ? 0 : chunk * 16);
  };
#pragma unroll
  for (int i = 0; i < XL; ++i) off_x[i] = source((wave * XL + i) * 8 + (lane >> 3), rows_x);
#pragma unroll
  for (int i = 0; i < WL; ++i) off_w[i] = source((wave * WL + i) * 8 + (lane >> 3), rows_w);
  auto load_one = [&](int kt, auto ec) {
    constexpr int e = decltype(ec)::value;
    const int at = (k_first + (kt < nk ? kt : nk - 1)) * kPiece;    // past the end: a stage again, into a buffer that nobody reads
    uint8_t* const b = smem + (kt & (kStages - 1)) * STAGE;
    if constexpr (AS_IS) {
      // the chunk that reaches past the row's end, and those behind it, are the row's last 16 bytes
      const int in = at + ((lane & 7) ^ (lane >> 3)) * 16, last = (int)pitch - 16, from = in < last ? in : last;
      if constexpr (e < XL) load_to_lds(rx, b + (wave * XL + e) * 1024, off_x[e] + from, 0);
      else load_to_lds(rw, b + BM * kPiece + (wave * WL + e - XL) * 1024, off_w[e - XL] + from, 0);
    } else {
      if constexpr (e < XL) load_to_lds(rx, b + (wave * XL + e) * 1024, off_x[e], at);
      else load_to_lds(rw, b + BM * kPiece + (wave * WL + e - XL) * 1024, off_w[e - XL], at);
    }
  };
  auto load_stage = [&](int kt) { static_for<XL + WL>([&](auto e) { load_one(kt, e); }); };

  const int wm0 = wave % WAVES_M * WM, wn0 = wave / WAVES_M * WN;
  // A fragment: 16 rows, the lane's 16 bytes of row lane % 16.  The two of a row in a stage: bfloat16, the 32 elements of its first and
  // of its second half; fp32, the 32 high parts and the 32 low ones.
  int off_f[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int q = lane >> 4, chunk = SPLIT ? (q >> 1) * 4 + (q & 1) + 2 * h : 4 * h + q;
    off_f[h] = (lane & 15) * kPiece + 16 * (chunk ^ (lane & 7));
  }
  using std::integral_constant;
  auto fragment = [&](int kt, int h, int row) { return *(const v4i*)(smem + (kt & (kStages - 1)) * STAGE + off_f[h] + row * kPiece); };
  auto read_x = [&](int kt, int h, v4i(&f)[TM], auto ic) { f[decltype(ic)::value] = fragment(kt, h, wm0 + decltype(ic)::value * 16); };
  auto read_w = [&](int kt, int h, v4i(&f)[TN], auto jc) { f[decltype(jc)::value] = fragment(kt, h, BM + wn0 + decltype(jc)::value * 16); };
  auto multiply_one = [&](const v4i& w, const v4i& x, v4f& c) {
    if constexpr (SPLIT) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w), __builtin_bit_cast(v8h, x), c, 0, 0, 0);
    else if constexpr (MODE >= kF32Direct)
      static_for<4>([&](auto e) {
        constexpr int E = decltype(e)::value;
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(w[E]), __int_as_float(x[E]), c, 0, 0, 0);
      });
    else c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w), __builtin_bit_cast(v8bf, x), c, 0, 0, 0);
  };
  // Products of all tiles, token tile by token tile, with event(q) pinned in front of the q-th: the compiler would gather the LDS
  // reads in front of their use.
  constexpr int NM = TM * TN, NL = XL + WL;
  auto products = [&](const v4i(&w)[TN], v4i(&x)[TM], auto&& event) {
    __builtin_amdgcn_sched_barrier(0);
    static_for<NM>([&](auto q) {
      constexpr int i = decltype(q)::value / TN, j = decltype(q)::value % TN;
      event(q);
      multiply_one(w[j], x[i], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // A row's last chunk holds bytes of the chunk before it as well, and those behind it nothing else: in both operands they are zero.
  auto mask = [&](int kt, int h, v4i(&w)[TN], v4i(&x)[TM]) {
    if ((int64_t)(k_first + kt + 1) * kPiece <= pitch) return;     // the same in all lanes
    const int before = (k_first + kt) * kPiece + (4 * h + (lane >> 4)) * 16 - ((int)pitch - 16);   // bytes of the chunk that are not its own
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int cut = before - 4 * e;
      const uint32_t keep = cut >= 4 ? 0u : cut > 0 ? ~0u << (8 * cut) : ~0u;
#pragma unroll
      for (int j = 0; j < TN; ++j) w[j][e] &= keep;
#pragma unroll
      for (int i = 0; i < TM; ++i) x[i][e] &= keep;
    }
  };
  // This wave's loads have arrived and its LDS reads are done; then everybody's.
  auto meet = [&]() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Events: the e-th of a list of N in front of product FIRST + e * STEP ...
  auto at = [](auto q, auto first, auto step, auto n, auto&& f) {
    constexpr int d = decltype(q)::value - decltype(first)::value, S = decltype(step)::value;
    if constexpr (d >= 0 && d % S == 0 && d / S < decltype(n)::value) f(integral_constant<int, d / S>{});
  };
#define HOT_INT(V) integral_constant<int, (V)>{}
  load_stage(0);
  load_stage(1);
  if (!go()) {
    meet();      // nothing of this is on its way to LDS any more
    return false;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0, 0, 0, 0};
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(NL) : "memory");   // the first stage
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  v4i wa[TN], wb[TN], xa[TM];
  if constexpr (MODE != kF32Wide) {
    static_for<TN>([&](auto j) { read_w(0, 0, wa, j); });
    static_for<TM>([&](auto i) { read_x(0, 0, xa, i); });
  }
  if constexpr (MODE == kF32Wide) {     // a half of a stage at a time: the kernel's other path takes the registers
    auto nothing = [](auto) {};
    for (int kt = 0; kt < nk; ++kt) {
      static_for<2>([&](auto h) {
        static_for<TN>([&](auto j) { read_w(kt, decltype(h)::value, wa, j); });
        static_for<TM>([&](auto i) { read_x(kt, decltype(h)::value, xa, i); });
        mask(kt, decltype(h)::value, wa, xa);
        products(wa, xa, nothing);
      });
      meet();
      load_stage(kt + 2);
    }
  } else if constexpr (DIRECT) {
    v4i xb[TM];
    auto nothing = [](auto) {};
    for (int kt = 0; kt < nk; ++kt) {
      static_for<TN>([&](auto j) { read_w(kt, 1, wb, j); });
      static_for<TM>([&](auto i) { read_x(kt, 1, xb, i); });
      mask(kt, 0, wa, xa);
      products(wa, xa, nothing);
      meet();
      load_stage(kt + 2);
      static_for<TN>([&](auto j) { read_w(kt + 1, 0, wa, j); });
      static_for<TM>([&](auto i) { read_x(kt + 1, 0, xa, i); });
      mask(kt, 1, wb, xb);
      products(wb, xb, nothing);
    }
  } else if constexpr (!SPLIT) {
    const int scheduled = AS_IS ? nk - 1 : nk;
    for (int kt = 0; kt < scheduled; ++kt) {
      // a token tile's fragment is read anew once its products are issued
      products(wa, xa, [&](auto q) {
        at(q, HOT_INT(0), HOT_INT(NM / 2 / TN), HOT_INT(TN), [&](auto j) { read_w(kt, 1, wb, j); });
        at(q, HOT_INT(TN), HOT_INT(TN), HOT_INT(TM - 1), [&](auto i) { read_x(kt, 1, xa, i); });
      });
      read_x(kt, 1, xa, HOT_INT(TM - 1));
      // behind the last stage comes a repeated one, whose first half is read and not used
      products(wb, xa, [&](auto q) {
        if constexpr (decltype(q)::value == TN) meet();
        at(q, HOT_INT(TN), HOT_INT(TN > 4 ? 2 : 1), HOT_INT(TN), [&](auto j) { read_w(kt + 1, 0, wa, j); });
        at(q, HOT_INT(TN), HOT_INT(TN), HOT_INT(TM - 1), [&](auto i) { read_x(kt + 1, 0, xa, i); });
        at(q, HOT_INT(TN + 1), HOT_INT(TN > 4 ? 2 : 1), HOT_INT(NL), [&](auto e) { load_one(kt + 2, e); });
      });
      read_x(kt + 1, 0, xa, HOT_INT(TM - 1));
    }
    if constexpr (AS_IS) {     // the last stage, masked
      auto nothing = [](auto) {};
      static_for<TN>([&](auto j) { read_w(nk - 1, 1, wb, j); });
      mask(nk - 1, 0, wa, xa);
      products(wa, xa, nothing);
      static_for<TM>([&](auto i) { read_x(nk - 1, 1, xa, i); });
      mask(nk - 1, 1, wb, xa);
      products(wb, xa, nothing);
    }
  } else {
    v4i xb[TM];
    for (int kt = 0; kt < nk; ++kt) {
      products(wa, xa, [&](auto q) {
        at(q, HOT_INT(0), HOT_INT(1), HOT_INT(TM), [&](auto i) { read_x(kt, 1, xb, i); });
        at(q, HOT_INT(TM), HOT_INT(1), HOT_INT(TN), [&](auto j) { read_w(kt, 1, wb, j); });
      });
      meet();
      products(wa, xb, [&](auto q) { at(q, HOT_INT(0), HOT_INT(NM / NL), HOT_INT(NL), [&](auto e) { load_one(kt + 2, e); }); });
      products(wb, xa, [&](auto q) {
        at(q, HOT_INT(0), HOT_INT(NM / 2 / TN), HOT_INT(TN), [&](auto j) { read_w(kt + 1, 0, wa, j); });
        at(q, HOT_INT(TN), HOT_INT(TN), HOT_INT(TM - 1), [&](auto i) { read_x(kt + 1, 0, xa, i); });
      });
      read_x(kt + 1, 0, xa, HOT_INT(TM - 1));
    }
  }
#undef HOT_INT
  meet();
  return true;
}

// The same for plain fp32 rows of fewer than four columns, which are shorter than a load: from memory, element by element.
template <int BM, int BN, int WM, int WN>
__device__ __forceinline__ void tile_short_rows(const float* x, const float* w, int I, int64_t L, int O, int64_t m0, int n0,
                                                v4f (&acc)[WM / 16][WN / 16]) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int64_t row = m0 + wave % (BM / WM) * WM + (lane & 15);
  const int col = n0 + wave / (BM / WM) * WN + 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < WM / 16; ++i)
#pragma unroll
    for (int j = 0; j < WN / 16; ++j) acc[i][j] = v4f{0, 0, 0, 0};
#pragma unroll 1
  for (int k = 0; k < I; ++k) {
    float xs[WM / 16];
#pragma unroll
    for (int i = 0; i < WM / 16; ++i) xs[i] = x[(row + i * 16 < L ? row + i * 16 : L - 1) * I + k];
#pragma unroll
    for (int j = 0; j < WN / 16; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int c = col + j * 16 + r;
        const float ws = w[(uint32_t)((c < O ? c : O - 1) * I + k)];     // O < 2^24, I < 4
#pragma unroll
        for (int i = 0; i < WM / 16; ++i) acc[i][j][r] = fmaf(xs[i], ws, acc[i][j][r]);
      }
  }
}

template <int BM, int BN, int WM, int WN, int MODE, class TY>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN), 2) void linear_tile_kernel(const TileArgs g) {
  constexpr bool SPLIT = MODE == kSplitRows;
  constexpr int WAVES_M = BM / WM, WAVES = WAVES_M * (BN / WN);
  constexpr int TM = WM / 16, TN = WN / 16;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // A workgroup of a whole tile, or of a slice of one: slices of a tile are neighbours in dispatch order but for their XCD.
  const int rest = g.tiles_m * g.tiles_n - g.whole, part = (int)blockIdx.x - g.whole;
  const bool sliced = part >= 0;
  const int z = sliced ? part / rest : 0, tail = sliced ? part % rest : 0;
  int tm, tn;
  tile_at(sliced ? g.whole + tail : xcd_contiguous((int)blockIdx.x, g.whole), g.tiles_m, g.tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;
  const int stages = (int)((g.pitch + kPiece - 1) / kPiece);    // those of plain fp32 rows are as many as those of their parts
  const int k_first = sliced ? (int)((int64_t)stages * z / g.slices) : 0;
  const int nk = sliced ? (int)((int64_t)stages * (z + 1) / g.slices) - k_first : stages;
  const int64_t rows_x = g.out.L - m0 < BM ? g.out.L - m0 : BM, rows_w = g.out.O - n0 < BN ? g.out.O - n0 : BN;
  const int wm0 = wave % WAVES_M * WM, wn0 = wave / WAVES_M * WN;
  v4f acc[TM][TN];
  int scaled = 0;      // all bits: the sums are those of scaled rows
  const auto always = [] { return true; };
  if constexpr (SPLIT) {
    const RowRanges<BM> of_x(g.ex + m0, (int)rows_x);
    const RowRanges<BN> of_w(g.ew + n0, (int)rows_w);
    scaled = -(int)tile_products<BM, BN, WM, WN, kSplitRows>(g.x, g.w, g.pitch, m0, n0, rows_x, rows_w, k_first, nk, smem, acc,
                                                             [&] { return !wide_tile<BM, BN>(of_x, of_w); });
    if (!scaled) {
      if (g.plain_pitch >= 16)
        tile_products<BM, BN, WM, WN, kF32Wide>(g.x_plain, g.w_plain, g.plain_pitch, m0, n0, rows_x, rows_w, k_first, nk, smem, acc, always);
      else
        tile_short_rows<BM, BN, WM, WN>((const float*)g.x_plain, (const float*)g.w_plain, (int)g.plain_pitch / 4, g.out.L, g.out.O, m0, n0, acc);
    }
  } else {
    tile_products<BM, BN, WM, WN, MODE>(g.x, g.w, g.pitch, m0, n0, rows_x, rows_w, k_first, nk, smem, acc, always);
  }

  if (sliced) {
    if constexpr (SPLIT) {
      if (scaled) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          int ew[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int c = n0 + wn0 + j * 16 + 4 * (lane >> 4) + r;
            ew[r] = word_exponent(g.ew[c < g.out.O ? c : g.out.O - 1]);
          }
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            const int64_t row = m0 + wm0 + i * 16 + (lane & 15);
            const int ex = word_exponent(g.ex[row < g.out.L ? row : g.out.L - 1]);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = __builtin_ldexpf(acc[i][j][r], ex + ew[r]);
          }
        }
      }
    }
    // 16 bytes a lane and accumulator tile, as linear_combine_kernel reads them
    float* const image = g.images + ((int64_t)tail * g.slices + z) * (BM * BN) + tid * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) *(v4f*)(image + (i * TN + j) * (256 * WAVES)) = acc[i][j];
    return;
  }
  // CB columns of 64 / CH tokens at a time: as long runs of a row as the wave's columns divide into
  constexpr int PITCH = WN + 4, CB = WN % 128 == 0 ? 128 : WN % 64 == 0 ? 64 : 32, CH = CB / 8, RPI = 64 / CH;
  static_assert(WN % CB == 0, "column blocks");
  float* const strip = (float*)smem + wave * 32 * PITCH;
#pragma unroll
  for (int i = 0; i < TM / 2; ++i) {
    // accumulator register r of a 16 x 16 tile: output 4 (lane / 16) + r, token lane % 16
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < TN; ++j) *(v4f*)&strip[(h * 16 + (lane & 15)) * PITCH + j * 16 + 4 * (lane >> 4)] = acc[2 * i + h][j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int cb = 0; cb < WN; cb += CB) {
      const int c = n0 + wn0 + cb + lane % CH * 8, n = g.out.O - c;
      float bias[8];
      load_bias8(g.out, c, n, bias);
      int ew[8];
      if constexpr (SPLIT) {
#pragma unroll
        for (int e = 0; e < 8; ++e) ew[e] = word_exponent(g.ew[c + e < g.out.O ? c + e : g.out.O - 1]) & scaled;
      }
#pragma unroll 2
      for (int t0 = 0; t0 < 32; t0 += RPI) {
        const int t = t0 + lane / CH;
        const int64_t row = m0 + wm0 + i * 32 + t;
        const float* const p = &strip[t * PITCH + cb + lane % CH * 8];
        const v4f lo = *(const v4f*)p, hi = *(const v4f*)(p + 4);
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = lo[e];
          v[e + 4] = hi[e];
        }
        if (row < g.out.L) {
          if constexpr (SPLIT) {
            const int ex = word_exponent(g.ex[row]) & scaled;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __builtin_ldexpf(v[e], ex + ew[e]);
          }
          linear_finish8<TY>(g.out, row, c, n, bias, v);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The sums of a tile's slices, in slice order, and the epilogue.  A thread takes eight outputs of a token: those of lanes l + 32 h and
// l + 32 h + 16 of a 16 x 16 accumulator tile; four threads its 32 outputs.  Bound by the images' way through the caches.
template <int BM, int BN, int WM, int WN, class TY>
__global__ __launch_bounds__(256) void linear_combine_kernel(const TileArgs g) {
  constexpr int WAVES_M = BM / WM, WAVES = WAVES_M * (BN / WN), TN = WN / 16;
  constexpr int PER_TILE = BM * BN / 2048;    // workgroups of a tile
  const int tail = (int)blockIdx.x / PER_TILE;
  const int sub = (int)blockIdx.x % PER_TILE * 4 + ((int)threadIdx.x >> 6);      // 16 tokens x 32 outputs: wave fastest
  const int q = (int)threadIdx.x & 3, l = ((int)threadIdx.x >> 2) & 15;
  const int wave = sub % WAVES, i = sub / WAVES / (TN / 2), j = sub / WAVES % (TN / 2) * 2 + (q >> 1), h = q & 1;
  int tm, tn;
  tile_at(g.whole + tail, g.tiles_m, g.tiles_n, tm, tn);
  const float* const image = g.images + (int64_t)tail * g.slices * (BM * BN) + (i * TN + j) * (256 * WAVES) + (wave * 64 + h * 32 + l) * 4;
  float v[8] = {};
#pragma unroll 4
  for (int z = 0; z < g.slices; ++z) {
    const float* const p = image + (int64_t)z * (BM * BN);
    const v4f lo = *(const v4f*)p, hi = *(const v4f*)(p + 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] += lo[e];
      v[e + 4] += hi[e];
    }
  }
  const int64_t row = (int64_t)tm * BM + wave % WAVES_M * WM + i * 16 + l;
  const int c = tn * BN + wave / WAVES_M * WN + j * 16 + 8 * h, n = g.out.O - c;
  if (row >= g.out.L) return;
  float bias[8];
  load_bias8(g.out, c, n, bias);
  linear_finish8<TY>(g.out, row, c, n, bias, v);
}

// Operand rows of the fp32 product: row r of the L + O rows of x and w, scaled by 2^(14 - e), e the exponent of its largest value,
// as [16 high | 16 low] pieces; words[r]: e - 14 and the row's range, the share of its columns that are large (a scaled value of 2^5 or
// more in x, 2^7 in w, of at most 2^15), rounded down, and of those whose parts are off by more than 2^-22 of the value, rounded up; a row
// of zeros is held exactly, one with an infinity or a NaN not at all.  Padded columns are zero.  Bound by HBM: a row stays in the
// registers of the T lanes that work on it, NV times eight columns each, or (NV = 0: rows beyond 16384) is read a second time, from the
// caches.  8192 + 8192 rows of 8192 columns 177 us, 6.1 TB/s read and written; 250 when such rows were read twice.
__device__ __forceinline__ int row_exponent(uint32_t top) {   // of the largest magnitude's bits; subnormal ones too
  // infinities and NaNs stay what they are under any scale
  return top >= 0x7F800000u || top == 0 ? 0 : ilogbf(__uint_as_float(top));
}
// Called by all lanes of a wave; large, lossy: the wave's counts.
__device__ __forceinline__ void store_parts(uint8_t* dst, int64_t c, bool store, const float (&v)[8], int e, float large_from, int& large,
                                            int& lossy) {
  v8h hi, lo;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = __builtin_ldexpf(v[i], 14 - e);
    hi[i] = (_Float16)s;
    const float rest = s - (float)hi[i];
    lo[i] = (_Float16)rest;
    large += __popcll(__builtin_amdgcn_ballot_w64(fabsf(s) >= large_from));
    lossy += __popcll(__builtin_amdgcn_ballot_w64(fabsf(rest - (float)lo[i]) > 0x1p-22f * fabsf(s)));
    if (e > 15) lossy += __popcll(__builtin_amdgcn_ballot_w64(s == 0.0f && v[i] != 0.0f));   // below the smallest number when scaled
  }
  if (!store) return;
  uint8_t* const p = dst + (c >> 4) * 64 + (c & 8) * 2;
  *(v8h*)p = hi;
  *(v8h*)(p + 32) = lo;
}
template <int T, int NV>
__global__ __launch_bounds__(256) void linear_split_kernel(const float* x, const float* w, int64_t L, int64_t O, int64_t I, int64_t pitch,
                                                           uint8_t* px, uint8_t* pw, uint32_t* words, int64_t first) {
  __shared__ uint32_t s_top[4];
  __shared__ int s_large[4], s_lossy[4];
  const int lane = (int)threadIdx.x % T;
  const int64_t r = first + (int64_t)blockIdx.x * (256 / T) + (int)threadIdx.x / T;
  if (r >= L + O) return;    // T = 256: one row a workgroup
  const float* const src = r < L ? x + r * I : w + (r - L) * I;
  uint8_t* const dst = r < L ? px + r * pitch : pw + (r - L) * pitch;
  const int64_t padded = pitch / 4;
  auto have = [&](int64_t c) { return (int)(I - c < 0 ? 0 : I - c < 8 ? I - c : 8); };
  uint32_t top = 0;
  Raw8<float> raw[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (lane + j * T) * 8;
      raw[j] = load8(src + c, have(c));
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[8];
      widen(raw[j], v);
      top = max(top, magnitude8(v));
    }
  } else {
#pragma unroll 4
    for (int64_t c = lane * 8; c < I; c += T * 8) {
      float v[8];
      load_values(src + c, have(c), v);
      top = max(top, magnitude8(v));
    }
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if constexpr (T > 64) {
    if (((int)threadIdx.x & 63) == 0) s_top[(int)threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3]));
  }
  const int e = __builtin_amdgcn_readfirstlane(row_exponent(top));    // a wave is on one row
  const float large_from = r < L ? 0x1p5f : 0x1p7f;
  int large = 0, lossy = 0;
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (lane + j * T) * 8;
      float v[8];
      widen(raw[j], v);
      store_parts(dst, c, c < padded, v, e, large_from, large, lossy);
    }
  } else {
#pragma unroll 2
    for (int64_t c0 = 0; c0 < padded; c0 += T * 8) {
      const int64_t c = c0 + lane * 8;
      float v[8];
      load_values(src + c, have(c), v);
      store_parts(dst, c, c < padded, v, e, large_from, large, lossy);
    }
  }
  if constexpr (T > 64) {
    if (((int)threadIdx.x & 63) == 0) {
      s_large[(int)threadIdx.x >> 6] = large;
      s_lossy[(int)threadIdx.x >> 6] = lossy;
    }
    __syncthreads();
    large = s_large[0] + s_large[1] + s_large[2] + s_large[3];
    lossy = s_lossy[0] + s_lossy[1] + s_lossy[2] + s_lossy[3];
  }
  if (lane == 0) {
    // shares of 1 / 1024, rounded down and up: the quotient is off by 2^-21 of itself at most
    const float unit = 1024.0f * __builtin_amdgcn_rcpf((float)I);
    const uint32_t some = (uint32_t)((float)large * unit * (1.0f - 0x1p-20f));
    const uint32_t off = min(1024u, (uint32_t)ceilf((float)lossy * unit * (1.0f + 0x1p-20f)));
    words[r] = top >= 0x7F800000u ? row_word(0, 0, 1024) : top == 0 ? row_word(0, 1024, 0) : row_word(e - 14, some, off);
  }
}

// f(first, rows) for the runs of rows, `lanes` lanes each, that a launch holds.
template <class F>
hipError_t each_run(int64_t rows, int64_t lanes, F&& f) {
  const int64_t run = kMaxLaunch / lanes;
  for (int64_t first = 0; first < rows; first += run)
    if (const hipError_t e = f(first, rows - first < run ? rows - first : run); e != hipSuccess) return e;
  return hipSuccess;
}

hipError_t launch_split(const float* x, const float* w, int64_t L, int64_t O, int64_t I, int64_t pitch, uint8_t* px, uint8_t* pw,
                        uint32_t* words, hipStream_t s) {
  auto go = [&](auto t, auto nv) {
    constexpr int T = decltype(t)::value;
    return each_run(L + O, T, [&](int64_t first, int64_t rows) {
      linear_split_kernel<T, decltype(nv)::value><<<dim3((unsigned)ceil_div(rows, 256 / T)), dim3(256), 0, s>>>(x, w, L, O, I, pitch, px, pw,
                                                                                                              words, first);
      return hipGetLastError();
    });
  };
  using std::integral_constant;
  if (I <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (I <= 1024) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (I <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (I <= 4096) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (I <= 8192) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (I <= 16384) return go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  return go(integral_constant<int, 256>{}, integral_constant<int, 0>{});
}

// Rows of bfloat16 operands of an odd width, padded with zeros to a multiple of 64.  Bound by HBM.
__global__ __launch_bounds__(256) void linear_pad_kernel(const bf16* x, const bf16* w, int64_t L, int64_t O, int64_t I, int64_t pitch,
                                                         uint8_t* px, uint8_t* pw, int64_t first) {
  const int lane = (int)threadIdx.x & 63;
  const int64_t r = first + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= L + O) return;
  const bf16* const src = r < L ? x + r * I : w + (r - L) * I;
  uint8_t* const dst = r < L ? px + r * pitch : pw + (r - L) * pitch;
#pragma unroll 4
  for (int64_t c = lane * 8; c < pitch / 2; c += 512) {
    const int64_t n = I - c;
    const Raw8<bf16> v = load8(src + c, (int)(n < 0 ? 0 : n < 8 ? n : 8));
    *(h8_any*)(dst + c * 2) = v.a;
  }
}

// What the large tiles need besides their operands: fp32 rows in parts with their words; bfloat16 rows of an odd width, or shorter than
// 16 bytes, padded: rows that begin at odd multiples of two bytes are loaded at half the rate.
struct TileLayout {
  int64_t pitch;
  bool packed;
  size_t w, words, total;    // x's rows come first
};
TileLayout tile_layout(hot_type type, int64_t L, int64_t O, int64_t I) {
  TileLayout t;
  t.packed = type == HOT_F32 || I % 2 != 0 || I < 8;
  t.pitch = type == HOT_F32 ? round_up(I, 32) * 4 : t.packed ? round_up(I, 64) * 2 : I * 2;
  t.w = t.packed ? (size_t)round_up(L * t.pitch, 256) : 0;
  t.words = t.w + (t.packed ? (size_t)round_up(O * t.pitch, 256) : 0);
  t.total = t.words + (type == HOT_F32 ? (size_t)(L + O) * 4 : 0);
  return t;
}

// How a product is worked on.
struct Plan {
  bool tiles;          // else linear_rows_kernel
  bool direct;         // small tiles of x and w as they are
  int bm, bn;          // tile: 256 x 256, one workgroup a compute unit, 128 x 128, two, or, direct, 64 x 64 or 32 x 128
  int64_t tiles_m, tiles_n;
  int64_t whole;       // tiles with a workgroup each; the rest in `slices` slices of K
  int slices;
  int nt, mt;          // linear_rows_kernel: 16 nt outputs and 16 mt tokens a workgroup
};

// Times in microseconds of the ways to do a product, for the choice between them.  The constants are a fit to launches of all
// kernels over random shapes (1 to 60000 rows, widths of 64 to 11008, both types, every split below); over 597 others the way they
// choose takes 1.03 times the fastest one's time on average, 1.41 times at worst (profiles/linear_plan_shapes.txt), and 0.3 us of the
// host's.  A second launch costs the caller's thread as well.
constexpr double kLaunch = 2.5;
// Two resources used beside each other: little more than the longer time.
double beside(double a, double b) { return sqrt(sqrt(a * a * a * a + b * b * b * b)); }

// Workgroups that the busiest compute unit has; for many of them, as they come and go, half a workgroup more than the mean.
double rounds_of(int64_t n) { return n <= 1024 ? (double)ceil_div(n, 256) : n / 256.0 + 0.5; }

// Tiles: a stage of 128 bytes of K in a round of workgroups, what a round takes besides (filling the buffers, the epilogue), the
// outputs, the images' way to memory and back.  256 x 256 moves half as much through LDS for each product, 128 x 128 fills the chip
// with a quarter of the outputs: 3550 x 4380 x 5888 bfloat16 150 us against 214, 18 x 9042 x 1024 26 us against 14.
// Slices of the tiles that leave compute units idle: 81 x 9536 x 320 bfloat16 88 -> 16 us, 1767 x 321 x 1728 fp32 26 us whole, 33 in slices.
double tile_time(int size, hot_type type, int64_t L, int64_t O, int64_t pitch, Plan* p) {
  const bool big = size == 256, f32 = type == HOT_F32;
  const int64_t stages = ceil_div(pitch, kPiece);
  const int64_t slots = big ? 256 : 512;
  *p = Plan{};
  p->tiles = true;
  p->bm = p->bn = size;
  p->tiles_m = ceil_div(L, size);
  p->tiles_n = ceil_div(O, size);
  const int64_t count = p->tiles_m * p->tiles_n, rest = count % slots;
  p->whole = count;
  p->slices = 1;
  const double loads = pitch % kPiece ? 1.1 : 1.0;      // rows that begin anywhere (8000 x 4000 x 4000 bfloat16 229 us, x 4032 209)
  const double full = loads * (big ? (f32 ? 1.37 : 1.06) : (f32 ? 1.23 : 0.96));    // a stage with every slot taken
  const double half = big ? full : loads * (f32 ? 0.54 : 0.50);                     // 128 x 128, one workgroup a compute unit
  const double round = big ? (f32 ? 11.7 : 8.9) : (f32 ? 4.1 : 3.1);
  double t = (count / slots) * (stages * full + round);
  if (rest) {
    int64_t most = slots / rest;                            // slices that still fill one round,
    most = most < stages / 4 ? most : stages / 4;           // of four stages at least
    most = most < 16 ? most : 16;
    double best = 1e30;
    for (int64_t k = 1; k <= (most > 1 ? most : 1); ++k) {
      const int64_t n = rest * k;
      const double stage = big || n <= 256 ? half : half + (full - half) * (double)(n - 256) / 256;
      const double e = ceil_div(stages, k) * stage + round + (k > 1 ? kLaunch + (double)n * size * size * 8 / (big ? 6.9e6 : 4.6e6) : 0.0);
      if (e < best) {
        best = e;
        p->slices = (int)k;
        p->whole = k > 1 ? count - rest : count;
      }
    }
    t += best;
  }
  return (big ? 2.4 : 4.5) + t + (double)L * O / 3e6;
}

// linear_rows_kernel: a compute unit's matrix instructions and loads, both in units of 2000 cycles' worth a microsecond and for as many
// rounds of workgroups as there are, beside the operands' way from HBM.  Rows of an odd number of bfloat16 elements are not
// 4-byte aligned, which costs their loads three times the time.
double rows_time(hot_type type, int64_t L, int64_t O, int64_t I, Plan* p) {
  const bool f32 = type == HOT_F32;
  const double hbm = ((double)O * I + (double)L * I) * (f32 ? 4 : 2) / 9e6 + (double)L * O * 4 / 9e6;
  const int64_t turn = kWaves * kSteps * (f32 ? 16 : 32);    // elements of K a workgroup has on their way
  const double odd = !f32 && I % 2 ? 3.0 : 1.0;
  double best = 1e30;
  for (int nt = 1; nt <= 2; ++nt)
    for (int mt = 1; mt <= 4; mt *= 2) {
      if (mt > 1 && (mt / 2) * 16 >= L) continue;
      const int64_t tm = ceil_div(L, 16 * mt), tn = ceil_div(O, 16 * nt);
      if (tm * tn > kMaxLaunch / (64 * kWaves)) continue;
      for (int s = 1; s <= 16; ++s) {
        if (s > 1 && (tm * tn * s > 512 || I / s < turn)) break;
        const double k = (double)I / s * odd / 2000;
        const double cu = rounds_of(tm * tn * s) * (f32 ? k * (1.82 * nt * mt + 1.94 * (nt + mt)) + 0.38 * nt * mt
                                        : k * (0.253 * nt * mt + 1.23 * (nt + mt)) + 0.265 * nt * mt);
        const double t = (f32 ? 5.2 + sqrt(cu * cu + hbm * hbm) : 5.7 + beside(cu, hbm)) + (s > 1 ? kLaunch + 2.3 + (double)s * L * O * 8 / 4e6 : 0.0);
        if (t < best) {
          best = t;
          *p = Plan{};
          p->tiles_m = tm;
          p->tiles_n = tn;
          p->slices = s;
          p->nt = nt;
          p->mt = mt;
        }
      }
    }
  return best;
}

// Small tiles of the operands as they are: a compute unit's matrix instructions and loads, the time of a workgroup by itself.  32 x 128
// reads less of a wide weight twice where tokens are few (10 x 9408 x 4352 fp32 37 us, 58 with 64 x 64), 64 x 64 less in all
// (48 x 8704 x 9152 bfloat16 34 us, 53 with 32 x 128).  K in slices: 729 x 64 x 10240 bfloat16 69 -> 17 us; 1872 x 624 x 640 9.7 us
// whole, 17.2 in slices.
double direct_time(int bm, int bn, hot_type type, int64_t L, int64_t O, int64_t I, Plan* p) {
  const bool f32 = type == HOT_F32;
  const int64_t bytes = I * (f32 ? 4 : 2), stages = ceil_div(bytes, kPiece);
  *p = Plan{};
  p->tiles = p->direct = true;
  p->bm = bm;
  p->bn = bn;
  p->tiles_m = ceil_div(L, bm);
  p->tiles_n = ceil_div(O, bn);
  p->slices = 1;
  const int64_t count = p->tiles_m * p->tiles_n;
  if (count > kMaxLaunch / 256) return 1e30;
  p->whole = count;
  // loads that begin at odd multiples of two bytes: the stages' share, a workgroup's by itself, what is moved (fitted apart)
  const bool unaligned = !f32 && I % 2;
  const double odd = !unaligned ? 1.0 : bm == 64 ? 2.2 : 2.8, alone = unaligned ? 1.6 : 1.0, bytes_odd = unaligned ? 2.0 : 1.0;
  const double moved = bytes_odd * (((double)L + O) * bytes + (double)L * O * 4) / (f32 ? 49e6 : 15e6);
  double best = 1e30;
  for (int64_t k = 1; k <= 16; ++k) {
    if (k > 1 && (count * k > 1024 || stages / k < 4)) break;
    const int64_t n = count * k, each = ceil_div(stages, k);
    const double cu = rounds_of(n) * (f32 ? each * 0.484 + 0.90 : each * odd * 0.149 + 0.39), one = each * (f32 ? 0.461 : alone * 0.235);
    const double t = 5.3 + beside(cu, one) + moved + (k > 1 ? kLaunch + 3.0 + (double)n * bm * bn * 8 / 5.5e6 : 0.0);
    if (t < best) {
      best = t;
      p->slices = (int)k;
      p->whole = k > 1 ? 0 : count;
    }
  }
  return best;
}

Plan make_plan(hot_type type, int64_t L, int64_t O, int64_t I) {
  const TileLayout lay = tile_layout(type, L, O, I);
  const bool f32 = type == HOT_F32;
  Plan rows{}, a{}, b{}, c{}, d{};
  const double tr = rows_time(type, L, O, I, &rows);
  if (lay.pitch * 256 >= (1ll << 31)) return rows;     // a tile's rows must be within the reach of a buffer descriptor
  const double operands = lay.packed ? kLaunch + 2.5 + (double)(L + O) * I * (f32 ? 8 : 4) / 5.2e6 : 0.0;
  const double ta = operands + tile_time(128, type, L, O, lay.pitch, &a), tb = operands + tile_time(256, type, L, O, lay.pitch, &b);
  const bool direct = I * (f32 ? 4 : 2) >= 16;     // a load is 16 bytes
  const double tc = direct ? direct_time(64, 64, type, L, O, I, &c) : 1e30, td = direct ? direct_time(32, 128, type, L, O, I, &d) : 1e30;
  const Plan* p = &rows;
  double t = tr;
  if (ta < t) { t = ta; p = &a; }
  if (tb < t) { t = tb; p = &b; }
  if (tc < t) { t = tc; p = &c; }
  if (td < t) { t = td; p = &d; }
  return *p;
}

size_t images_offset(const Plan& p, const TileLayout& t) { return p.direct ? 0 : (size_t)round_up((int64_t)t.total, 256); }
size_t scratch_bytes(const Plan& p, const TileLayout& t, int64_t L, int64_t O) {
  if (!p.tiles) return p.slices > 1 ? (size_t)p.slices * L * sums_pitch(O) * 4 : 0;
  const size_t images = p.slices > 1 ? (size_t)((p.tiles_m * p.tiles_n - p.whole) * p.slices) * p.bm * p.bn * 4 : 0;
  return images ? images_offset(p, t) + images : p.direct ? 0 : t.total;
}

template <int BM, int BN, int WM, int WN, int MODE, class TY>
hipError_t tiles_sized(const TileArgs& g, hipStream_t s) {
  constexpr int LDS = kTileLds<BM, BN, WM, WN>, THREADS = 64 * (BM / WM) * (BN / WN);
  auto kern = linear_tile_kernel<BM, BN, WM, WN, MODE, TY>;
  static std::atomic<uint64_t> raised{0};
  if (const hipError_t e = raise_lds_limit((const void*)kern, LDS, raised); e != hipSuccess) return e;
  const int64_t rest = (int64_t)g.tiles_m * g.tiles_n - g.whole;
  kern<<<dim3((unsigned)(g.whole + rest * g.slices)), dim3(THREADS), LDS, s>>>(g);
  if (rest) linear_combine_kernel<BM, BN, WM, WN, TY><<<dim3((unsigned)(rest * (BM * BN / 2048))), dim3(256), 0, s>>>(g);
  return hipGetLastError();
}

template <class T, class TY>
hipError_t tiles_typed(const LinearForward& a, const Plan& p, const LinearOut& o, hipStream_t s) {
  constexpr bool F32 = sizeof(T) == 4;
  const TileLayout t = tile_layout(a.type, a.L, a.O, a.I);
  TileArgs g{(const uint8_t*)a.x, (const uint8_t*)a.w, t.pitch, (const uint8_t*)a.x, (const uint8_t*)a.w, a.I * (int64_t)sizeof(T), nullptr, nullptr,
             (int)p.tiles_m, (int)p.tiles_n,
             (int)p.whole, p.slices, nullptr, o};
  if (p.slices > 1) g.images = (float*)((uint8_t*)a.ws + images_offset(p, t));
  if (p.direct) {
    g.pitch = a.I * (int64_t)sizeof(T);
    constexpr int MODE = F32 ? kF32Direct : kBf16Direct;
    stage_begin(kStLinear, s);
    const hipError_t e = p.bm == 64 ? tiles_sized<64, 64, 32, 32, MODE, TY>(g, s) : tiles_sized<32, 128, 32, 32, MODE, TY>(g, s);
    stage_end(kStLinear, s);
    return e;
  }
  if (t.packed) {
    uint8_t* const px = (uint8_t*)a.ws;
    uint8_t* const pw = px + t.w;
    uint32_t* const words = (uint32_t*)(px + t.words);
    stage_begin(kStLinearOperands, s);
    hipError_t e;
    if constexpr (F32) {
      e = launch_split((const float*)a.x, (const float*)a.w, a.L, a.O, a.I, t.pitch, px, pw, words, s);
    } else {
      e = each_run(a.L + a.O, 64, [&](int64_t first, int64_t rows) {
        linear_pad_kernel<<<dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, s>>>((const bf16*)a.x, (const bf16*)a.w, a.L, a.O, a.I, t.pitch,
                                                                                 px, pw, first);
        return hipGetLastError();
      });
    }
    stage_end(kStLinearOperands, s);
    if (e != hipSuccess) return e;
    g.x = px;
    g.w = pw;
    g.ex = words;
    g.ew = words + a.L;
  }
  auto go = [&](auto mode) {
    constexpr int MODE = decltype(mode)::value;
    stage_begin(kStLinear, s);
    const hipError_t e = p.bm == 256 ? tiles_sized<256, 256, 64, 128, MODE, TY>(g, s) : tiles_sized<128, 128, 64, 64, MODE, TY>(g, s);
    stage_end(kStLinear, s);
    return e;
  };
  if constexpr (F32) return go(std::integral_constant<int, kSplitRows>{});
  else if (t.pitch % kPiece == 0) return go(std::integral_constant<int, kBf16Rows>{});
  else return go(std::integral_constant<int, kBf16Ragged>{});
}

template <class T, class TY>
hipError_t rows_typed(const LinearForward& a, const Plan& p, const LinearOut& o, hipStream_t s) {
  auto go = [&](auto nt, auto mt) {
    constexpr int NT = decltype(nt)::value, MT = decltype(mt)::value;
    float* const sums = p.slices > 1 ? (float*)a.ws : nullptr;
    linear_rows_kernel<T, TY, NT, MT><<<dim3((unsigned)(p.tiles_m * p.tiles_n * p.slices)), dim3(64 * kWaves), 0, s>>>(
        (const T*)a.x, (const T*)a.w, a.I, (int)p.tiles_m, p.slices, sums, o);
    if (sums) {
      const int chunks = (int)(o.k.codes ? o.k.pitch / 8 : sums_pitch(a.O) / 8);    // a checkpoint's groups are whole
      linear_rows_combine_kernel<TY><<<dim3((unsigned)ceil_div(a.L * chunks, 256)), dim3(256), 0, s>>>(sums, p.slices, chunks, o);
    }
    return hipGetLastError();
  };
  using std::integral_constant;
  auto with_nt = [&](auto mt) {
    if (p.nt == 1) return go(integral_constant<int, 1>{}, mt);
    return go(integral_constant<int, 2>{}, mt);
  };
  if (p.mt == 1) return with_nt(integral_constant<int, 1>{});
  if (p.mt == 2) return with_nt(integral_constant<int, 2>{});
  return with_nt(integral_constant<int, 4>{});
}

Plan run_plan(hot_type type, int64_t L, int64_t O, int64_t I, bool kept) {
  Plan p = make_plan(type, L, O, I);
  if (kept && !p.tiles && p.slices == 1 && p.nt == 1) {   // a group is finished by one workgroup
    p.nt = 2;
    p.tiles_n = ceil_div(O, 32);
  }
  return p;
}

template <class T, class TY>
hipError_t linear_run(const LinearForward& a, const CkptView& k, hipStream_t s) {
  LinearOut o{a.bias, a.residual, a.y, k, a.L, (int)a.O, a.fn, stream_output(a.L, a.O * (int64_t)sizeof(TY))};
  const Plan p = run_plan(a.type, a.L, a.O, a.I, k.codes != nullptr);
  if (p.tiles) return tiles_typed<T, TY>(a, p, o, s);
  stage_begin(kStLinear, s);
  const hipError_t e = rows_typed<T, TY>(a, p, o, s);
  stage_end(kStLinear, s);
  return e;
}

// Rows of one plan: a longer x is worked on in runs, one after another on the same scratch, which bounds that and every launch.
constexpr int64_t kRunRows = 1 << 23;

template <class T, class TY>
hipError_t linear_typed(const LinearForward& a, hipStream_t s) {
  const CkptLayout l = ckpt_layout(a.L, a.O);
  for (int64_t first = 0; first < a.L; first += kRunRows) {
    LinearForward r = a;
    r.L = a.L - first < kRunRows ? a.L - first : kRunRows;
    r.x = (const T*)a.x + first * a.I;
    r.y = (TY*)a.y + first * a.O;
    if (a.residual) r.residual = (const TY*)a.residual + first * a.O;
    CkptView k{};
    if (a.ckpt) k = CkptView{(uint8_t*)a.ckpt + first * l.pitch, (uint8_t*)a.ckpt + l.exps + first * (l.pitch / kCkGroup), l.pitch};
    if (const hipError_t e = linear_run<T, TY>(r, k, s); e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t run_scratch_bytes(hot_type type, int64_t L, int64_t O, int64_t I) {
  return L ? scratch_bytes(make_plan(type, L, O, I), tile_layout(type, L, O, I), L, O) : 0;
}

}  // namespace

size_t linear_scratch_bytes(hot_type type, int64_t L, int64_t O, int64_t I) {
  if (L <= kRunRows) return run_scratch_bytes(type, L, O, I);
  const size_t run = run_scratch_bytes(type, kRunRows, O, I), last = run_scratch_bytes(type, L % kRunRows, O, I);
  return run > last ? run : last;
}

void describe_linear(hot_type type, hot_type y_type, int64_t L, int64_t O, int64_t I, bool kept, hot_linear_plan* out) {
  if (L > kRunRows) L = kRunRows;
  const Plan p = run_plan(type, L, O, I, kept);
  const TileLayout t = tile_layout(type, L, O, I);
  const int64_t bytes = I * (type == HOT_F32 ? 4 : 2), count = p.tiles_m * p.tiles_n;
  out->way = !p.tiles ? HOT_LINEAR_ROWS : p.direct ? HOT_LINEAR_DIRECT : t.packed ? HOT_LINEAR_PACKED : HOT_LINEAR_TILES;
  out->tile_rows = p.tiles ? p.bm : 16 * p.mt;
  out->tile_cols = p.tiles ? p.bn : 16 * p.nt;
  out->tiles = (int32_t)count;
  out->whole = (int32_t)(p.tiles ? p.whole : p.slices > 1 ? 0 : count);
  out->slices = p.slices;
  out->masked = (out->way == HOT_LINEAR_DIRECT || out->way == HOT_LINEAR_TILES) && bytes % kPiece != 0;
  out->streams = stream_output(L, O * (y_type == HOT_F32 ? 4 : 2));
}

hipError_t launch_linear(const LinearForward& a, hipStream_t s) {
  if (a.type == HOT_F32) return linear_typed<float, float>(a, s);
  if (a.y_type == HOT_F32) return linear_typed<bf16, float>(a, s);
  return linear_typed<bf16, bf16>(a, s);
}

}  // namespace hot
