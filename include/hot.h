/*
 * hot.h - C ABI of the MI355X (gfx950) implementation of the HOT linear-layer
 * backward pass (arxiv 2503.21261, "HOT: Hadamard-based Optimized Training").
 *
 * Notation (Sec. 4.1, Eq. 7-8): x [L x I] input activation, w [O x I] weight,
 * y = x.w^T [L x O], g_y [L x O] output gradient,
 *     g_x = g_y . w   [L x I]      g_w = g_y^T . x   [O x I].
 * L is the flattened token index (batch x sequence), tiled consecutively in
 * blocks of n for the token-direction transform.
 *
 * Conventions for every call
 *   - All tensor pointers are DEVICE pointers to row-major, contiguous buffers,
 *     16-byte aligned, fp32 unless stated.  Pointers marked "host" are host
 *     memory.  The caller owns every buffer; the library never allocates, frees
 *     or keeps device memory between calls.
 *   - `ws` is caller-provided device scratch of at least hot_workspace_bytes()
 *     bytes, 256-byte aligned (checked: HOT_ERR_ARG otherwise).  Its first
 *     HOT_WS_PREFIX_BYTES hold scalars, exchange slots and flags; the packed
 *     operands of the call follow, and the hot_debug_* calls decode them.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Calls enqueue work and return without synchronising, except
 *     hot_select_quantizer, which waits for its own result.
 *   - Errors are return codes; arguments are checked on the host before any
 *     launch, so a failing call has launched nothing.  Inputs must be finite.
 *   - Two calls that share a workspace or an output must be ordered by the
 *     caller (same stream, or events).
 *   - HIP graphs: the kernels whose workgroups exchange values through the
 *     workspace (single-pass transforms, split-K GEMM) tell a launch's values
 *     from stale ones by a tag.  By default the host chooses it per call, and a
 *     replayed graph would repeat it: such calls must not be recorded.  With
 *     hot_config.replayable set, every call first advances a 64-bit epoch in the
 *     workspace (one more one-thread kernel) and the kernels derive their tags
 *     from it on the device, so that the call may be recorded and replayed (with
 *     the buffers it was recorded with; call it once with the same shapes before
 *     recording: launch plans are made on first use).  hot_select_quantizer waits
 *     for its result and cannot be recorded either way.
 */
#ifndef HOT_H
#define HOT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HOT_OK = 0,
  HOT_ERR_ARG = 1,        /* null pointer, bad enum, bad config field            */
  HOT_ERR_SHAPE = 2,      /* a size the method or the int32 accumulators forbid  */
  HOT_ERR_WORKSPACE = 3,  /* ws_bytes smaller than hot_workspace_bytes()         */
  HOT_ERR_DEVICE = 4,     /* a HIP runtime call failed                           */
  HOT_ERR_UNIMPLEMENTED = 5,
  HOT_ERR_SCRATCH_LIMIT = 6 /* hot_linear_backward_gx_noalloc: the shape needs more than
                               HOT_NOALLOC_SCRATCH_BYTES of scratch                      */
} hot_status;

/* Sec. 5.2.2: granularity of the scale of the rotated g_y. */
typedef enum { HOT_Q_PER_TENSOR = 0, HOT_Q_PER_TOKEN = 1 } hot_quantizer;

/* Sec. 5.1: the paper's quantiser rounds pseudo-stochastically; nearest-even is
 * offered so the half-step round-trip bound can be checked. */
typedef enum {
  HOT_ROUND_NEAREST_EVEN = 0,
  HOT_ROUND_PSEUDO_STOCHASTIC = 1,
  HOT_ROUND_DRAWN = 3      /* 8-bit moments of hot_adamw_step alone (below)                        */
} hot_rounding;

typedef struct {
  int32_t block;           /* n: WHT tile, 16 (paper, Supp. D) | 32 | 64                */
  int32_t keep;            /* r: rows of each n-block kept by HLA on the g_w path,
                              1..n (paper: 8 of 16, Supp. B)                          */
  const int32_t* keep_idx; /* host, r distinct natural-order row indices in [0,n), or
                              NULL = the r rows of lowest sequency, by increasing
                              sequency (Sec. 3.3)                                     */
  int32_t gx_bits;         /* 4 (paper, Sec. 5.1) | 8 (INT8 warm-up, Supp. B)         */
  int32_t gw_bits;         /* 8 (Sec. 5.2) | 16: bfloat16 operands, fp32 accumulation   */
  int32_t rounding;        /* hot_rounding                                            */
  float lqs_threshold;     /* 0.5 (Sec. 5.2.2)                                        */
  int32_t sample_tokens;   /* 0: the L tokens are one run, tiled in blocks of n (needs
                              L % n == 0).  S > 0: L = B x S tokens of B samples; the
                              token-direction transform (ABC, g_w path) tiles every sample
                              separately and pads its last block with zero tokens, so
                              S need not be a multiple of n (ViT: S = 197); then
                              L*r/n below reads B * ceil(S/n) * r                       */
  int32_t replayable;      /* 0: launch tags from the host (default).  1: from an epoch in
                              the workspace that every call advances with one more
                              launch; calls may then be recorded into a HIP graph        */
} hot_config;

/* Fills *cfg with the paper's defaults: n = 16, r = 8, low-sequency rows, INT4 /
 * INT8, pseudo-stochastic rounding, threshold 0.5, one run of tokens, host tags. */
void hot_default_config(hot_config* cfg);

const char* hot_status_string(hot_status s);

/* Bytes of the compressed activation buffer for x [L x I] (Sec. 5.2.1): a
 * 256-byte header holding the scale, then L*r/n x I INT8 codes stored with the
 * reduced token index contiguous (row pitch rounded up to 128 bytes).  Returns 0
 * for an invalid config or shape. */
size_t hot_act_buffer_bytes(const hot_config* cfg, int64_t L, int64_t I);

/* Bytes every workspace starts with (scales, abs-max exchange slots, split-K flags); the
 * whole workspace of hot_compress_activation and hot_quantize_weight. */
#define HOT_WS_PREFIX_BYTES 24832

/* Scratch bytes sufficient for every call below at this (L, O, I); 0 = invalid.  A function
 * of the configuration and the shape only: launch plans, and with them the scratch of the
 * split-K GEMMs, are made for the 256 compute units of the MI355X whatever device is
 * current. */
size_t hot_workspace_bytes(const hot_config* cfg, int64_t L, int64_t O, int64_t I);

/*
 * Activation Buffer Compression, Sec. 5.2.1, run right after the forward pass:
 *   x_hat = rows keep_idx of (H_n applied to every block of n consecutive tokens
 *   of x), INT8 with one abs-max scale for the tensor.
 * x: device [L x I] (in).  act_buf: device, hot_act_buffer_bytes() bytes (out).
 * ws: at least HOT_WS_PREFIX_BYTES (nothing beyond them is touched).
 * Requires L % n == 0, L*r/n <= 133144.
 */
hot_status hot_compress_activation(const hot_config* cfg, const float* x, int64_t L, int64_t I,
                                   void* act_buf, void* ws, size_t ws_bytes, void* stream);

/*
 * Activation-gradient path, Sec. 5.1 (Eq. 3-4 with Q = INT4):
 *   g_x = dequant( Q(g_y.H^T) . Q(H.w) ),  H block-diagonal along O.
 * g_y: device [L x O] (in); w: device [O x I] (in); g_x: device [L x I] (out).
 * gy_quantizer: scale of the rotated g_y per token or per tensor (Sec. 4.3,
 * 5.2.2); the rotated w always has one scale.  Requires O % n == 0.
 */
hot_status hot_linear_backward_gx(const hot_config* cfg, const float* g_y, const float* w,
                                  int64_t L, int64_t O, int64_t I, hot_quantizer gy_quantizer,
                                  float* g_x, void* ws, size_t ws_bytes, void* stream);

/*
 * hot_linear_backward_gx for callers that cannot allocate device memory or pass a
 * workspace: code under HIP graph capture set-up, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, same kernels, same g_x bit for bit, but the scratch is
 * an array inside the library's code object (HOT_NOALLOC_SCRATCH_BYTES, 64 MiB, held on
 * every GPU the library runs on until the process ends) instead of `ws`.  The call
 * allocates and frees nothing, on the device or through any library.
 *   - A shape whose hot_linear_backward_gx workspace layout exceeds the array returns
 *     HOT_ERR_SCRATCH_LIMIT before anything is launched (ViT-B fc1 at 12608 tokens needs
 *     59.5 MB and fits; 50432 tokens do not).
 *   - The array belongs to the device that is current at the call; `stream` must be a
 *     stream of that device.
 *   - All calls on one GPU share the array, which keeps the last call's contents.  Nothing
 *     in it has to be cleared between calls, but two calls that overlap in time on one GPU
 *     (different streams, different threads) race on it: order them.
 */
#define HOT_NOALLOC_SCRATCH_BYTES (64u << 20)
hot_status hot_linear_backward_gx_noalloc(const hot_config* cfg, const float* g_y, const float* w,
                                          int64_t L, int64_t O, int64_t I,
                                          hot_quantizer gy_quantizer, float* g_x, void* stream);

/*
 * Frozen weights (Sec. 5.3: with LoRA-style fine-tuning the base weights stay fixed and
 * only g_x is needed): quantise H.w once, reuse it every step.
 * hot_weight_buffer_bytes: a 256-byte header holding the scale, then I rows of O codes
 * (gx_bits each, row pitch rounded up to 128 bytes); 0 for an invalid config or shape.
 * hot_quantize_weight: w device [O x I] (in) -> wq_buf device (out); ws: at least
 * HOT_WS_PREFIX_BYTES.
 * hot_linear_backward_gx_cached: hot_linear_backward_gx with the weight operand taken
 * from wq_buf (same cfg, O, I); same g_x bit for bit.  Its ws holds no weight codes:
 * hot_gx_cached_workspace_bytes() (never more than hot_workspace_bytes()) is enough, and a
 * smaller one is HOT_ERR_WORKSPACE.
 */
size_t hot_weight_buffer_bytes(const hot_config* cfg, int64_t O, int64_t I);
size_t hot_gx_cached_workspace_bytes(const hot_config* cfg, int64_t L, int64_t O, int64_t I);
hot_status hot_quantize_weight(const hot_config* cfg, const float* w, int64_t O, int64_t I,
                               void* wq_buf, void* ws, size_t ws_bytes, void* stream);
hot_status hot_linear_backward_gx_cached(const hot_config* cfg, const float* g_y,
                                         const void* wq_buf, int64_t L, int64_t O, int64_t I,
                                         hot_quantizer gy_quantizer, float* g_x, void* ws,
                                         size_t ws_bytes, void* stream);

/*
 * Weight-gradient path, Sec. 5.2 (Eq. 5 with INT8 operands):
 *   g_w = dequant( Q(HLA(g_y))^T . x_hat ),  HLA along the token index L.
 * With gw_bits = 16 (g_w is the gradient Sec. 4.2 finds sensitive to quantisation) the two
 * low-rank operands are rounded to bfloat16 instead (nearest even, no scales; the
 * activation buffer is then 25 % of fp32), multiplied on the bf16 matrix cores with fp32
 * accumulation and divided by n; no limit on L*r/n.  The sums of a long reduction are made in
 * slices that follow from the shape alone, so that g_w has the same bits in every call.
 * g_y: device [L x O] (in); act_buf: what hot_compress_activation wrote for the
 * same cfg, L, I (in); g_w: device [O x I] (out).  Requires L % n == 0.
 */
hot_status hot_linear_backward_gw(const hot_config* cfg, const float* g_y, const void* act_buf,
                                  int64_t L, int64_t O, int64_t I, float* g_w, void* ws,
                                  size_t ws_bytes, void* stream);

/*
 * Both gradients of one layer in one call (Sec. 5.1 and 5.2 on the same g_y): the same
 * g_x and g_w, bit for bit, as hot_linear_backward_gx followed by
 * hot_linear_backward_gw.  Where it is faster (16-row blocks and a g_y too large for the
 * single-pass token-direction kernel) the two quantised views of g_y (rotated along O,
 * and HLA-compressed along L) come out of shared reads of g_y: two passes over it instead
 * of three; otherwise each path makes its own, in one launch for small layers.  Both GEMMs run
 * behind the operands, in one launch where that is faster.
 * Arguments as for the two separate calls.  Requires O % n == 0 and L % n == 0
 * (or whole samples with sample_tokens).
 */
hot_status hot_linear_backward(const hot_config* cfg, const float* g_y, const float* w,
                               const void* act_buf, int64_t L, int64_t O, int64_t I,
                               hot_quantizer gy_quantizer, float* g_x, float* g_w, void* ws,
                               size_t ws_bytes, void* stream);

/*
 * Layer-wise Quantizer Selection, Sec. 5.2.2, for one layer's calibration g_y:
 * mean squared error between g_y and its rotated, gx_bits-quantised,
 * de-rotated version with per-token and with per-tensor scales; per-token is
 * chosen iff mse_tensor > 0 and (mse_tensor - mse_token) >= lqs_threshold *
 * mse_tensor.  choice / mse_token / mse_tensor are HOST pointers (the two MSE
 * pointers may be NULL).  Synchronises the stream.
 */
hot_status hot_select_quantizer(const hot_config* cfg, const float* g_y, int64_t L, int64_t O,
                                hot_quantizer* choice, double* mse_token, double* mse_tensor,
                                void* ws, size_t ws_bytes, void* stream);

/*
 * Low-pass rows by the LP_L1 criterion (Supp. B, "Hyper-parameter of HLA": the paper keeps
 * the top 8 of 16 vectors by the LP_L1 criterion of the 2-D transform it builds on).  Host
 * only.  Reading taken (the criterion is defined in that earlier work, not in the paper):
 * the n tokens of a block are a grid in raster order (4 x 4 for n = 16, 8 x 8 for n = 64,
 * 4 rows of 8 for n = 32); H_n = H_rows (x) H_cols, so natural row k = a * cols + b has
 * vertical sequency seq(a) and horizontal sequency seq(b); rows are listed by increasing
 * seq(a) + seq(b), ties by increasing max of the two, then by increasing seq(a).
 * keep_idx: host, `keep` entries (out), to be passed as hot_config.keep_idx.
 */
hot_status hot_lowpass_l1_rows(int32_t block, int32_t keep, int32_t* keep_idx);

/* ---- the operators around the linear backward --------------------------------
 *
 * What a training step of a transformer block runs beside the calls above: the
 * forward product, the activation, the layer norm, and an 8-bit form of what
 * those keep for their backward pass (hot_compress_activation's buffer serves g_w
 * only).  The conventions at the top of this file hold, and:
 *   - Tensors are [rows x cols], row-major and contiguous; a `hot_type` argument
 *     says what a tensor's elements are.  Sums, statistics and the values between a
 *     load and a store are fp32 (the layer norm's mean is summed in 64 bits); a bfloat16
 *     result is rounded once, to nearest even.
 *   - rows and cols are 1 or more; rows < 2^31, cols < 2^24 (16384 for the layer norm).
 *   - No output may overlap an input or another output (checked: HOT_ERR_ARG).
 *   - Kernels of one call exchange values only from one launch to the next, in
 *     stream order: every call may be recorded into a HIP graph and replayed, without
 *     `replayable`.  Two graphs may share a workspace if they never run at once.
 *   - Results have the same bits in every call (no atomics).
 *   - An infinity or a NaN in a row reaches that row's results (and the sums over
 *     rows) as the formulas have it, never another row's.
 */
typedef enum { HOT_F32 = 0, HOT_BF16 = 1 } hot_type;

/* RELU max(x, 0) (slope 0 at 0, NaN at a NaN); GELU x Phi(x); GELU_TANH its tanh form,
 * x / 2 (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))); SILU x / (1 + exp(-x)). */
typedef enum {
  HOT_ACT_NONE = 0, HOT_ACT_RELU = 1, HOT_ACT_GELU = 2, HOT_ACT_GELU_TANH = 3, HOT_ACT_SILU = 4
} hot_act_fn;

/*
 * 8-bit checkpoint of a tensor: 32 consecutive columns of a row (a row's last group may be
 * shorter) share a step s = 2^(e - 133), the smallest power of two from 2^-125 on that leaves
 * the group's largest magnitude within 127 steps after rounding; code = round(t / s), half to
 * even, one signed byte; the value read back is code * s, exact in either type, at most s / 2 off
 * (at the type's end, where there is no larger step, 127.5 steps and more are held at 127: up to s off).
 * A group that holds an infinity or a NaN reads back as NaN.  Layout: rows x pitch codes, pitch =
 * cols rounded up to 32 (codes past cols are 0), then, from the next multiple of 256 bytes on,
 * rows x pitch / 32 bytes e (255: NaN).  25.8 % of fp32.
 * hot_checkpoint_bytes: size of that buffer, 0 for a size out of range.
 * hot_checkpoint_write: x -> ckpt.  hot_checkpoint_read: ckpt -> x.
 */
size_t hot_checkpoint_bytes(int64_t rows, int64_t cols);
hot_status hot_checkpoint_write(const void* x, hot_type type, int64_t rows, int64_t cols, void* ckpt, void* stream);
hot_status hot_checkpoint_read(const void* ckpt, int64_t rows, int64_t cols, void* x, hot_type type, void* stream);

/*
 * y = f(x) point by point, fn not HOT_ACT_NONE; ckpt: the checkpoint of x, from the same read
 * (NULL: none is made).
 */
hot_status hot_activation_forward(hot_act_fn fn, const void* x, hot_type type, int64_t rows, int64_t cols, void* y,
                                  void* ckpt, void* stream);

/*
 * g_x = g_y f'(x), with x as it was (`x`) or from its checkpoint (`ckpt`): exactly one of the
 * two is given.  `type` is that of g_y, g_x and x; the checkpoint of either type may be used.
 * g_bias: fp32 [cols], the sum of g_x over the rows before it is rounded (the gradient of a bias in
 * front of the activation), or NULL; with it `ws` is at least
 * hot_activation_backward_workspace_bytes() bytes of scratch, 256-byte aligned, otherwise ws may be
 * NULL.  HOT_ACT_NONE is allowed here (g_x = g_y, with the sums).
 */
size_t hot_activation_backward_workspace_bytes(int64_t rows, int64_t cols);
hot_status hot_activation_backward(hot_act_fn fn, const void* g_y, hot_type type, const void* x, const void* ckpt,
                                   int64_t rows, int64_t cols, void* g_x, float* g_bias, void* ws, size_t ws_bytes,
                                   void* stream);

/*
 * Layer norm over the columns, with the residual addition in front of it:
 *   h = x + residual (rounded to x_type; h = x without a residual),
 *   y = (h - mean) rstd gamma + beta,  rstd = 1 / sqrt(var + eps), var over cols (biased).
 * residual: [rows x cols] of x_type, or NULL; h: [rows x cols] of x_type (out), required with a
 * residual and NULL without one.  gamma, beta: fp32 [cols], or NULL (1 and 0).  y: y_type; x_type
 * HOT_BF16 takes y_type HOT_BF16 only.  mean, rstd: fp32 [rows] (out).  eps >= 0.  ckpt: the
 * checkpoint of h (NULL: none is made).
 */
hot_status hot_layer_norm_forward(const void* x, hot_type x_type, const void* residual, const float* gamma,
                                  const float* beta, float eps, int64_t rows, int64_t cols, void* h, void* y,
                                  hot_type y_type, float* mean, float* rstd, void* ckpt, void* stream);

/*
 * Gradients of the layer norm: with n = (h - mean) rstd and t = g_y gamma,
 *   g_x = rstd (t - mean(t) - n mean(t n)) + g_residual,  g_gamma = sum of g_y n over the rows,
 *   g_beta = sum of g_y.  g_x is the gradient of x and of the residual alike.
 * g_y: y_type; h (x_type) or its checkpoint: exactly one of the two; g_residual: x_type, the gradient
 * that reaches h past the norm, or NULL; g_x: x_type (out).  mean, rstd: what the forward call wrote.
 * g_gamma and g_beta: fp32 [cols] (out), both or neither; with them `ws` is at least
 * hot_layer_norm_backward_workspace_bytes() bytes of scratch, 256-byte aligned, otherwise ws may be NULL.
 */
size_t hot_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols);
hot_status hot_layer_norm_backward(const void* g_y, hot_type y_type, const void* h, const void* ckpt, hot_type x_type,
                                   const float* gamma, const float* mean, const float* rstd, const void* g_residual,
                                   int64_t rows, int64_t cols, void* g_x, float* g_gamma, float* g_beta, void* ws,
                                   size_t ws_bytes, void* stream);

/*
 * Forward product of a linear layer: z = x.w^T + bias, y = f(z) + residual.
 * x: [L x I], w: [O x I] of `type`; bias: fp32 [O] or NULL; residual: [L x O] of y_type or NULL;
 * y: [L x O] of y_type (HOT_F32 operands take y_type HOT_F32 only).  fn may be HOT_ACT_NONE.
 * ckpt: the checkpoint of z as [L x O], for hot_activation_backward (NULL: none is made).
 * bfloat16 operands are multiplied exactly and summed in fp32.  fp32 operands: x.w^T is within 2^-20 of the sum of
 * |x| |w| of the exact one, beside the roundings of its fp32 additions, whatever the operands and the sizes.  Small
 * products run on the fp32 instructions; large ones on two 16-bit parts of each factor, but for the tiles whose rows
 * hold numbers of so wide a range, or so few that are not small, that the parts could not give that (infinities
 * and NaN too): those run on the fp32 instructions, in about three times the time.  So the last bits of a row may depend
 * on the other rows, within that bound.  I < 2^24, O < 2^24.
 * ws: at least hot_linear_forward_workspace_bytes() bytes of scratch, 256-byte aligned (where that is
 * 0, ws may be NULL).  A smaller product may need more than a larger one, whose tiles need no slices: a workspace
 * for several sizes is as large as the largest of theirs (a smaller one is refused).
 */
size_t hot_linear_forward_workspace_bytes(hot_type type, int64_t L, int64_t O, int64_t I);
hot_status hot_linear_forward(const void* x, const void* w, hot_type type, const float* bias, const void* residual,
                              int64_t L, int64_t O, int64_t I, hot_act_fn fn, void* y, hot_type y_type, void* ckpt,
                              void* ws, size_t ws_bytes, void* stream);

/* ---- the operators of a fine-tuning step -----------------------------------------
 *
 * With frozen weights (Sec. 5.3) a step runs hot_linear_forward and
 * hot_linear_backward_gx_cached for the weights themselves; these are what it trains and ends with:
 * low-rank adapters, the log probabilities of the tokens, the optimiser.  The first two serve
 * requests as well.  The conventions of the operators around the linear backward hold; where a
 * call allows an output on an input, it says so.
 */

/*
 * Low-rank adapters beside a shared projection, each row l with the adapter k of its request:
 *   u = x A_k^T,  y = base + scale_k u B_k^T.
 * x: [L x I], a: [adapters x rank x I], b: [adapters x O x rank], base: [L x O] or NULL (zeros), y: [L x O],
 * all of `type`; base may be y.  scale: device fp32 [adapters] or NULL (1).  u: fp32 [L x rank] (out), for the
 * backward call, or NULL.
 * offsets: device int32 [segments + 1], ascending, and index: device int32 [segments]: rows
 * offsets[s] .. offsets[s + 1] - 1 (none, one or many) have adapter index[s]; several segments may have the
 * same.  An index outside [0, adapters) is no adapter: y = base, u = 0.  Rows in front of the first segment
 * and behind the last one are left as they were, in y and in u.  offsets and index NULL (segments 0): all rows have
 * adapter 0.  Both are read by the kernels, so that a recorded call follows what they hold at each replay;
 * offsets that do not ascend or leave [0, L] give undefined results within the buffers.
 * 1 <= rank <= 128 (adapters of lower rank beside it: zeros in a and b), L < 2^27, segments <= 2^24,
 * adapters <= 65536, adapters * (O + I) < 2^27.
 * Products and sums are fp32; bfloat16 operands are exact, u enters the second product within 2^-16 of itself.  An infinity or
 * a NaN in a row stays in it; one in an adapter makes infinities or NaNs in the outputs that its elements have a part in.
 * The same call gives the same bits; the same row at another place of a batch may differ in its last ones (the order of its sums).
 * ws: at least hot_adapter_forward_workspace_bytes() bytes of scratch, 256-byte aligned.
 */
size_t hot_adapter_forward_workspace_bytes(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters,
                                           int64_t segments);
hot_status hot_adapter_forward(const void* x, const void* a, const void* b, hot_type type, const float* scale,
                               const int32_t* offsets, const int32_t* index, int64_t segments, int64_t adapters, int64_t L, int64_t O,
                               int64_t I, int64_t rank, const void* base, void* y, float* u, void* ws, size_t ws_bytes,
                               void* stream);

/*
 * Gradients of the adapters: with g_u = scale_k g_y B_k,
 *   g_x = g_base + g_u A_k,  g_A_k = sum of g_u^T x,  g_B_k = scale_k sum of g_y^T u  over the rows of adapter k.
 * g_y: [L x O], x: [L x I], g_base: [L x I] or NULL (the gradient that reaches x past the adapters,
 * hot_linear_backward_gx_cached's), g_x: [L x I] (out) or NULL, all of `type`; g_base may be g_x.  u: what the
 * forward call wrote.  g_a, g_b: fp32, of the shapes of a and b (out), both or neither, written whole: zeros for an
 * adapter that has no rows.  g_x, or g_a and g_b, must be given; x and u are needed for g_a and g_b, a for
 * g_x.  Rows without an adapter have g_x = g_base; g_x's rows outside the segments are left as they were.
 * ws: at least hot_adapter_backward_workspace_bytes() bytes of scratch, 256-byte aligned; nothing in it is kept between calls.  It
 * grows with adapters * rank * (O + I), whether they have rows or not.
 */
size_t hot_adapter_backward_workspace_bytes(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters,
                                            int64_t segments);
hot_status hot_adapter_backward(const void* g_y, const void* x, const float* u, const void* a, const void* b, hot_type type,
                                const float* scale, const int32_t* offsets, const int32_t* index, int64_t segments,
                                int64_t adapters, int64_t L, int64_t O, int64_t I, int64_t rank, const void* g_base, void* g_x,
                                float* g_a, float* g_b, void* ws, size_t ws_bytes, void* stream);

/*
 * Log probabilities of given tokens, row by row over [rows x vocab] logits z:
 *   m = max z, log S = log sum exp(z - m), log p = z - m - log S, logp = log p[target],
 *   entropy = -sum p log p (0 log 0 is 0).
 * targets: device int64 [rows], with logp: fp32 [rows] (out), both or neither; a target outside [0, vocab) is not
 * scored, its logp is 0.  entropy: fp32 [rows] (out) or NULL.  stats: fp32 [rows x 2] (out), m and log S,
 * for the backward call, or NULL.  top_logp: fp32 and top_ids: int32 [rows x top] (out), the log probabilities and
 * numbers of the `top` likeliest tokens in order, among equals the lower number first; top <= HOT_MAX_TOP, top <= vocab,
 * 0 and NULLs for none.  One output at least must be wanted.
 * A logit of -inf is a token that cannot come.  A row that holds nothing else has m = -inf, log S = 0, entropy 0, and
 * log p = -inf for every token.  A NaN or +inf makes all of its row's log probabilities and its entropy NaN; NaNs come first
 * among the likeliest.  vocab < 2^24.
 * ws: at least hot_token_logprobs_workspace_bytes() bytes of scratch, 256-byte aligned (where that is 0, ws may be
 * NULL; fewer rows may need more: a workspace for several sizes is as large as the largest of theirs).
 */
#define HOT_MAX_TOP 32
size_t hot_token_logprobs_workspace_bytes(hot_type type, int64_t rows, int64_t vocab, int32_t top);
hot_status hot_token_logprobs(const void* logits, hot_type type, int64_t rows, int64_t vocab, const int64_t* targets, float* logp,
                              float* entropy, float* stats, int32_t top, float* top_logp, int32_t* top_ids, void* ws,
                              size_t ws_bytes, void* stream);

/*
 * Gradient of the logits: g_z = g_logp (1[target] - p) - g_entropy p (log p + entropy).
 * targets with g_logp (fp32 [rows]), both or neither; entropy (what the forward call wrote) with g_entropy (fp32 [rows]), both
 * or neither; one of the pairs at least.  A row whose target is not scored has no part of g_logp; a row of -inf alone has
 * gradient 0.  A p below 2^-126 counts as 0, here and in the entropy.  g_logits: [rows x vocab] of `type` (out); it may be logits.
 */
hot_status hot_token_logprobs_backward(const void* logits, hot_type type, int64_t rows, int64_t vocab, const int64_t* targets,
                                       const float* stats, const float* entropy, const float* g_logp, const float* g_entropy,
                                       void* g_logits, void* stream);

/*
 * One optimiser step (AdamW) over many tensors at once:
 *   m' = beta1 m + (1 - beta1) g,  v' = beta2 v + (1 - beta2) g^2,
 *   p' = p - lr (weight_decay p + (m' / c1) / (sqrt(v' / c2) + eps)),  c = 1 - beta^step.
 * Each operation of m' and v' is one fp32 operation, in the order written ((1 - beta2) g times g).
 *
 * Moments are fp32 [n] (HOT_STATE_F32) or held in 8 bits (HOT_STATE_8BIT): blocks of 1024 elements, 1024 codes and then 32 bytes
 * e, one for every 32 of them; a new state is all zeros.  m: a signed code times 2^(e - 133), as in the 8-bit
 * checkpoint.  v: code 0 is zero, another one 1.fff x 2^(x + e - 158) with x its upper five bits and fff the lower three; e is
 * that of the largest of the 32 (32 at least), and a v' above zero is never held as zero but as code 1 at least.  e = 255: NaN, for a
 * group that held an infinity or a NaN.  Codes past n are zero.  The new weights come from m' and v' before they are
 * rounded.
 * rounding: HOT_ROUND_DRAWN is the one to train with: up with the probability that the fraction is, so that moments are right on
 * average over the steps, to 2^-20 of a code of v and 2^-17 of one of m (a v that swings by a fifth, for beta2 = 0.999).  An
 * element's 32 bits R, from its place i in its block, the step's seed and m' and v' themselves, all modulo 2^32:
 *   R = f(seed + i / 8) + (i % 8) 0x9E379E37 + bits(m') + bits(v'),  f(x): x ^= x >> 16, x *= 0x6A09E667, x ^= x >> 15,
 *   x *= 0xBB67AE85, x ^= x >> 16;  v' is held as (bits(v') + (R >> 12)) >> 20, m' as floor(m' / step + ((R & 0xFFFF) + 0.5) / 2^16).
 *   seed: from 0, x -> f(seed ^ x ^ 0x9E3779B9) for the bits of lr, c1 and c2 in fp32 and a last word: step where c1 and c2 are those
 *   of the step before, 0 otherwise; with `dynamic`, its fifth number's bits, 0 where there are four.
 * So the same call gives the same bits, and a step number must not be used twice.
 * The other two are for comparing a step's results and not for training: with HOT_ROUND_NEAREST_EVEN a v that a step moves by less than
 * half a code (all of them, for beta2 = 0.999) stays where it is; HOT_ROUND_PSEUDO_STOCHASTIC, up where the fraction is more than the low 11
 * bits are, read as a fraction, of what is rounded (m' in steps of its group; v' itself), takes the same way in every step whose gradient
 * does not change those bits: with gradients of zero, constant or rare ones v does not follow.
 */
typedef enum { HOT_STATE_F32 = 0, HOT_STATE_8BIT = 1 } hot_state_form;
typedef enum { HOT_MOMENT_M = 0, HOT_MOMENT_V = 1 } hot_moment;
typedef struct {
  const void* grad;        /* grad_type [n]                                                            */
  void *param, *m, *v;     /* param_type [n]; moments                                                  */
  void *param_out, *m_out, *v_out; /* results, apart from all inputs; NULL: in place                   */
  void* copy;              /* bfloat16 [n] (out): the new weights rounded, for the products; HOT_F32 weights only; or NULL */
  int64_t n;               /* 1 .. 2^40 - 1                                                            */
  int32_t param_type, grad_type;   /* hot_type                                                         */
  float weight_decay;
  float lr_factor;         /* the tensor's learning rate in units of the call's                        */
} hot_adamw_tensor;
typedef struct {
  double lr, beta1, beta2, eps;    /* 0 <= beta < 1, eps > 0                                            */
  int64_t step;            /* 1 for the first one                                                       */
  int32_t rounding;        /* hot_rounding, of 8-bit moments: HOT_ROUND_DRAWN to train with              */
  int32_t dynamic_count;   /* numbers at `dynamic`: 4 (or 0, the same), or 5                             */
  const float* dynamic;    /* NULL, or device fp32 [4]: lr, c1, c2 and a factor of every gradient (loss scale, clipping), read
                              by the kernels in place of lr and step: for recorded calls; apart from the tensors.  A fifth one
                              for HOT_ROUND_DRAWN, which has to differ from step to step (the step, say): without it, steps whose lr,
                              c1 and c2 are alike (from some thousand steps on, where lr does not change) round alike */
} hot_adamw_config;

/* Bytes of one moment of n elements; 0 for a size out of range. */
size_t hot_adamw_state_bytes(hot_state_form form, int64_t n);
/* An 8-bit moment as values (exact in either type), and values (v: none below zero) as an 8-bit moment, rounded to nearest. */
hot_status hot_adamw_state_read(const void* state, hot_moment moment, int64_t n, void* out, hot_type type, void* stream);
hot_status hot_adamw_state_write(const void* x, hot_type type, hot_moment moment, int64_t n, void* state, void* stream);

/* The tensors of a step, checked once and written into `table`, HOST memory of hot_adamw_table_bytes(count) bytes that the
 * caller keeps (0: count below 1), aligned to 8: it holds addresses, so that other gradients, ones allocated anew for each step among
 * them, need another table.  No output of any tensor may lie on another one or on an input (HOT_ERR_ARG); moments
 * of all tensors have the same form. */
size_t hot_adamw_table_bytes(int32_t count);
hot_status hot_adamw_table(const hot_adamw_tensor* tensors, int32_t count, hot_state_form state, void* table, size_t table_bytes);

/* One step: a launch for every forty tensors.  A recorded call keeps the tensors, lr, step and the other numbers it was
 * recorded with, but for what `dynamic` points to; the table is not read after the call returns. */
hot_status hot_adamw_step(const void* table, const hot_adamw_config* cfg, void* stream);

/* ---- parity views (not on the timed path): logical forms of packed data ---- */

/* Compressed activation as row-major codes [L*r/n x I] and its scale [1].  With
 * gw_bits = 16 `codes` receives bfloat16 bit patterns, two bytes each (pass an int16
 * buffer), and the scale is 1. */
hot_status hot_debug_unpack_activation(const hot_config* cfg, const void* act_buf, int64_t L,
                                       int64_t I, int8_t* codes, float* scale, void* stream);

/* Quantised weights as row-major codes [O x I] (one code per byte) and their scale [1]. */
hot_status hot_debug_unpack_weight(const hot_config* cfg, const void* wq_buf, int64_t O, int64_t I,
                                   int8_t* codes, float* scale, void* stream);

/* Operands left in `ws` by the last hot_linear_backward_gx with these arguments:
 * codes of the rotated g_y [L x O] and w [O x I] (row-major, one code per byte),
 * scales of g_y ([L] per token, [1] per tensor) and of w [1], and the int32
 * integer product [L x I] recomputed from those operands by the GEMM the call itself
 * used (the GEMM scratch at the end of `ws` is overwritten).  Any output may be NULL. */
hot_status hot_debug_gx_operands(const hot_config* cfg, void* ws, int64_t L, int64_t O,
                                 int64_t I, hot_quantizer gy_quantizer, int8_t* gy_codes,
                                 float* gy_scales, int8_t* w_codes, float* w_scale, int32_t* acc,
                                 void* stream);

/* Operands left in `ws` by the last hot_linear_backward_gw: codes of HLA(g_y)
 * [L*r/n x O] row-major, its scale [1], and the int32 product [O x I] recomputed
 * from those codes and act_buf.  Any output may be NULL.  With gw_bits = 16 the codes are
 * bfloat16 bit patterns (two bytes each) and `acc` receives the fp32 accumulators' bit
 * patterns. */
hot_status hot_debug_gw_operands(const hot_config* cfg, void* ws, const void* act_buf,
                                 int64_t L, int64_t O, int64_t I, int8_t* gy_codes,
                                 float* gy_scale, int32_t* acc, void* stream);

/* Operands left in `ws` by the last hot_linear_backward (block size 16 or 32): the
 * outputs of both views above.  Any output may be NULL. */
hot_status hot_debug_fused_operands(const hot_config* cfg, void* ws, const void* act_buf,
                                    int64_t L, int64_t O, int64_t I, hot_quantizer gy_quantizer,
                                    int8_t* gy_codes, float* gy_scales, int8_t* w_codes,
                                    float* w_scale, int32_t* acc_gx, int8_t* gyT_codes,
                                    float* gyT_scale, int32_t* acc_gw, void* stream);

/* Strategy of hot_linear_backward: 0 = chosen by the library (default), 1 = never the shared
 * passes over g_y, 2 = the shared passes whenever they exist (block sizes 16 and
 * 32, INT8 g_w operands, one run of tokens), 3 = as 1 with every kernel in a launch of its own
 * (by default small layers have their operands made in one launch, weights and per-token g_y rows
 * of larger ones in another, and both GEMMs share a launch where that is faster; the setting also
 * applies to hot_linear_backward_gx).
 * Results do not depend on it.  Process-wide. */
hot_status hot_debug_set_backward_strategy(int strategy);

/* Tensors small enough to stay in the register files of the resident workgroups (x and
 * w of the ViT-sized layers) are transformed and quantised by a single-pass kernel whose
 * workgroups exchange their abs-max through the workspace and wait for each other at most
 * `us` microseconds (default 200) before computing what is missing themselves; results
 * do not depend on the value.  us = 0: never wait (exercises the self-computed path);
 * us < 0: always use the two-pass kernels.  The same bound (us <= 0: never wait) applies
 * to a split-K GEMM's wait for another workgroup's partial sums.  Process-wide setting. */
hot_status hot_debug_set_exchange_wait_us(int us);

/* Work distribution of the GEMMs: 0 = chosen by the library (default: K is split for
 * outputs with no more tiles than compute units), 1 = one workgroup per output tile,
 * s = 2..8: the K range cut into s slices, one workgroup each, wherever a split of the
 * 128x128 tile applies (integer operands, at least 4 K stages per slice); the slices'
 * partial sums are handed to the last one through the workspace; 10 / 11 / 12 / 13: every
 * GEMM on 128x128 / 192x256 / 256x256 / 128x256 tiles, one workgroup per tile (11 and 13
 * exist for INT4 operands only; INT8 and bfloat16 GEMMs then take 256x256).  Integer results, and
 * therefore all outputs, do not depend on it; a bfloat16 GEMM whose sums are made in slices keeps
 * them, and the 128x128 tile, in every mode.  Process-wide. */
hot_status hot_debug_set_gemm_mode(int mode);

/* ---- stage timing for benchmarks (off by default) ---- */

/* Kernel roles timed separately; hot_debug_stage_name() gives their names.  The first HOT_NUM_STAGES are those of the
 * linear backward, the next nine those of the operators around it; 24 is none, and those of a fine-tuning step follow. */
#define HOT_NUM_STAGES 15
#define HOT_NUM_STAGES_ALL 36

/* From this call on, every kernel the library launches is bracketed by two HIP
 * events recorded on its stream.  Host-side state only; not thread-safe against
 * concurrent hot_* calls from other threads' streams being interleaved. */
hot_status hot_debug_profile_begin(void);

/* Stops recording, waits for the recorded events, and returns per stage the
 * summed elapsed milliseconds and the number of launches (host arrays of
 * HOT_NUM_STAGES entries: the stages of the linear backward alone). */
hot_status hot_debug_profile_end(float* stage_ms, int64_t* stage_launches);

/* The same for the first `count` stages of all (host arrays of `count` entries; those past
 * HOT_NUM_STAGES_ALL become 0). */
hot_status hot_debug_profile_end_all(float* stage_ms, int64_t* stage_launches, int32_t count);

/* The stages of the recording that the last hot_debug_profile_end closed, in launch order:
 * writes up to `capacity` stage ids to `stages` (host; may be NULL) and returns how many
 * launches there were. */
int64_t hot_debug_profile_sequence(int32_t* stages, int64_t capacity);

const char* hot_debug_stage_name(int stage);

/* How the GEMMs of a layer are distributed in the modes set above, with a full-size workspace (host only, nothing
 * is launched): whether hot_linear_backward makes one launch of both, and for each its tile rows and columns, its
 * K slices, whether a second kernel adds the slices' sums, and whether the output is stored with the streaming hint;
 * the last two are those of hot_linear_backward_gx (also with cached weights) and hot_linear_backward_gw. */
typedef struct hot_gemm_plan {
  int32_t one_launch;
  int32_t gx[5], gw[5], gx_alone[5], gw_alone[5];
} hot_gemm_plan;
hot_status hot_debug_gemm_plan(const hot_config* cfg, int64_t L, int64_t O, int64_t I, hot_gemm_plan* plan);

/* How hot_linear_forward works on a product (host only, nothing is launched; of the first 2^23 rows of a longer x):
 * rows and outputs a workgroup, how many such tiles there are, how many have a workgroup each (the others are summed in
 * `slices` slices of the columns), whether rows end inside a 128-byte piece of the tiles that take operands as they are, and
 * whether y is stored with the streaming hint. */
typedef enum {
  HOT_LINEAR_ROWS = 0,     /* few rows: operands from memory to the matrix instructions */
  HOT_LINEAR_DIRECT = 1,   /* small tiles of the operands as they are                   */
  HOT_LINEAR_TILES = 2,    /* large tiles of bfloat16 operands as they are              */
  HOT_LINEAR_PACKED = 3    /* large tiles of operands that a first launch packs         */
} hot_linear_way;
typedef struct hot_linear_plan {
  int32_t way, tile_rows, tile_cols;
  int32_t tiles, whole, slices;
  int32_t masked, streams;
} hot_linear_plan;
hot_status hot_debug_linear_plan(hot_type type, hot_type y_type, int64_t L, int64_t O, int64_t I, int32_t with_ckpt,
                                 hot_linear_plan* plan);

/* Machine-peak probes (context for the roofline figures, not the method): one launch of
 * kind 0 = read `bytes` of buf, 1 = write them (4 = with the streaming, non-temporal, hint the
 * GEMM epilogue uses), 2 / 3 = `iters` x 16 int8 32x32x32 matrix
 * instructions per wave on all SIMDs with constant / pseudo-random register operands
 * (buf, >= 1 MiB, receives a checksum).  The caller times the launch. */
hot_status hot_debug_probe(int kind, void* buf, size_t bytes, int iters, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HOT_H */
