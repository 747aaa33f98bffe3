// Host-side declarations of the operators of a fine-tuning step: low-rank adapters, token log probabilities, the
// optimiser step.
#pragma once
#include "hot_host.h"

namespace hot {

// ---- optimiser ----
// An 8-bit moment: blocks of 1024 elements, 1024 codes and then one exponent for every 32 of them.
constexpr int kStateBlock = 1024, kStateBlockBytes = kStateBlock + kStateBlock / 32;
inline int64_t state_bytes(int64_t n) { return ceil_div(n, kStateBlock) * kStateBlockBytes; }

// Elements a workgroup updates, and tensors a launch takes: their entries travel as the kernel's argument (4 KB at most), so that a
// recorded launch holds them and nothing of the caller's has to outlive the call.
constexpr int kAdamWChunk = 2048, kAdamWEntries = 40;
struct AdamWEntry {
  const void* p;
  void* p_out;
  void* copy;        // null: none
  const void* g;
  const void *m, *v;
  void *m_out, *v_out;
  int64_t n;
  float decay, lr;   // weight decay; factor of the call's learning rate
  uint32_t types;    // bit 0: parameters are bfloat16, bit 1: gradients are
  uint32_t pad;
};
struct AdamWStep {
  float beta1, rest1, beta2, rest2;   // rest = 1 - beta
  float eps, lr, corr1, corr2;        // corr = 1 - beta^step
  const float* dyn;                   // device: lr, corr1, corr2, factor of the gradients, and (`words`) a word of the seed; or null
  uint32_t word, words;               // the seed's last word, where dyn has none
};
// `count` entries; the first one from element `first` on (a multiple of the chunk), the last one to element `last`.
struct AdamWArgs {
  AdamWStep s;
  int64_t first;
  uint32_t count;
  uint32_t block[kAdamWEntries + 1];  // first workgroup of each entry; of those past the last, beyond the grid
  AdamWEntry e[kAdamWEntries];
};
static_assert(sizeof(AdamWArgs) <= 4096, "kernel arguments");
hipError_t launch_adamw(const AdamWArgs& a, uint32_t blocks, bool eight, hot_rounding rounding, hipStream_t s);
hipError_t launch_state_read(const void* state, bool second, int64_t n, void* out, hot_type type, hipStream_t s);
hipError_t launch_state_write(const void* x, hot_type type, bool second, int64_t n, void* state, hipStream_t s);

// ---- token log probabilities ----
struct LogProbs {
  const void* logits;
  hot_type type;
  int64_t rows, vocab;
  const int64_t* targets;
  float *logp, *entropy, *stats;      // targets and logp, entropy, stats: each may be null
  int top;
  float* top_logp;
  int32_t* top_ids;
  void* ws;
};
size_t logprob_scratch_bytes(int64_t rows, int64_t vocab, int top);
hipError_t launch_logprobs(const LogProbs& a, hipStream_t s);
struct LogProbGrad {
  const void* logits;
  hot_type type;
  int64_t rows, vocab;
  const int64_t* targets;
  const float *stats, *entropy, *g_logp, *g_entropy;
  void* g_logits;
};
hipError_t launch_logprob_grad(const LogProbGrad& a, hipStream_t s);

}  // namespace hot
