// C ABI of the operators of a fine-tuning step: argument checks, workspace layouts and the launches behind each call.
#include <math.h>

#include <algorithm>
#include <new>

#include "adapter_host.h"
#include "block_host.h"
#include "call_checks.h"
#include "tune_host.h"

namespace hot {

namespace {

// ---- adapters ----
constexpr int64_t kMaxBatchRows = 1ll << 27, kMaxSegments = 1ll << 24, kMaxAdapters = 1ll << 16, kMaxAdapterCols = 1ll << 27;   // fewer than 2^32 lanes a launch

bool adapter_size_ok(int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters, int64_t segments) {
  return size_ok(L, O) && size_ok(L, I) && L < kMaxBatchRows && rank >= 1 && rank <= kMaxRank && adapters >= 1 &&
         adapters <= kMaxAdapters && adapters * (O + I) < kMaxAdapterCols && segments >= 0 && segments <= kMaxSegments;
}
bool batch_ok(const int32_t* offsets, const int32_t* index, int64_t segments) {
  return !offsets == !index && !offsets == (segments == 0);
}

// ---- optimiser ----
constexpr uint64_t kTableMark = 0x31574d6164746f68ull;
constexpr int64_t kMaxElements = 1ll << 40, kMaxBlocks = 1ll << 23;   // 2^31 lanes a launch
struct TableHead {
  uint64_t mark;
  int32_t count, state;
};
static_assert(sizeof(TableHead) == 16, "entries follow");

struct Interval {
  uintptr_t lo, hi;
  bool out;
};
// Whether no output lies on an input or on another output.
bool apart(Interval* t, size_t n) {
  std::sort(t, t + n, [](const Interval& a, const Interval& b) { return a.lo < b.lo; });
  uintptr_t ends = 0, out_ends = 0;      // of those before
  for (size_t i = 0; i < n; ++i) {
    if (t[i].lo < (t[i].out ? ends : out_ends)) return false;
    ends = std::max(ends, t[i].hi);
    if (t[i].out) out_ends = std::max(out_ends, t[i].hi);
  }
  return true;
}

}  // namespace
}  // namespace hot

using namespace hot;

extern "C" {

size_t hot_adapter_forward_workspace_bytes(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters,
                                           int64_t segments) {
  if (!type_ok(type) || !adapter_size_ok(L, O, I, rank, adapters, segments)) return 0;
  return adapter_plan(type, L, O, I, rank, adapters, segments).forward;
}
size_t hot_adapter_backward_workspace_bytes(hot_type type, int64_t L, int64_t O, int64_t I, int64_t rank, int64_t adapters,
                                            int64_t segments) {
  if (!type_ok(type) || !adapter_size_ok(L, O, I, rank, adapters, segments)) return 0;
  return adapter_plan(type, L, O, I, rank, adapters, segments).backward;
}

hot_status hot_adapter_forward(const void* x, const void* a, const void* b, hot_type type, const float* scale,
                               const int32_t* offsets, const int32_t* index, int64_t segments, int64_t adapters, int64_t L, int64_t O,
                               int64_t I, int64_t rank, const void* base, void* y, float* u, void* ws, size_t ws_bytes,
                               void* stream) {
  if (!x || !a || !b || !y || !ws || !aligned256(ws) || !type_ok(type) || !batch_ok(offsets, index, segments)) return HOT_ERR_ARG;
  if (!adapter_size_ok(L, O, I, rank, adapters, segments)) return HOT_ERR_SHAPE;
  const AdapterPlan p = adapter_plan(type, L, O, I, rank, adapters, segments);
  Buffers k;
  k.in(x, bytes_of(type, L, I));
  k.in(a, bytes_of(type, adapters * rank, I));
  k.in(b, bytes_of(type, adapters * O, rank));
  k.in(scale, adapters * 4);
  k.in(offsets, (segments + 1) * 4);
  k.in(index, segments * 4);
  if (base != y) k.in(base, bytes_of(type, L, O));
  k.out(y, bytes_of(type, L, O));
  k.out(u, L * rank * 4);
  k.out(ws, (int64_t)p.forward);
  if (!k.ok()) return HOT_ERR_ARG;
  if (ws_bytes < p.forward) return HOT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const AdapterBatch batch{offsets, index, (int)segments, (int)adapters, L};
  char* const w = (char*)ws;
  const bool sliced = p.slices_forward > 1;
  AdapterShrink shrink{batch, x, a, (float*)ws, I, rank * I, 0, (int)rank, p.pitch, p.slices_forward, p.slice_forward,
                       sliced ? nullptr : u, sliced ? nullptr : w + p.factors, scale, p.chunks};
  if (p.pack_forward) {
    const AdapterPrepare prepare{batch, nullptr, a, nullptr, w + p.wt, I, I, I, 1, p.wt_stride, (int)rank, nullptr, nullptr, nullptr};
    HOT_STAGE(kStAdapterPrepare, launch_adapter_prepare(prepare, type, s));
    shrink.w = w + p.wt;
    shrink.w_stride = p.wt_stride;
    shrink.w_packed = 1;
  }
  HOT_STAGE(kStAdapterShrink, launch_adapter_shrink(shrink, p.tile, type, s));
  const AdapterExpand expand{batch, (const float*)ws, b, base, scale, y, sliced ? u : nullptr, shrink.packed, O, rank, O * rank, (int)rank,
                             p.pitch, p.slices_forward};
  HOT_STAGE(kStAdapterExpand, launch_adapter_expand(expand, p.rows, type, s));
  return HOT_OK;
}

hot_status hot_adapter_backward(const void* g_y, const void* x, const float* u, const void* a, const void* b, hot_type type,
                                const float* scale, const int32_t* offsets, const int32_t* index, int64_t segments,
                                int64_t adapters, int64_t L, int64_t O, int64_t I, int64_t rank, const void* g_base, void* g_x,
                                float* g_a, float* g_b, void* ws, size_t ws_bytes, void* stream) {
  if (!g_y || !b || !ws || !aligned256(ws) || !type_ok(type) || !batch_ok(offsets, index, segments)) return HOT_ERR_ARG;
  if (!g_a != !g_b || (!g_x && !g_a) || (g_x && !a) || (g_a && (!x || !u)) || (g_base && !g_x)) return HOT_ERR_ARG;
  if (!adapter_size_ok(L, O, I, rank, adapters, segments)) return HOT_ERR_SHAPE;
  const AdapterPlan p = adapter_plan(type, L, O, I, rank, adapters, segments);
  Buffers k;
  k.in(g_y, bytes_of(type, L, O));
  k.in(x, bytes_of(type, L, I));
  k.in(u, L * rank * 4);
  k.in(a, bytes_of(type, adapters * rank, I));
  k.in(b, bytes_of(type, adapters * O, rank));
  k.in(scale, adapters * 4);
  k.in(offsets, (segments + 1) * 4);
  k.in(index, segments * 4);
  if (g_base != g_x) k.in(g_base, bytes_of(type, L, I));
  k.out(g_x, bytes_of(type, L, I));
  k.out(g_a, adapters * rank * I * 4);
  k.out(g_b, adapters * rank * O * 4);
  k.out(ws, (int64_t)p.backward);
  if (!k.ok()) return HOT_ERR_ARG;
  if (ws_bytes < p.backward) return HOT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  char* const w = (char*)ws;
  float* const g_u = (float*)w;
  int32_t* const order = (int32_t*)(w + p.sorted);
  int32_t* const start = order + segments;
  int32_t* const first = start + segments + 1;
  const AdapterBatch batch{offsets, index, (int)segments, (int)adapters, L};
  const bool sort = offsets && g_a;
  const AdapterPrepare prepare{batch, a, b, g_x ? w + p.at : nullptr, w + p.wt, I, O, 1, rank, p.wt_stride, (int)rank,
                               sort ? order : nullptr, start, first};
  HOT_STAGE(kStAdapterPrepare, launch_adapter_prepare(prepare, type, s));
  const bool sliced = p.slices_backward > 1;
  const AdapterShrink shrink{batch, g_y, w + p.wt, g_u, O, p.wt_stride, 1, (int)rank, p.pitch, p.slices_backward, p.slice_backward,
                             nullptr, sliced || !g_x ? nullptr : w + p.factors, scale, p.chunks};
  HOT_STAGE(kStAdapterShrink, launch_adapter_shrink(shrink, p.tile, type, s));
  if (g_x) {
    const AdapterExpand expand{batch, g_u, w + p.at, g_base, scale, g_x, nullptr, shrink.packed, I, rank, I * rank, (int)rank, p.pitch,
                               p.slices_backward};
    HOT_STAGE(kStAdapterExpand, launch_adapter_expand(expand, p.rows, type, s));
  }
  if (g_a) {
    const int64_t half = (type == HOT_BF16 ? 6 : 4) * round_up(rank, 16) * p.positions;
    AdapterPack pack{};
    pack.b = batch;
    pack.g_u = g_u;
    pack.u = u;
    pack.g_out = w + p.packed;
    pack.u_out = w + p.packed + half;
    if (offsets) {
      pack.order = order;
      pack.start = start;
      pack.first = first;
    }
    pack.rows = first + adapters + 1;
    pack.rank = (int)rank;
    pack.g_pitch = p.pitch;
    pack.slices = p.slices_backward;
    HOT_STAGE(kStAdapterPack, launch_adapter_pack(pack, type, s));
    AdapterOuter outer{};
    outer.b = batch;
    outer.a[0] = AdapterOuterOperand{pack.g_out, x, (float*)(w + p.part_a), I};
    outer.a[1] = AdapterOuterOperand{pack.u_out, g_y, (float*)(w + p.part_b), O};
    outer.scale = scale;
    outer.first = pack.first;
    outer.rows = pack.rows;
    outer.rank = (int)rank;
    outer.parts = p.parts;
    HOT_STAGE(kStAdapterOuter, launch_adapter_outer(outer, type, s));
    const AdapterReduce reduce{outer.first, L, I, O, outer.a[0].part, outer.a[1].part, g_a, g_b, (int)rank, p.parts, (int)adapters};
    HOT_STAGE(kStAdapterSums, launch_adapter_reduce(reduce, s));
  }
  return HOT_OK;
}

size_t hot_token_logprobs_workspace_bytes(hot_type type, int64_t rows, int64_t vocab, int32_t top) {
  if (!type_ok(type) || !size_ok(rows, vocab) || top < 0 || top > HOT_MAX_TOP || top > vocab) return 0;
  return logprob_scratch_bytes(rows, vocab, top);
}

hot_status hot_token_logprobs(const void* logits, hot_type type, int64_t rows, int64_t vocab, const int64_t* targets, float* logp,
                              float* entropy, float* stats, int32_t top, float* top_logp, int32_t* top_ids, void* ws,
                              size_t ws_bytes, void* stream) {
  if (!logits || !type_ok(type) || !targets != !logp || !top_logp != !top_ids || !top_logp != (top == 0)) return HOT_ERR_ARG;
  if (!logp && !entropy && !stats && !top) return HOT_ERR_ARG;
  if (!size_ok(rows, vocab) || top < 0 || top > HOT_MAX_TOP || top > vocab) return HOT_ERR_SHAPE;
  const size_t need = logprob_scratch_bytes(rows, vocab, top);
  if (need && (!ws || !aligned256(ws))) return HOT_ERR_ARG;
  Buffers b;
  b.in(logits, bytes_of(type, rows, vocab));
  b.in(targets, rows * 8);
  b.out(logp, rows * 4);
  b.out(entropy, rows * 4);
  b.out(stats, rows * 8);
  b.out(top_logp, rows * top * 4);
  b.out(top_ids, rows * top * 4);
  if (need) b.out(ws, (int64_t)need);
  if (!b.ok()) return HOT_ERR_ARG;
  if (ws_bytes < need) return HOT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const LogProbs a{logits, type, rows, vocab, targets, logp, entropy, stats, top, top_logp, top_ids, ws};
  HOT_STAGE(kStLogProbs, launch_logprobs(a, s));
  return HOT_OK;
}

hot_status hot_token_logprobs_backward(const void* logits, hot_type type, int64_t rows, int64_t vocab, const int64_t* targets,
                                       const float* stats, const float* entropy, const float* g_logp, const float* g_entropy,
                                       void* g_logits, void* stream) {
  if (!logits || !type_ok(type) || !stats || !g_logits || !targets != !g_logp || !entropy != !g_entropy || (!g_logp && !g_entropy))
    return HOT_ERR_ARG;
  if (!size_ok(rows, vocab)) return HOT_ERR_SHAPE;
  Buffers b;
  if (logits != g_logits) b.in(logits, bytes_of(type, rows, vocab));
  b.in(targets, rows * 8);
  b.in(stats, rows * 8);
  b.in(entropy, rows * 4);
  b.in(g_logp, rows * 4);
  b.in(g_entropy, rows * 4);
  b.out(g_logits, bytes_of(type, rows, vocab));
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  const LogProbGrad a{logits, type, rows, vocab, targets, stats, entropy, g_logp, g_entropy, g_logits};
  HOT_STAGE(kStLogProbsGrad, launch_logprob_grad(a, s));
  return HOT_OK;
}

size_t hot_adamw_state_bytes(hot_state_form form, int64_t n) {
  if (n < 1 || n >= kMaxElements) return 0;
  return form == HOT_STATE_F32 ? (size_t)n * 4 : form == HOT_STATE_8BIT ? (size_t)state_bytes(n) : 0;
}

hot_status hot_adamw_state_read(const void* state, hot_moment moment, int64_t n, void* out, hot_type type, void* stream) {
  if (!state || !out || !type_ok(type) || (moment != HOT_MOMENT_M && moment != HOT_MOMENT_V)) return HOT_ERR_ARG;
  if (n < 1 || n >= kMaxElements) return HOT_ERR_SHAPE;
  Buffers b;
  b.in(state, state_bytes(n));
  b.out(out, bytes_of(type, 1, n));
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  HOT_STAGE(kStStateRead, launch_state_read(state, moment == HOT_MOMENT_V, n, out, type, s));
  return HOT_OK;
}

hot_status hot_adamw_state_write(const void* x, hot_type type, hot_moment moment, int64_t n, void* state, void* stream) {
  if (!state || !x || !type_ok(type) || (moment != HOT_MOMENT_M && moment != HOT_MOMENT_V)) return HOT_ERR_ARG;
  if (n < 1 || n >= kMaxElements) return HOT_ERR_SHAPE;
  Buffers b;
  b.in(x, bytes_of(type, 1, n));
  b.out(state, state_bytes(n));
  if (!b.ok()) return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  HOT_STAGE(kStStateWrite, launch_state_write(x, type, moment == HOT_MOMENT_V, n, state, s));
  return HOT_OK;
}

size_t hot_adamw_table_bytes(int32_t count) { return count < 1 ? 0 : sizeof(TableHead) + (size_t)count * sizeof(AdamWEntry); }

hot_status hot_adamw_table(const hot_adamw_tensor* tensors, int32_t count, hot_state_form state, void* table, size_t table_bytes) {
  if (!tensors || !table || (reinterpret_cast<uintptr_t>(table) & 7u) || (state != HOT_STATE_F32 && state != HOT_STATE_8BIT)) return HOT_ERR_ARG;
  if (count < 1) return HOT_ERR_SHAPE;
  if (table_bytes < hot_adamw_table_bytes(count)) return HOT_ERR_WORKSPACE;
  Interval* const held = new (std::nothrow) Interval[(size_t)count * 8];
  if (!held) return HOT_ERR_DEVICE;
  TableHead* const head = (TableHead*)table;
  AdamWEntry* const e = (AdamWEntry*)(head + 1);
  head->mark = 0;                       // until all is found right
  size_t n = 0;
  hot_status st = HOT_OK;
  const auto hold = [&](const void* p, int64_t bytes, bool out) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    if (at & 15u) st = HOT_ERR_ARG;
    held[n++] = Interval{at, at + (uintptr_t)bytes, out};
  };
  for (int32_t i = 0; i < count && st == HOT_OK; ++i) {
    const hot_adamw_tensor& t = tensors[i];
    const hot_type pt = (hot_type)t.param_type, gt = (hot_type)t.grad_type;
    if (!t.param || !t.grad || !t.m || !t.v || !type_ok(pt) || !type_ok(gt) || (t.copy && pt != HOT_F32) || !std::isfinite(t.weight_decay) ||
        !std::isfinite(t.lr_factor)) {
      st = HOT_ERR_ARG;
      break;
    }
    if (t.n < 1 || t.n >= kMaxElements) {
      st = HOT_ERR_SHAPE;
      break;
    }
    AdamWEntry& k = e[i];
    k = AdamWEntry{t.param, t.param_out ? t.param_out : t.param, t.copy, t.grad, t.m, t.v, t.m_out ? t.m_out : t.m, t.v_out ? t.v_out : t.v,
                   t.n, t.weight_decay, t.lr_factor, (pt == HOT_BF16 ? 1u : 0u) | (gt == HOT_BF16 ? 2u : 0u), 0};
    const int64_t moment = (int64_t)hot_adamw_state_bytes(state, t.n);
    hold(k.p_out, bytes_of(pt, 1, t.n), true);
    hold(k.m_out, moment, true);
    hold(k.v_out, moment, true);
    if (k.copy) hold(k.copy, bytes_of(HOT_BF16, 1, t.n), true);
    hold(k.g, bytes_of(gt, 1, t.n), false);
    if (k.p != k.p_out) hold(k.p, bytes_of(pt, 1, t.n), false);
    if (k.m != k.m_out) hold(k.m, moment, false);
    if (k.v != k.v_out) hold(k.v, moment, false);
  }
  if (st == HOT_OK && !apart(held, n)) st = HOT_ERR_ARG;
  delete[] held;
  if (st != HOT_OK) return st;
  head->count = count;
  head->state = state;
  head->mark = kTableMark;
  return HOT_OK;
}

hot_status hot_adamw_step(const void* table, const hot_adamw_config* cfg, void* stream) {
  if (!table || !cfg || (reinterpret_cast<uintptr_t>(table) & 7u) || (reinterpret_cast<uintptr_t>(cfg->dynamic) & 15u)) return HOT_ERR_ARG;
  const TableHead* const head = (const TableHead*)table;
  const AdamWEntry* const e = (const AdamWEntry*)(head + 1);
  if (head->mark != kTableMark) return HOT_ERR_ARG;
  const hot_rounding rounding = (hot_rounding)cfg->rounding;
  if (rounding != HOT_ROUND_NEAREST_EVEN && rounding != HOT_ROUND_PSEUDO_STOCHASTIC && rounding != HOT_ROUND_DRAWN) return HOT_ERR_ARG;
  if (cfg->dynamic_count != 0 && cfg->dynamic_count != 4 && cfg->dynamic_count != 5) return HOT_ERR_ARG;
  if (!(cfg->beta1 >= 0 && cfg->beta1 < 1) || !(cfg->beta2 >= 0 && cfg->beta2 < 1) || !((float)cfg->eps > 0) || !std::isfinite(cfg->eps) ||
      !std::isfinite(cfg->lr) || (!cfg->dynamic && cfg->step < 1))
    return HOT_ERR_ARG;
  hipStream_t s = (hipStream_t)stream;
  AdamWArgs a{};
  a.s.beta1 = (float)cfg->beta1;
  a.s.rest1 = (float)(1.0 - cfg->beta1);
  a.s.beta2 = (float)cfg->beta2;
  a.s.rest2 = (float)(1.0 - cfg->beta2);
  a.s.eps = (float)cfg->eps;
  a.s.lr = (float)cfg->lr;
  a.s.corr1 = (float)(1.0 - std::pow(cfg->beta1, (double)cfg->step));
  a.s.corr2 = (float)(1.0 - std::pow(cfg->beta2, (double)cfg->step));
  a.s.dyn = cfg->dynamic;
  a.s.words = cfg->dynamic_count == 5;
  // The step's number is in the seed only where the corrections no longer tell the step from the one before, so that until then recorded
  // calls, which have lr and the corrections, round as this one does.
  const double before = (double)cfg->step - 1;
  if (a.s.corr1 == (float)(1.0 - std::pow(cfg->beta1, before)) && a.s.corr2 == (float)(1.0 - std::pow(cfg->beta2, before)))
    a.s.word = (uint32_t)cfg->step;
  int32_t next = 0;
  int64_t from = 0;                       // first block of tensor `next` that is still to be done
  while (next < head->count) {
    int64_t blocks = 0;
    int in = 0;
    a.first = from * kAdamWChunk;
    while (next < head->count && in < kAdamWEntries && blocks < kMaxBlocks) {
      const int64_t all = ceil_div(e[next].n, kAdamWChunk), take = std::min(all - from, kMaxBlocks - blocks);
      a.e[in] = e[next];
      a.block[in++] = (uint32_t)blocks;
      blocks += take;
      from += take;
      if (from < all) break;
      from = 0;
      ++next;
    }
    a.count = (uint32_t)in;
    for (int i = in; i <= kAdamWEntries; ++i) a.block[i] = 0xFFFFFFFFu;
    HOT_STAGE(kStAdamW, launch_adamw(a, (uint32_t)blocks, head->state == HOT_STATE_8BIT, rounding, s));
  }
  return HOT_OK;
}

}  // extern "C"
