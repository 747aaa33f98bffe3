// What the C entry points of the operators check and record: types, sizes, buffers, stages.
#pragma once
#include "hot_host.h"

namespace hot {

constexpr int64_t kMaxRows = 1ll << 31, kMaxCols = 1ll << 24;

inline bool size_ok(int64_t rows, int64_t cols) { return rows >= 1 && cols >= 1 && rows < kMaxRows && cols < kMaxCols; }
inline bool type_ok(hot_type t) { return t == HOT_F32 || t == HOT_BF16; }
inline int64_t bytes_of(hot_type t, int64_t rows, int64_t cols) { return rows * cols * (t == HOT_BF16 ? 2 : 4); }
inline bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

// Collects a call's buffers: aligned, and no output on top of an input or of another output.
class Buffers {
 public:
  void in(const void* p, int64_t bytes) { add(p, bytes, false); }
  void out(const void* p, int64_t bytes) { add(p, bytes, true); }
  bool ok() const {
    for (int i = 0; i < n_; ++i) {
      if (!aligned_) return false;
      for (int j = 0; j < i; ++j)
        if ((out_[i] || out_[j]) && lo_[i] < hi_[j] && lo_[j] < hi_[i]) return false;
    }
    return true;
  }

 private:
  void add(const void* p, int64_t bytes, bool out) {
    if (!p) return;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (a & 15u) aligned_ = false;
    lo_[n_] = a;
    hi_[n_] = a + (uintptr_t)bytes;
    out_[n_++] = out;
  }
  uintptr_t lo_[16], hi_[16];
  bool out_[16];
  int n_ = 0;
  bool aligned_ = true;
};

#define HOT_STAGE(stage, expr)                   \
  do {                                           \
    stage_begin(stage, s);                       \
    const hipError_t e_ = (expr);                \
    stage_end(stage, s);                         \
    if (e_ != hipSuccess) return HOT_ERR_DEVICE; \
  } while (0)

}  // namespace hot
