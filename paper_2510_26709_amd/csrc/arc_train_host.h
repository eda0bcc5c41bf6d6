// Host-side parts that the training operators' entry points share: the token
// context, its argument checks, and helpers of contexts.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <vector>

#include "arc_context.h"
#include "arc_objective.h"
#include "arc_train.h"

struct arc_tokens {
  int64_t vocab = 0, max_rows = 0;
  int32_t bf16 = 0, top = 0;
  float scale = 1.f;
  hipStream_t stream = nullptr;
  int device = 0;
  void* workspace = nullptr;
  // Between a loss's two launches [max_rows] each: sums (two), entropies; and for
  // the objectives log probabilities and the gradients of those and of entropies.
  float* row_values = nullptr;
  arc::ObjectiveScratch* scratch = nullptr;
  float* entropies() const { return row_values + 2 * max_rows; }
  float* logps() const { return row_values + 3 * max_rows; }
  float* d_logps() const { return row_values + 4 * max_rows; }
  float* d_entropies() const { return row_values + 5 * max_rows; }

  void release() {
    (void)hipStreamSynchronize(stream);
    if (workspace) (void)hipFree(workspace);
    if (row_values) (void)hipFree(row_values);
    if (scratch) (void)hipFree(scratch);
  }
};

namespace arc {

// Work goes to the context's device whatever the caller's current one is.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    if (hipGetDevice(&before_) == hipSuccess && before_ != device) {
      changed_ = true;
      (void)hipSetDevice(device);
    }
  }
  ~OnDevice() {
    if (changed_) (void)hipSetDevice(before_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;

 private:
  int before_ = 0;
  bool changed_ = false;
};

struct Range {
  const void* p;
  int64_t bytes;
};

inline bool overlap(const Range& a, const Range& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes <= 0 || b.bytes <= 0) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  return pa < pb + static_cast<uintptr_t>(b.bytes) && pb < pa + static_cast<uintptr_t>(a.bytes);
}

// Whether an output overlaps another one or an input.
inline bool any_overlap(std::initializer_list<Range> outputs, std::initializer_list<Range> inputs) {
  for (const Range* a = outputs.begin(); a != outputs.end(); ++a) {
    for (const Range* b = a + 1; b != outputs.end(); ++b)
      if (overlap(*a, *b)) return true;
    for (const Range& b : inputs)
      if (overlap(*a, b)) return true;
  }
  return false;
}

inline bool finite(float v) { return std::isfinite(v); }

template <typename T>
arc_status device_copy(T** to, const std::vector<T>& from, const char* what) {
  const size_t bytes = std::max<size_t>(from.size(), 1) * sizeof(T);
  hipError_t e = hipMalloc(reinterpret_cast<void**>(to), bytes);
  if (e != hipSuccess) {
    *to = nullptr;
    (void)hipGetLastError();
    return arc::fail_hip(e, what);
  }
  if (!from.empty())
    ARC_HIP(hipMemcpy(*to, from.data(), from.size() * sizeof(T), hipMemcpyHostToDevice), what);
  return ARC_OK;
}

inline int64_t row_bytes(const arc_tokens* c, int64_t rows, int64_t stride) {
  return rows <= 0 ? 0 : ((rows - 1) * stride + c->vocab) * (c->bf16 ? 2 : 4);
}

inline arc_status check_rows(const arc_tokens* c, int64_t rows, const void* logits, int64_t stride) {
  if (c == nullptr) return fail(ARC_ERR_INVALID, "ctx is NULL");
  if (rows < 0 || rows > c->max_rows) return fail(ARC_ERR_INVALID, "rows must be in 0..max_rows");
  if (rows > 0 && logits == nullptr) return fail(ARC_ERR_INVALID, "logits is NULL");
  if (stride < c->vocab) return fail(ARC_ERR_INVALID, "stride must be at least vocab");
  if (stride > INT64_MAX / 8 / std::max<int64_t>(rows, 1))
    return fail(ARC_ERR_INVALID, "rows * stride overflows");
  return ARC_OK;
}

inline TokenArgs token_args(const arc_tokens* c, int64_t rows, const void* logits, int64_t stride,
                          const int64_t* targets) {
  TokenArgs a;
  a.logits = logits;
  a.targets = targets;
  a.rows = rows;
  a.stride = stride;
  a.vocab = c->vocab;
  a.scale = c->scale;
  a.bf16 = c->bf16;
  a.top = c->top;
  return a;
}

inline arc_status check_score(const arc_tokens* c, int64_t rows, const void* logits, int64_t stride,
                       const int64_t* targets, const TokenScores& out) {
  if (rows > 0 && out.logp != nullptr && targets == nullptr)
    return fail(ARC_ERR_INVALID, "logp needs targets");
  if ((out.top_ids == nullptr) != (out.top_logp == nullptr))
    return fail(ARC_ERR_INVALID, "top_ids and top_logp are given together");
  const int64_t v = rows * 4, k = v * c->top;
  if (any_overlap({{out.logp, v}, {out.entropy, v}, {out.lse, v}, {out.top_ids, k},
                   {out.top_logp, k}},
                  {{logits, row_bytes(c, rows, stride)}, {targets, rows * 8}}))
    return fail(ARC_ERR_INVALID, "outputs must not overlap one another or the inputs");
  return ARC_OK;
}

inline arc_status check_grad(const arc_tokens* c, int64_t rows, const void* logits, int64_t stride,
                      const int64_t* targets, const TokenGrad& g) {
  if (rows > 0 && g.grad == nullptr) return fail(ARC_ERR_INVALID, "grad is NULL");
  if (g.stride < c->vocab) return fail(ARC_ERR_INVALID, "grad_stride must be at least vocab");
  if (g.stride > INT64_MAX / 8 / std::max<int64_t>(rows, 1))
    return fail(ARC_ERR_INVALID, "rows * grad_stride overflows");
  if (rows > 0 && g.d_logp != nullptr && targets == nullptr)
    return fail(ARC_ERR_INVALID, "d_logp needs targets");
  const int64_t v = rows * 4;
  const bool in_place = g.grad == logits && g.stride == stride;
  if (any_overlap({{g.grad, row_bytes(c, rows, g.stride)}},
                  {{in_place ? nullptr : logits, row_bytes(c, rows, stride)}, {targets, rows * 8},
                   {g.lse, v}, {g.entropy, v}, {g.d_logp, v}, {g.d_entropy, v}, {g.d_lse, v}}))
    return fail(ARC_ERR_INVALID,
                "grad must not overlap the inputs (unless it is the logits themselves)");
  return ARC_OK;
}

}  // namespace arc
