// Host side of the training operators: argument checks, the contexts' tables
// and workspace, and the enqueue on the context's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "arc_context.h"
#include "arc_train.h"
#include "arc_train_host.h"

static_assert(arc::kStateBlock == ARC_STATE_BLOCK, "one block size");

struct arc_optim {
  std::vector<arc::OptimTensor> tensors;
  std::vector<int32_t> chunk_tensor, norm_tensor;  // of each run of elements
  int64_t state_elems = 0;
  int32_t optim_run = arc::kOptimChunkMost, norm_run = arc::kNormChunkMost;
  bool cached = false;  // a step's bytes are few enough to be stored through the caches
  int32_t state = ARC_STATE_F32, stochastic = 0;
  bool any_param_bf16 = false;
  uint64_t seed = 0;
  hipStream_t stream = nullptr;
  int device = 0;
  arc::OptimTensor* tensors_dev = nullptr;
  int32_t *chunk_tensor_dev = nullptr, *norm_tensor_dev = nullptr;
  double* partial_dev = nullptr;  // a sum of squares of each run
  double* squares_dev = nullptr;  // of each tensor, and the count of those done
  uint32_t* arrived() const { return reinterpret_cast<uint32_t*>(squares_dev + tensors.size()); }

  void release() {
    (void)hipStreamSynchronize(stream);
    for (void* p : {static_cast<void*>(tensors_dev), static_cast<void*>(chunk_tensor_dev),
                    static_cast<void*>(norm_tensor_dev), static_cast<void*>(partial_dev),
                    static_cast<void*>(squares_dev)})
      if (p) (void)hipFree(p);
  }
};

namespace {

using arc::any_overlap;
using arc::check_grad;
using arc::check_rows;
using arc::check_score;
using arc::device_copy;
using arc::fail;
using arc::finite;
using arc::OnDevice;
using arc::overlap;
using arc::row_bytes;
using arc::token_args;

// ---------------------------------------------------------------- optimizer

uint64_t splitmix64(uint64_t seed, uint64_t number) {
  uint64_t z = seed + (number + 1) * 0x9E3779B97F4A7C15ull;
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

// Bytes of a step with 32-bit states up to which it stores through the caches.
constexpr int64_t kCachedBytes = 800000000;
constexpr int64_t kMaxElements = int64_t{1} << 42;
// Workgroups of one launch: their threads stay below 2^32.
constexpr int64_t kMaxGroups = int64_t{1} << 23;

arc_status check_optim(const arc_optim_config* cfg) {
  if (cfg == nullptr) return fail(ARC_ERR_INVALID, "cfg is NULL");
  if (cfg->tensors == nullptr) return fail(ARC_ERR_INVALID, "tensors is NULL");
  if (cfg->num_tensors < 1 || cfg->num_tensors > (1 << 20))
    return fail(ARC_ERR_INVALID, "num_tensors must be in 1..2^20");
  if (cfg->state != ARC_STATE_F32 && cfg->state != ARC_STATE_F8)
    return fail(ARC_ERR_INVALID, "state must be ARC_STATE_F32 or ARC_STATE_F8");
  if (cfg->stochastic != 0 && cfg->stochastic != 1)
    return fail(ARC_ERR_INVALID, "stochastic must be 0 or 1");
  if (cfg->reserved != 0) return fail(ARC_ERR_INVALID, "reserved must be 0");
  int64_t left = kMaxElements;
  for (int32_t i = 0; i < cfg->num_tensors; ++i) {
    const arc_optim_tensor& t = cfg->tensors[i];
    if (t.count < 0 || t.count > left)
      return fail(ARC_ERR_INVALID, "counts must be >= 0 and 2^42 at most in all");
    left -= t.count;
    for (int32_t dt : {t.param_dtype, t.grad_dtype})
      if (dt != ARC_DTYPE_F32 && dt != ARC_DTYPE_BF16)
        return fail(ARC_ERR_INVALID, "dtypes must be ARC_DTYPE_F32 or ARC_DTYPE_BF16");
    if (!(t.weight_decay >= 0.f) || !finite(t.weight_decay) || !(t.lr_scale >= 0.f) ||
        !finite(t.lr_scale))
      return fail(ARC_ERR_INVALID, "weight_decay and lr_scale must be >= 0 and finite");
  }
  return ARC_OK;
}

// The tables of a checked configuration (may throw std::bad_alloc).
void plan_optim(const arc_optim_config* cfg, arc_optim* c) {
  c->tensors.reserve(static_cast<size_t>(cfg->num_tensors));
  const auto runs = [](int64_t count, int64_t of) {
    return static_cast<size_t>((count + of - 1) / of);
  };
  int64_t all = 0;
  for (int32_t i = 0; i < cfg->num_tensors; ++i) all += cfg->tensors[i].count;
  // Enough runs to fill the card, and few enough for the second launch (a
  // ResNet-18's 1.1e7 values in runs of 32,768: 20.2 us).
  while (c->norm_run > arc::kNormChunkLeast && all / c->norm_run < 4096) c->norm_run /= 2;
  while (c->optim_run > arc::kOptimChunkLeast && all / c->optim_run < 2048) c->optim_run /= 2;
  c->cached = all * 28 <= kCachedBytes;
  size_t chunks = 0, norms = 0;
  for (int32_t i = 0; i < cfg->num_tensors; ++i) {
    chunks += runs(cfg->tensors[i].count, c->optim_run);
    norms += runs(cfg->tensors[i].count, c->norm_run);
  }
  c->chunk_tensor.reserve(chunks);
  c->norm_tensor.reserve(norms);
  for (int32_t i = 0; i < cfg->num_tensors; ++i) {
    const arc_optim_tensor& in = cfg->tensors[i];
    arc::OptimTensor t{};
    t.count = in.count;
    t.state = c->state_elems;
    t.weight_decay = in.weight_decay;
    t.lr_scale = in.lr_scale;
    t.first_chunk = static_cast<int32_t>(c->chunk_tensor.size());
    t.first_norm = static_cast<int32_t>(c->norm_tensor.size());
    t.param_bf16 = in.param_dtype == ARC_DTYPE_BF16;
    t.grad_bf16 = in.grad_dtype == ARC_DTYPE_BF16;
    c->any_param_bf16 = c->any_param_bf16 || t.param_bf16;
    c->tensors.push_back(t);
    c->state_elems += (in.count + arc::kStateBlock - 1) / arc::kStateBlock * arc::kStateBlock;
    c->chunk_tensor.insert(c->chunk_tensor.end(), runs(in.count, c->optim_run), i);
    c->norm_tensor.insert(c->norm_tensor.end(), runs(in.count, c->norm_run), i);
  }
  c->state = cfg->state;
  c->stochastic = cfg->stochastic;
  c->seed = cfg->seed;
}

// Calls launch(batch, tensors) for batches of at most `tensors` tensors and
// kMaxGroups runs that together hold every run once.
template <typename Launch>
arc_status each_batch(const arc_optim* c, int32_t tensors, const std::vector<int32_t>& runs,
                      const int32_t* runs_dev, int32_t arc::OptimTensor::*first_run,
                      const Launch& launch) {
  const auto num = static_cast<int32_t>(c->tensors.size());
  const auto all = static_cast<int64_t>(runs.size());
  for (int32_t first = 0; first < num; first += tensors) {
    const int32_t next = std::min(num, first + tensors);
    const int64_t end = next < num ? c->tensors[static_cast<size_t>(next)].*first_run : all;
    for (int64_t at = c->tensors[static_cast<size_t>(first)].*first_run; at < end;
         at += kMaxGroups) {
      arc::OptimBatch b;
      b.tensors = c->tensors_dev;
      b.chunk_tensor = runs_dev;
      b.first = first;
      b.first_chunk = static_cast<int32_t>(at);
      b.chunks = static_cast<int32_t>(std::min(end - at, kMaxGroups));
      const arc_status st = launch(b, next - first);
      if (st != ARC_OK) return st;
    }
  }
  return ARC_OK;
}

arc_status check_pointers(const arc_optim* c, const void* const* p, const char* what) {
  if (p == nullptr) return fail(ARC_ERR_INVALID, std::string(what) + " is NULL");
  for (size_t i = 0; i < c->tensors.size(); ++i)
    if (p[i] == nullptr && c->tensors[i].count > 0)
      return fail(ARC_ERR_INVALID, std::string(what) + " holds a NULL");
  return ARC_OK;
}

}  // namespace

extern "C" {

arc_status arc_tokens_create(const arc_tokens_config* cfg, void* hip_stream, arc_tokens** out) {
  if (out == nullptr) return fail(ARC_ERR_INVALID, "out is NULL");
  *out = nullptr;
  if (cfg == nullptr) return fail(ARC_ERR_INVALID, "cfg is NULL");
  if (cfg->vocab < 1 || cfg->vocab > INT32_MAX)
    return fail(ARC_ERR_INVALID, "vocab must be in 1..2^31-1");
  if (cfg->max_rows < 1 || cfg->max_rows > INT32_MAX)
    return fail(ARC_ERR_INVALID, "max_rows must be in 1..2^31-1");
  if (cfg->dtype != ARC_DTYPE_F32 && cfg->dtype != ARC_DTYPE_BF16)
    return fail(ARC_ERR_INVALID, "dtype must be ARC_DTYPE_F32 or ARC_DTYPE_BF16");
  if (cfg->top < 0 || cfg->top > ARC_MAX_TOP || cfg->top > cfg->vocab)
    return fail(ARC_ERR_INVALID, "top must be in 0..min(vocab, ARC_MAX_TOP)");
  if (!(cfg->scale >= 0x1p-64f && cfg->scale <= 0x1p64f))
    return fail(ARC_ERR_INVALID, "scale must be in 2^-64..2^64");
  if (cfg->reserved != 0) return fail(ARC_ERR_INVALID, "reserved must be 0");
  arc_tokens* c = new (std::nothrow) arc_tokens();
  if (c == nullptr) return fail(ARC_ERR_NOMEM, "host allocation failed");
  c->vocab = cfg->vocab;
  c->max_rows = cfg->max_rows;
  c->bf16 = cfg->dtype == ARC_DTYPE_BF16;
  c->top = cfg->top;
  c->scale = cfg->scale;
  c->stream = static_cast<hipStream_t>(hip_stream);
  const size_t bytes = arc::token_workspace_bytes();
  hipError_t e = hipGetDevice(&c->device);
  if (e == hipSuccess) {
    e = hipMalloc(&c->workspace, bytes);
    if (e != hipSuccess) c->workspace = nullptr;
  }
  if (e == hipSuccess) {
    e = hipMalloc(reinterpret_cast<void**>(&c->row_values),
                  static_cast<size_t>(c->max_rows) * 6 * sizeof(float));
    if (e != hipSuccess) c->row_values = nullptr;
  }
  if (e == hipSuccess) {
    e = hipMalloc(reinterpret_cast<void**>(&c->scratch), sizeof(arc::ObjectiveScratch));
    if (e != hipSuccess) c->scratch = nullptr;
  }
  if (e == hipSuccess) e = hipMemset(c->scratch, 0, sizeof(arc::ObjectiveScratch));
  if (e == hipSuccess) e = hipMemset(c->workspace, 0, bytes);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipGetLastError();
    c->release();
    delete c;
    return arc::fail_hip(e, "token workspace");
  }
  *out = c;
  return ARC_OK;
}

arc_status arc_tokens_score(arc_tokens* c, int64_t rows, const void* logits, int64_t stride,
                            const int64_t* targets, float* logp, float* entropy, float* lse,
                            int32_t* top_ids, float* top_logp) {
  arc_status st = check_rows(c, rows, logits, stride);
  if (st != ARC_OK) return st;
  const arc::TokenScores out{logp, entropy, lse, top_ids, top_logp};
  if ((st = check_score(c, rows, logits, stride, targets, out)) != ARC_OK) return st;
  const OnDevice here(c->device);
  ARC_HIP(arc::launch_token_score(token_args(c, rows, logits, stride, targets), out,
                                  c->workspace, c->stream),
          "token score launch");
  return ARC_OK;
}

arc_status arc_tokens_grad(arc_tokens* c, int64_t rows, const void* logits, int64_t stride,
                           const int64_t* targets, const float* lse, const float* entropy,
                           const float* d_logp, const float* d_entropy, const float* d_lse,
                           void* grad, int64_t grad_stride) {
  arc_status st = check_rows(c, rows, logits, stride);
  if (st != ARC_OK) return st;
  if (rows > 0 && lse == nullptr) return fail(ARC_ERR_INVALID, "lse is NULL");
  if (rows > 0 && d_entropy != nullptr && entropy == nullptr)
    return fail(ARC_ERR_INVALID, "d_entropy needs entropy");
  const arc::TokenGrad g{lse, entropy, d_logp, d_entropy, d_lse, grad, grad_stride};
  if ((st = check_grad(c, rows, logits, stride, targets, g)) != ARC_OK) return st;
  const OnDevice here(c->device);
  ARC_HIP(arc::launch_token_grad(token_args(c, rows, logits, stride, targets), g, c->stream),
          "token gradient launch");
  return ARC_OK;
}

arc_status arc_tokens_loss(arc_tokens* c, int64_t rows, const void* logits, int64_t stride,
                           const int64_t* targets, const float* d_logp, const float* d_entropy,
                           const float* d_lse, float* logp, float* entropy, float* lse,
                           void* grad, int64_t grad_stride) {
  arc_status st = check_rows(c, rows, logits, stride);
  if (st != ARC_OK) return st;
  arc::TokenScores out{logp, entropy, lse, nullptr, nullptr};
  arc::TokenGrad g{lse, entropy, d_logp, d_entropy, d_lse, grad, grad_stride};
  if ((st = check_score(c, rows, logits, stride, targets, out)) != ARC_OK ||
      (st = check_grad(c, rows, logits, stride, targets, g)) != ARC_OK)
    return st;
  if (any_overlap({{logp, rows * 4}, {entropy, rows * 4}, {lse, rows * 4}},
                  {{d_logp, rows * 4}, {d_entropy, rows * 4}, {d_lse, rows * 4},
                   {grad, row_bytes(c, rows, grad_stride)}}))
    return fail(ARC_ERR_INVALID, "outputs must not overlap one another or the inputs");
  const OnDevice here(c->device);
  const arc::TokenArgs a = token_args(c, rows, logits, stride, targets);
  hipError_t e;
  if (arc::launch_token_loss(a, out, g, c->stream, &e)) {
    ARC_HIP(e, "token loss launch");
    return ARC_OK;
  }
  out.sums = c->row_values;
  if (entropy == nullptr) out.entropy = c->entropies();
  g.sums = out.sums;
  g.entropy = out.entropy;
  ARC_HIP(arc::launch_token_score(a, out, c->workspace, c->stream), "token score launch");
  ARC_HIP(arc::launch_token_grad(a, g, c->stream), "token gradient launch");
  return ARC_OK;
}

arc_status arc_tokens_destroy(arc_tokens* c) {
  if (c == nullptr) return ARC_OK;
  c->release();
  delete c;
  return ARC_OK;
}

arc_status arc_optim_create(const arc_optim_config* cfg, void* hip_stream, arc_optim** out) {
  if (out == nullptr) return fail(ARC_ERR_INVALID, "out is NULL");
  *out = nullptr;
  arc_status st = check_optim(cfg);
  if (st != ARC_OK) return st;
  arc_optim* c = new (std::nothrow) arc_optim();
  if (c == nullptr) return fail(ARC_ERR_NOMEM, "host allocation failed");
  try {
    plan_optim(cfg, c);
  } catch (const std::exception&) {
    delete c;
    return fail(ARC_ERR_NOMEM, "host allocation failed");
  }
  c->stream = static_cast<hipStream_t>(hip_stream);
  const auto bail = [&](arc_status s) {
    c->release();
    delete c;
    return s;
  };
  hipError_t e = hipGetDevice(&c->device);
  if (e != hipSuccess) return bail(arc::fail_hip(e, "hipGetDevice"));
  if ((st = device_copy(&c->tensors_dev, c->tensors, "optimizer tables")) != ARC_OK ||
      (st = device_copy(&c->chunk_tensor_dev, c->chunk_tensor, "optimizer tables")) != ARC_OK ||
      (st = device_copy(&c->norm_tensor_dev, c->norm_tensor, "optimizer tables")) != ARC_OK)
    return bail(st);
  const auto room = [&](double** p, size_t count) {
    e = hipMalloc(reinterpret_cast<void**>(p), std::max<size_t>(count, 1) * sizeof(double));
    if (e != hipSuccess) *p = nullptr;
    return e == hipSuccess;
  };
  if (room(&c->partial_dev, c->norm_tensor.size()) &&
      room(&c->squares_dev, c->tensors.size() + 1))
    e = hipMemset(c->arrived(), 0, sizeof(double));
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return bail(arc::fail_hip(e, "optimizer workspace"));
  }
  *out = c;
  return ARC_OK;
}

int64_t arc_optim_state_elems(const arc_optim* c) { return c ? c->state_elems : -1; }

int64_t arc_optim_state_offset(const arc_optim* c, int32_t i) {
  if (c == nullptr || i < 0 || static_cast<size_t>(i) >= c->tensors.size()) return -1;
  return c->tensors[static_cast<size_t>(i)].state;
}

arc_status arc_optim_norm(arc_optim* c, const void* const* grads, float scale, float max_norm,
                          float* norms, float* total) {
  if (c == nullptr) return fail(ARC_ERR_INVALID, "ctx is NULL");
  arc_status st = check_pointers(c, grads, "grads");
  if (st != ARC_OK) return st;
  if (total == nullptr) return fail(ARC_ERR_INVALID, "total is NULL");
  if (!(scale >= 0.f) || !finite(scale)) return fail(ARC_ERR_INVALID, "scale must be finite, >= 0");
  if (!(max_norm > 0.f)) return fail(ARC_ERR_INVALID, "max_norm must be > 0");
  const auto num = static_cast<int32_t>(c->tensors.size());
  if (overlap({norms, int64_t{4} * num}, {total, 8}))
    return fail(ARC_ERR_INVALID, "norms and total must not overlap");
  const OnDevice here(c->device);
  st = each_batch(c, arc::kNormBatch, c->norm_tensor, c->norm_tensor_dev,
                  &arc::OptimTensor::first_norm,
                  [&](const arc::OptimBatch& b, int32_t count) -> arc_status {
                    arc::NormPointers p;
                    std::copy(grads + b.first, grads + b.first + count, p.grad);
                    ARC_HIP(arc::launch_norm_chunks(b, p, c->norm_run, c->partial_dev, c->stream),
                            "norm launch");
                    return ARC_OK;
                  });
  if (st != ARC_OK) return st;
  ARC_HIP(arc::launch_norm_tensors(c->tensors_dev, num, c->norm_run, c->partial_dev, c->squares_dev,
                                   c->arrived(), scale, max_norm, norms, total, c->stream),
          "norm launch");
  return ARC_OK;
}

arc_status arc_optim_adamw(arc_optim* c, const arc_adamw_config* ac, int64_t t,
                           void* const* params, const void* const* grads, void* const* copies,
                           const float* factor, void* m, void* v, float* m_scale,
                           float* v_scale) {
  if (c == nullptr) return fail(ARC_ERR_INVALID, "ctx is NULL");
  if (ac == nullptr) return fail(ARC_ERR_INVALID, "config is NULL");
  if (t < 0) return fail(ARC_ERR_INVALID, "t must be >= 0");
  if (!finite(ac->lr)) return fail(ARC_ERR_INVALID, "lr must be finite");
  if (!(ac->beta1 >= 0.f && ac->beta1 < 1.f) || !(ac->beta2 >= 0.f && ac->beta2 < 1.f))
    return fail(ARC_ERR_INVALID, "beta1 and beta2 must be in [0, 1)");
  if (!(ac->eps >= FLT_MIN) || !finite(ac->eps))
    return fail(ARC_ERR_INVALID, "eps must be finite and at least 2^-126");
  arc_status st;
  if ((st = check_pointers(c, params, "params")) != ARC_OK ||
      (st = check_pointers(c, grads, "grads")) != ARC_OK)
    return st;
  const bool f8 = c->state == ARC_STATE_F8;
  if (c->state_elems > 0 && (m == nullptr || v == nullptr || (f8 && (!m_scale || !v_scale))))
    return fail(ARC_ERR_INVALID, "the states must be non-NULL");
  if (!f8 && (m_scale != nullptr || v_scale != nullptr))
    return fail(ARC_ERR_INVALID, "scales are for ARC_STATE_F8");
  for (const void* p : {m, v, static_cast<void*>(m_scale), static_cast<void*>(v_scale)})
    if (reinterpret_cast<uintptr_t>(p) % 16)
      return fail(ARC_ERR_INVALID, "the states must be 16-byte aligned");
  const int64_t state_bytes = c->state_elems * (f8 ? 1 : 4);
  const int64_t scale_bytes = c->state_elems / arc::kStateBlock * 4;
  if (any_overlap({{m, state_bytes}, {v, state_bytes}, {m_scale, scale_bytes},
                   {v_scale, scale_bytes}},
                  {{factor, 4}}))
    return fail(ARC_ERR_INVALID, "the states must not overlap one another or factor");

  arc::AdamArgs a{};
  a.lr = ac->lr;
  a.beta1 = ac->beta1;
  a.beta2 = ac->beta2;
  a.one_minus_beta1 = 1.0f - ac->beta1;
  a.one_minus_beta2 = 1.0f - ac->beta2;
  a.eps = ac->eps;
  const double T = static_cast<double>(t) + 1.0;
  const double c1 = 1.0 - std::pow(static_cast<double>(ac->beta1), T);
  const double c2 = 1.0 - std::pow(static_cast<double>(ac->beta2), T);
  a.inv_c1 = static_cast<float>(1.0 / c1);
  a.inv_root_c2 = static_cast<float>(1.0 / std::sqrt(c2));
  const uint64_t key = splitmix64(c->seed, static_cast<uint64_t>(t));
  a.key_low = static_cast<uint32_t>(key);
  a.key_high = static_cast<uint32_t>(key >> 32);
  a.stochastic = c->stochastic && c->any_param_bf16;
  a.run = c->optim_run;
  a.factor = factor;
  a.m = m;
  a.v = v;
  a.m_scale = m_scale;
  a.v_scale = v_scale;
  const OnDevice here(c->device);
  return each_batch(c, arc::kOptimBatch, c->chunk_tensor, c->chunk_tensor_dev,
                    &arc::OptimTensor::first_chunk,
                    [&](const arc::OptimBatch& b, int32_t count) -> arc_status {
                      arc::OptimPointers p;
                      for (int32_t i = 0; i < count; ++i) {
                        p.param[i] = params[b.first + i];
                        p.grad[i] = grads[b.first + i];
                        p.copy[i] = copies ? static_cast<uint16_t*>(copies[b.first + i]) : nullptr;
                      }
                      ARC_HIP(arc::launch_adamw(f8, c->cached, b, p, a, c->stream), "AdamW launch");
                      return ARC_OK;
                    });
}

arc_status arc_optim_destroy(arc_optim* c) {
  if (c == nullptr) return ARC_OK;
  c->release();
  delete c;
  return ARC_OK;
}

}  // extern "C"
