// Host side of the training objectives: argument checks and the enqueue on the
// token context's stream.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "arc_context.h"
#include "arc_objective.h"
#include "arc_train.h"
#include "arc_train_host.h"

static_assert(ARC_POLICY_TOTALS == arc::kPolicyTotals, "one layout of totals");
static_assert(ARC_PREFERENCE_TOTALS == arc::kPreferenceTotals, "one layout of totals");

namespace {

using arc::any_overlap;
using arc::check_grad;
using arc::check_rows;
using arc::check_score;
using arc::fail;
using arc::finite;
using arc::OnDevice;
using arc::Range;
using arc::row_bytes;
using arc::token_args;

arc_status check_count(const arc_tokens* c, int64_t rows) {
  if (c == nullptr) return fail(ARC_ERR_INVALID, "ctx is NULL");
  if (rows < 0 || rows > c->max_rows) return fail(ARC_ERR_INVALID, "rows must be in 0..max_rows");
  return ARC_OK;
}

// ---------------------------------------------------------------- policy

arc_status check_policy(const arc_policy_config* cfg, int64_t rows, const int64_t* targets,
                        const float* ref_logp, const float* advantages, const float* totals) {
  if (cfg == nullptr) return fail(ARC_ERR_INVALID, "config is NULL");
  if (!(cfg->clip_low >= 0.f && cfg->clip_low <= 1.f))
    return fail(ARC_ERR_INVALID, "clip_low must be in 0..1");
  if (!(cfg->clip_high >= 0.f)) return fail(ARC_ERR_INVALID, "clip_high must be >= 0");
  if (cfg->dual != 0.f && (!(cfg->dual >= 1.f) || !finite(cfg->dual)))
    return fail(ARC_ERR_INVALID, "dual must be 0 or finite and at least 1");
  if (!(cfg->kl >= 0.f) || !finite(cfg->kl))
    return fail(ARC_ERR_INVALID, "kl must be finite and >= 0");
  if (!finite(cfg->entropy)) return fail(ARC_ERR_INVALID, "entropy must be finite");
  if (!finite(cfg->scale)) return fail(ARC_ERR_INVALID, "scale must be finite");
  if (totals == nullptr) return fail(ARC_ERR_INVALID, "totals is NULL");
  if (rows > 0 && (targets == nullptr || advantages == nullptr))
    return fail(ARC_ERR_INVALID, "targets and advantages must be non-NULL");
  if (rows > 0 && cfg->kl != 0.f && ref_logp == nullptr)
    return fail(ARC_ERR_INVALID, "kl needs ref_logp");
  return ARC_OK;
}

// So many rows have their terms and totals from the kernel that holds them, which costs a
// count of arrivals in one place, 16 ns a row, and saves a launch.  us, a launch of
// its own / inside: 8 rows of 1001 bf16 8.3 / 6.6, 64 of 50,257 bf16 14.7 / 12.1, 128 of
// 1001 8.5 / 8.2, 128 of 32,000 binary32 13.1 / 11.4, 200 of 1001 8.6 / 9.6, 512 of 50,257
// 25.0 / 28.1; called from Python one after the other 18.8 / 16.1.
constexpr int64_t kRowsInside = 128;
static_assert(kRowsInside <= arc::kTotalsGroups, "a place for each row");

arc::PolicyArgs policy_args(const arc_policy_config* cfg, const float* old_logp,
                            const float* ref_logp, const float* advantages,
                            const float* weights) {
  arc::PolicyArgs p;
  p.old_logp = old_logp;
  p.ref_logp = ref_logp;
  p.advantages = advantages;
  p.weights = weights;
  p.low = 1.f - cfg->clip_low;
  p.high = 1.f + cfg->clip_high;
  p.dual = cfg->dual;
  p.kl = cfg->kl;
  p.entropy = cfg->entropy;
  p.scale = cfg->scale;
  return p;
}

// ---------------------------------------------------------------- preference

constexpr int64_t kMaxPairs = int64_t{1} << 30;

arc_status check_preference(const arc_preference_config* cfg, int64_t rows,
                            const int64_t* targets, int64_t pairs, const int64_t* offsets,
                            const float* totals) {
  if (cfg == nullptr) return fail(ARC_ERR_INVALID, "config is NULL");
  if (cfg->kind != ARC_PREFERENCE_SIGMOID && cfg->kind != ARC_PREFERENCE_HINGE &&
      cfg->kind != ARC_PREFERENCE_SQUARED)
    return fail(ARC_ERR_INVALID, "kind must be an arc_preference");
  if (cfg->average != 0 && cfg->average != 1)
    return fail(ARC_ERR_INVALID, "average must be 0 or 1");
  if (!(cfg->beta >= 0x1p-20f && cfg->beta <= 0x1p20f))
    return fail(ARC_ERR_INVALID, "beta must be in 2^-20..2^20");
  if (!finite(cfg->margin)) return fail(ARC_ERR_INVALID, "margin must be finite");
  if (!(cfg->smoothing >= 0.f && cfg->smoothing <= 0.5f) ||
      (cfg->smoothing != 0.f && cfg->kind != ARC_PREFERENCE_SIGMOID))
    return fail(ARC_ERR_INVALID, "smoothing must be in 0..1/2, and 0 but for the sigmoid");
  if (!finite(cfg->scale)) return fail(ARC_ERR_INVALID, "scale must be finite");
  if (totals == nullptr) return fail(ARC_ERR_INVALID, "totals is NULL");
  if (pairs < 0 || pairs > kMaxPairs) return fail(ARC_ERR_INVALID, "pairs must be in 0..2^30");
  if (rows > 0 && targets == nullptr) return fail(ARC_ERR_INVALID, "targets is NULL");
  if (pairs > 0 && offsets == nullptr) return fail(ARC_ERR_INVALID, "offsets is NULL");
  return ARC_OK;
}

arc::PreferenceArgs preference_args(const arc_preference_config* cfg, int64_t rows,
                                    const float* logp, const int64_t* targets, int64_t pairs,
                                    const int64_t* offsets, const float* ref_logp,
                                    const float* weights) {
  arc::PreferenceArgs a;
  a.logp = logp;
  a.ref_logp = ref_logp;
  a.targets = targets;
  a.offsets = offsets;
  a.weights = weights;
  a.rows = rows;
  a.pairs = pairs;
  a.kind = cfg->kind;
  a.average = cfg->average;
  a.beta = cfg->beta;
  a.margin = cfg->margin;
  a.smoothing = cfg->smoothing;
  a.scale = cfg->scale;
  return a;
}

arc_status overlapping() {
  return fail(ARC_ERR_INVALID, "outputs must not overlap one another or the inputs");
}

}  // namespace

extern "C" {

arc_status arc_tokens_policy(arc_tokens* c, const arc_policy_config* cfg, int64_t rows,
                             const void* logits, int64_t stride, const int64_t* targets,
                             const float* old_logp, const float* ref_logp,
                             const float* advantages, const float* weights, float* logp,
                             float* entropy, float* lse, float* loss, float* ratio, float* kl,
                             float* totals, void* grad, int64_t grad_stride) {
  arc_status st = check_rows(c, rows, logits, stride);
  if (st != ARC_OK) return st;
  arc::TokenScores out{logp, entropy, lse, nullptr, nullptr};
  arc::TokenGrad g;
  g.grad = grad;
  g.stride = grad_stride;
  if ((st = check_policy(cfg, rows, targets, ref_logp, advantages, totals)) != ARC_OK ||
      (st = check_score(c, rows, logits, stride, targets, out)) != ARC_OK ||
      (st = check_grad(c, rows, logits, stride, targets, g)) != ARC_OK)
    return st;
  const int64_t v = rows * 4;
  const Range of_grad{grad, row_bytes(c, rows, grad_stride)};
  if (any_overlap({{logp, v}, {entropy, v}, {lse, v}, {loss, v}, {ratio, v}, {kl, v},
                   {totals, 4 * ARC_POLICY_TOTALS}},
                  {{logits, row_bytes(c, rows, stride)}, {targets, rows * 8}, {old_logp, v},
                   {ref_logp, v}, {advantages, v}, {weights, v}, of_grad}) ||
      any_overlap({of_grad}, {{old_logp, v}, {ref_logp, v}, {advantages, v}, {weights, v}}))
    return overlapping();
  const OnDevice here(c->device);
  const arc::TokenArgs a = token_args(c, rows, logits, stride, targets);
  const arc::PolicyArgs p = policy_args(cfg, old_logp, ref_logp, advantages, weights);
  if (out.logp == nullptr) out.logp = c->logps();
  if (out.entropy == nullptr) out.entropy = c->entropies();
  const arc::PolicyRows r{out.logp, out.entropy, targets, rows};
  arc::PolicyOutputs terms{loss, ratio, kl, nullptr, nullptr, totals};
  hipError_t e;
  arc::PolicyRowTerms inside;
  if (rows <= kRowsInside)
    inside = {loss, ratio, kl, totals, c->scratch, static_cast<uint32_t>(rows)};
  if (arc::launch_token_loss(a, out, g, c->stream, &e, &p, &inside)) {
    ARC_HIP(e, "policy loss launch");
    if (inside.rows > 0) return ARC_OK;
    ARC_HIP(arc::launch_policy_terms(p, r, terms, c->scratch, c->stream), "policy terms launch");
    return ARC_OK;
  }
  out.sums = c->row_values;
  terms.d_logp = c->d_logps();
  if (cfg->entropy != 0.f) terms.d_entropy = c->d_entropies();
  g.sums = out.sums;
  g.entropy = out.entropy;
  g.d_logp = terms.d_logp;
  g.d_entropy = terms.d_entropy;
  ARC_HIP(arc::launch_token_score(a, out, c->workspace, c->stream), "token score launch");
  ARC_HIP(arc::launch_policy_terms(p, r, terms, c->scratch, c->stream), "policy terms launch");
  ARC_HIP(arc::launch_token_grad(a, g, c->stream), "token gradient launch");
  return ARC_OK;
}

arc_status arc_tokens_policy_terms(arc_tokens* c, const arc_policy_config* cfg, int64_t rows,
                                   const float* logp, const float* entropy,
                                   const int64_t* targets, const float* old_logp,
                                   const float* ref_logp, const float* advantages,
                                   const float* weights, float* loss, float* ratio, float* kl,
                                   float* totals, float* d_logp, float* d_entropy) {
  arc_status st = check_count(c, rows);
  if (st != ARC_OK ||
      (st = check_policy(cfg, rows, targets, ref_logp, advantages, totals)) != ARC_OK)
    return st;
  if (rows > 0 && logp == nullptr) return fail(ARC_ERR_INVALID, "logp is NULL");
  if (rows > 0 && cfg->entropy != 0.f && entropy == nullptr)
    return fail(ARC_ERR_INVALID, "the coefficient of entropy needs entropy");
  const int64_t v = rows * 4;
  if (any_overlap({{loss, v}, {ratio, v}, {kl, v}, {d_logp, v}, {d_entropy, v},
                   {totals, 4 * ARC_POLICY_TOTALS}},
                  {{logp, v}, {entropy, v}, {targets, rows * 8}, {old_logp, v}, {ref_logp, v},
                   {advantages, v}, {weights, v}}))
    return overlapping();
  const OnDevice here(c->device);
  ARC_HIP(arc::launch_policy_terms(policy_args(cfg, old_logp, ref_logp, advantages, weights),
                                   {logp, entropy, targets, rows},
                                   {loss, ratio, kl, d_logp, d_entropy, totals}, c->scratch,
                                   c->stream),
          "policy terms launch");
  return ARC_OK;
}

arc_status arc_tokens_preference(arc_tokens* c, const arc_preference_config* cfg, int64_t rows,
                                 const void* logits, int64_t stride, const int64_t* targets,
                                 int64_t pairs, const int64_t* offsets, const float* ref_logp,
                                 const float* weights, float* logp, float* entropy, float* lse,
                                 float* loss, float* rewards, float* totals, void* grad,
                                 int64_t grad_stride) {
  arc_status st = check_rows(c, rows, logits, stride);
  if (st != ARC_OK) return st;
  arc::TokenScores out{logp, entropy, lse, nullptr, nullptr};
  arc::TokenGrad g;
  g.grad = grad;
  g.stride = grad_stride;
  if ((st = check_preference(cfg, rows, targets, pairs, offsets, totals)) != ARC_OK ||
      (st = check_score(c, rows, logits, stride, targets, out)) != ARC_OK ||
      (st = check_grad(c, rows, logits, stride, targets, g)) != ARC_OK)
    return st;
  const int64_t v = rows * 4, q = pairs * 4, o = pairs > 0 ? (2 * pairs + 1) * 8 : 0;
  const Range of_grad{grad, row_bytes(c, rows, grad_stride)};
  if (any_overlap({{logp, v}, {entropy, v}, {lse, v}, {loss, q}, {rewards, 2 * q},
                   {totals, 4 * ARC_PREFERENCE_TOTALS}},
                  {{logits, row_bytes(c, rows, stride)}, {targets, rows * 8}, {offsets, o},
                   {ref_logp, v}, {weights, q}, of_grad}) ||
      any_overlap({of_grad}, {{offsets, o}, {ref_logp, v}, {weights, q}}))
    return overlapping();
  const OnDevice here(c->device);
  const arc::TokenArgs a = token_args(c, rows, logits, stride, targets);
  if (out.logp == nullptr) out.logp = c->logps();
  out.sums = c->row_values;
  g.sums = out.sums;
  g.d_logp = c->d_logps();
  ARC_HIP(arc::launch_token_score(a, out, c->workspace, c->stream), "token score launch");
  ARC_HIP(arc::launch_preference(
              preference_args(cfg, rows, out.logp, targets, pairs, offsets, ref_logp, weights),
              {loss, rewards, c->d_logps(), totals}, c->scratch, c->stream),
          "preference launch");
  ARC_HIP(arc::launch_token_grad(a, g, c->stream), "token gradient launch");
  return ARC_OK;
}

arc_status arc_tokens_preference_terms(arc_tokens* c, const arc_preference_config* cfg,
                                       int64_t rows, const float* logp, const int64_t* targets,
                                       int64_t pairs, const int64_t* offsets,
                                       const float* ref_logp, const float* weights, float* loss,
                                       float* rewards, float* totals, float* d_logp) {
  arc_status st = check_count(c, rows);
  if (st != ARC_OK ||
      (st = check_preference(cfg, rows, targets, pairs, offsets, totals)) != ARC_OK)
    return st;
  if (rows > 0 && logp == nullptr) return fail(ARC_ERR_INVALID, "logp is NULL");
  const int64_t v = rows * 4, q = pairs * 4, o = pairs > 0 ? (2 * pairs + 1) * 8 : 0;
  if (any_overlap({{loss, q}, {rewards, 2 * q}, {d_logp, v}, {totals, 4 * ARC_PREFERENCE_TOTALS}},
                  {{logp, v}, {targets, rows * 8}, {offsets, o}, {ref_logp, v}, {weights, q}}))
    return overlapping();
  const OnDevice here(c->device);
  ARC_HIP(arc::launch_preference(
              preference_args(cfg, rows, logp, targets, pairs, offsets, ref_logp, weights),
              {loss, rewards, d_logp, totals}, c->scratch, c->stream),
          "preference launch");
  return ARC_OK;
}

}  // extern "C"
