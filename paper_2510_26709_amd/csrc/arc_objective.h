// Internal declarations of the training objectives over token log
// probabilities: the clipped policy loss and the preference loss
// (arc_objective.hip), and their host side (arc_objective.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace arc {

// ---------------------------------------------------------------- policy

// One token's inputs and what all tokens share.
struct PolicyArgs {
  const float *old_logp = nullptr, *ref_logp = nullptr;  // may be NULL
  const float* advantages = nullptr;
  const float* weights = nullptr;  // NULL: 1
  float low = 0.f, high = 0.f;     // borders of the ratio
  float dual = 0.f;                // 0: none
  float kl = 0.f, entropy = 0.f;   // coefficients
  float scale = 1.f;               // of all weights
};

struct PolicyRows {
  const float *logp = nullptr, *entropy = nullptr;  // entropy: NULL for zeros
  const int64_t* targets = nullptr;
  int64_t rows = 0;
};

struct PolicyOutputs {
  float *loss = nullptr, *ratio = nullptr, *kl = nullptr;
  float *d_logp = nullptr, *d_entropy = nullptr;
  float* totals = nullptr;  // loss, ratio, kl, entropy, clipped
};
constexpr int kPolicyTotals = 5;

struct ObjectiveScratch;

// For the kernel that holds rows of logits, a workgroup each: where it puts its rows'
// terms and, the last of `rows` workgroups, their totals.  rows 0: nowhere.
struct PolicyRowTerms {
  float *loss = nullptr, *ratio = nullptr, *kl = nullptr;
  float* totals = nullptr;
  ObjectiveScratch* scratch = nullptr;
  uint32_t rows = 0;
};

// ---------------------------------------------------------------- preference

struct PreferenceArgs {
  const float* logp = nullptr;
  const float* ref_logp = nullptr;  // NULL: zeros
  const int64_t* targets = nullptr;
  const int64_t* offsets = nullptr;  // [2 pairs + 1]
  const float* weights = nullptr;    // NULL: 1
  int64_t rows = 0, pairs = 0;
  int32_t kind = 0, average = 0;
  float beta = 1.f, margin = 0.f, smoothing = 0.f, scale = 1.f;
};

struct PreferenceOutputs {
  float *loss = nullptr, *rewards = nullptr;  // may be NULL
  float* d_logp = nullptr;                    // may be NULL
  float* totals = nullptr;                    // loss, margin, preferred
};
constexpr int kPreferenceTotals = 3;

// Scratch of both in a token context: the totals of workgroups, the sums of
// parts of sequences (one a workgroup), and counts of workgroups, one for launches of
// each number of them.  A count goes round, 0 after as many arrivals as its number, so
// that it is 0 between launches whatever came before: replays that overlap in time, which
// they must not, spoil their own totals, but no later call's.
constexpr int kTotalsGroups = 1024;
struct ObjectiveScratch {
  double totals[kTotalsGroups][kPolicyTotals];
  double sum[kTotalsGroups];
  int64_t count[kTotalsGroups];
  uint32_t arrived[kTotalsGroups + 1];
};

hipError_t launch_policy_terms(const PolicyArgs& p, const PolicyRows& r, const PolicyOutputs& out,
                               ObjectiveScratch* scratch, hipStream_t stream);
hipError_t launch_preference(const PreferenceArgs& a, const PreferenceOutputs& out,
                             ObjectiveScratch* scratch, hipStream_t stream);

}  // namespace arc
