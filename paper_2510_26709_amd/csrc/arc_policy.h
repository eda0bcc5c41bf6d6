// One token's policy loss on the device: for the kernels that hold rows of logits
// (arc_tokens.hip) and the one that has their log probabilities (arc_objective.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "arc_objective.h"

namespace arc {

struct PolicyTerm {
  float loss, ratio, kl;      // of the token, not weighted
  float d_logp, d_entropy;    // weighted
  float weight;
  bool clipped;
};

// e^x - x - 1 without the difference that cancels it near 0: its series up to
// |x| = 1/2 (what is left out is 2^-28 of the value), where the plain difference
// of binary32 numbers would lose two bits and, further in, all.
__device__ __forceinline__ float exp_beyond_line(float x, float exp_minus_1) {
  if (!(fabsf(x) < 0.5f)) return exp_minus_1 == INFINITY ? INFINITY : exp_minus_1 - x;
  float s = 1.f / 362880.f;
  s = fmaf(s, x, 1.f / 40320.f);
  s = fmaf(s, x, 1.f / 5040.f);
  s = fmaf(s, x, 1.f / 720.f);
  s = fmaf(s, x, 1.f / 120.f);
  s = fmaf(s, x, 1.f / 24.f);
  s = fmaf(s, x, 1.f / 6.f);
  s = fmaf(s, x, 0.5f);
  return s * x * x;
}

// Token i's terms; `given`: it has a token of its own.  What a token without one
// holds, and what one of weight 0 does to sums and gradients, is left out by
// selection, not by a product, so that no infinity or NaN there gets through.
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& p, int64_t i, bool given,
                                                  float logp, float H) {
  PolicyTerm t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, false};
  if (!given) return t;
  const float A = p.advantages[i];
  t.weight = p.weights ? p.weights[i] * p.scale : p.scale;
  t.ratio = p.old_logp ? expf(logp - p.old_logp[i]) : logp != logp ? logp : 1.f;
  const float held = fminf(fmaxf(t.ratio, p.low), p.high) * A;
  float gain = t.ratio * A;
  t.clipped = gain > held;  // (a ratio that is NaN is not, and stays one)
  if (t.clipped) gain = held;
  if (p.dual != 0.f && A < 0.f && gain < p.dual * A) {
    gain = p.dual * A;
    t.clipped = true;
  }
  float d = t.clipped ? 0.f : -t.ratio * A;
  t.loss = -gain;
  if (p.ref_logp) {
    const float away = p.ref_logp[i] - logp;
    const float grown = expm1f(away);
    t.kl = exp_beyond_line(away, grown);
    if (p.kl != 0.f) {
      t.loss = fmaf(p.kl, t.kl, t.loss);
      d = fmaf(-p.kl, grown, d);
    }
  }
  if (p.entropy != 0.f) t.loss = fmaf(-p.entropy, H, t.loss);
  if (t.weight != 0.f) {
    t.d_logp = t.weight * d;
    t.d_entropy = -p.entropy * t.weight;
  }
  return t;
}

}  // namespace arc
